"""Gathered attention weight, the choice of what stays, and its move, for both kinds of pool, against plain float64 / numpy forms."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2609_34388_b200 import binding, synth
from tests import _kv4
from tests._util import f64

pytestmark = pytest.mark.gpu

POOLS = [0, binding.FLAG_KV_4BIT]
TINY, B8, B14 = (4, 2, 64), (32, 8, 128), (40, 8, 128)


def make(heads, stride, max_tokens, max_req, flags, layers=2):
    nq, nkv, d = heads
    shape = synth.ModelShape(n_layers=layers, hidden=64, n_q_heads=nq, n_kv_heads=nkv, head_dim=d, ffn=64, vocab=64)
    return binding.Context(binding.make_config(shape, max_req, max_tokens, stride, flags))


# ---- gathered weight -----------------------------------------------------------------------------------------------------
def weights_case(heads, reqs, seed, flags, corr=None, decay=0.75, row_weight="mixed", chunked=False):
    nq, nkv, d = heads
    L, v, b = (list(x) for x in zip(*reqs))
    corr = corr or [()] * len(reqs)
    desc = synth.fixed_descriptor(L, v, b, seed=seed, corr=[[(i, 5) for i in c] for c in corr], corr_block=b)
    T = desc.n_tokens
    ctx = make(heads, desc.page_table.shape[1], T, len(reqs), flags)
    pool = binding.alloc_kv_pool(ctx, desc.n_pages, fill=None)
    pool.view(torch.uint8).fill_(255)                                    # NaN wherever nothing is written
    q = synth.queries(T, nq, d, seed=seed + 5)
    ks = []
    for r, n in enumerate(desc.rows):
        k_, v_ = synth.kv_values(L[r] + int(n), nkv, d, seed=seed * 100 + r)
        ks.append(k_)
        ctx.recg_kv_write(pool, desc.n_pages, 1, desc.page_table[r], 0, k_.cuda(), v_.cuda())
    batch = binding.Batch(L, v, b, None, desc.page_table, pool, desc.n_pages, **desc.branch_kwargs())
    lse = torch.empty((T, nq), device="cuda")
    o = torch.empty((T, nq, d), dtype=torch.bfloat16, device="cuda")
    ctx.recg_attention(batch, 1, q.cuda(), o, lse)
    g = torch.Generator().manual_seed(seed)
    rw = None
    if row_weight == "mixed":                                            # a third left out, one of them with an unusable lse
        rw = torch.rand(T, generator=g) * (torch.rand(T, generator=g) > 0.33)
        if (rw == 0).any():
            lse[int((rw == 0).nonzero()[0])] = float("nan")
    before = torch.rand((2, desc.n_pages, nkv, 16), generator=g) * 3
    w_in = before.cuda()
    w_out = torch.full_like(w_in, -7.0)
    rwd = None if rw is None else rw.cuda()
    ctx.recg_kv_weights(None, 1, q.cuda(), lse, w_in, w_out, rwd, decay)
    same = w_in.clone()
    ctx.recg_kv_weights(batch, 1, q.cuda(), lse, same, same, rwd, decay)      # in place, and with the batch given
    first = torch.full_like(w_in, -7.0)
    ctx.recg_kv_weights(None, 1, q.cuda(), lse, None, first, rwd, decay)
    ctx.recg_sync()
    got, got_same, got_first = f64(w_out), f64(same), f64(first)
    touched = np.zeros(got.shape, dtype=bool)
    t = 0
    for r, n in enumerate(desc.rows):
        n = int(n)
        kv_len = L[r] + n
        see = _kv4.visible(L[r], v[r], b[r], corr[r], b[r])
        held = _kv4.values(ks[r]) if flags else f64(ks[r])
        w = np.ones(n) if rw is None else f64(rw[t:t + n])
        want, err = _kv4.gathered(f64(q[t:t + n]), held, see, f64(lse[t:t + n]), w)
        pos = np.arange(kv_len)
        page, off = desc.page_table[r][pos // 16], pos % 16
        old = np.where(pos < L[r], decay, 0.0)[:, None] * f64(before)[1, page, :, off]
        for a, total in ((got, old + want.T), (got_same, old + want.T), (got_first, want.T)):
            over = np.abs(a[1, page, :, off] - total) / (err.T + 2.0 ** -22 * np.abs(total) + 1e-30)
            assert over.max() <= 1.0, (r, over.max())
        touched[1, page, :, off] = True
        t += n
    assert (got[~touched] == -7.0).all() and (got_same[~touched] == f64(before)[~touched]).all() and (got_first[~touched] == -7.0).all()
    assert np.array_equal(got[touched], got_same[touched])
    ctx.recg_free()


@pytest.mark.parametrize("flags", POOLS)
@pytest.mark.parametrize("heads", [TINY, B8])
@pytest.mark.parametrize("reqs", [[(0, 1, 0)], [(0, 0, 1)], [(15, 1, 0)], [(16, 2, 2)], [(127, 1, 0)], [(128, 1, 0)], [(200, 16, 16)],
                                  [(100, 4, 4), (7, 1, 8), (300, 16, 16), (64, 2, 2), (0, 8, 8)]])
def test_gathered_weight(heads, reqs, flags):
    weights_case(heads, reqs, seed=11, flags=flags)
    weights_case(heads, reqs, seed=12, flags=flags, row_weight=None, decay=0.0)


@pytest.mark.parametrize("flags", POOLS)
@pytest.mark.parametrize("heads,reqs,corr", [
    (B8, [(3000, 1, 0)] + [(50 + 37 * i, 1, 0) for i in range(20)], None), (B8, [(1000, 33, 31), (5, 40, 0)], None),
    (B14, [(300, 25, 25), (0, 3, 2), (40, 1, 8)], None), (B14, [(500, 200, 0)], None), (TINY, [(2500, 40, 30)], None),
    (B8, [(100, 8, 8), (0, 5, 4), (1030, 16, 7)], [(1, 6), (4,), (3, 15)]), ((16, 1, 128), [(500, 8, 1), (40, 1, 0)], None)])
def test_gathered_weight_of_long_contexts_branches_and_groups(heads, reqs, corr, flags):
    if (heads[0] + 2 * heads[1]) * heads[2] % 128:
        pytest.skip("the context asks for a qkv width of whole 128 columns")
    weights_case(heads, reqs, seed=21, flags=flags, corr=corr, decay=1.0)


@pytest.mark.parametrize("flags", POOLS)
@pytest.mark.parametrize("heads", [TINY, B8, B14])
def test_gathered_weight_of_many_requests(heads, flags):
    """Many short requests, whose rows are staged together, and among them some whose rows alone do not fit."""
    g = np.random.default_rng(5)
    reqs = [(int(g.integers(0, 90)), int(g.integers(1, 6)), int(g.integers(0, 4))) for _ in range(120)]
    for r, n in ((0, 70), (17, 33), (18, 140), (60, 26), (119, 65)):
        reqs[r] = (reqs[r][0], n, 3)
    reqs[80] = (4000, 2, 0)
    weights_case(heads, reqs, seed=31, flags=flags)
    weights_case(heads, reqs[:40], seed=32, flags=flags, row_weight=None, decay=0.5)


def test_weights_add_up_to_the_rows():
    """Every counted row hands out its weight once per query head: what a kv head's positions gather sums to rows x group."""
    desc = synth.fixed_descriptor([777], [9], [4], seed=3)
    ctx = make(B8, desc.page_table.shape[1], 32, 1, binding.FLAG_KV_4BIT)
    pool = binding.alloc_kv_pool(ctx, desc.n_pages)
    k, v = synth.kv_values(790, 8, 128, seed=4)
    ctx.recg_kv_write(pool, desc.n_pages, 0, desc.page_table[0], 0, k.cuda(), v.cuda())
    q = synth.queries(13, 32, 128, seed=6).cuda()
    lse, o, w = torch.empty((13, 32), device="cuda"), torch.empty_like(q), torch.zeros((2, desc.n_pages, 8, 16), device="cuda")
    ctx.recg_attention(binding.Batch([777], [9], [4], None, desc.page_table, pool, desc.n_pages), 0, q, o, lse)
    ctx.recg_kv_weights(None, 0, q, lse, None, w)
    ctx.recg_sync()
    assert torch.allclose(w[0].sum((0, 2)), torch.full((8,), 13.0 * 4, device="cuda"), rtol=1e-5)
    ctx.recg_free()


# ---- choice ---------------------------------------------------------------------------------------------------------------
def chosen(w, budget, sink, recent):
    """Positions that stay of one head, from the definition."""
    L = len(w)
    if L <= budget:
        return np.arange(L)
    forced = (np.arange(L) < sink) | (np.arange(L) >= L - recent)
    nan_last = np.isnan(w)
    w = np.where(nan_last, 0.0, w)
    return np.sort(np.lexsort((np.arange(L), -w, nan_last, ~forced))[:budget])


def draw_weights(n_layers, n_pages, nkv, seed, kind):
    g = torch.Generator().manual_seed(seed)
    w = torch.exp(3 * torch.randn((n_layers, n_pages, nkv, 16), generator=g))
    if kind == "ties":
        w = torch.round(w).clamp(max=6)                                   # few values, many zeros
    elif kind == "equal":
        w = torch.full_like(w, 0.25)
    elif kind == "signs":
        w = torch.randn(w.shape, generator=g)
        w[torch.rand(w.shape, generator=g) < 0.2] = 0.0
        w[torch.rand(w.shape, generator=g) < 0.1] = -0.0
    elif kind == "odd":
        for x, share in ((float("inf"), 0.02), (float("nan"), 0.1), (1e-45, 0.1), (0.0, 0.2), (-0.0, 0.1), (-1e30, 0.05)):
            w[torch.rand(w.shape, generator=g) < share] = x
    return w


@pytest.mark.parametrize("kind", ["plain", "ties", "equal", "signs", "odd"])
@pytest.mark.parametrize("reqs,sink,recent", [
    ([(0, 5), (1, 1), (16, 4), (17, 16), (100, 7), (333, 300), (64, 64), (50, 80)], 0, 0),
    ([(100, 5), (101, 6), (333, 300), (3, 9)], 4, 1), ([(9000, 1234), (8192, 64), (8193, 8192)], 4, 60), ([(40000, 39999)], 16, 0),
    ([(100000, 70001), (31, 30)], 4, 16), ([(300000, 1000)], 3, 50),
    ([(500, 20), (20, 20)], 0, 20)])
def test_choice(kind, reqs, sink, recent):
    nkv = 2
    L, budget = (np.array(x) for x in zip(*reqs))
    pt, n_pages = synth.page_tables(L, [1] * len(L), 16, seed=5, spare_pages=2)
    ctx = make(TINY, pt.shape[1], 32, len(L), 0, layers=3)
    w = draw_weights(3, n_pages, nkv, 7, kind)
    most = int(np.minimum(L, budget).max())
    keep = torch.full((2, len(L), nkv, most + 3), -9, dtype=torch.int32, device="cuda")
    ev = binding.Eviction(L, budget, pt, None, n_pages, w.cuda(), sink, recent, layers=(1, 3))
    ctx.recg_kv_select(ev, keep)
    ctx.recg_sync()
    got = keep.cpu().numpy()
    for layer in range(2):
        for r in range(len(L)):
            pos = np.arange(L[r])
            for h in range(nkv):
                want = chosen(w[layer + 1, pt[r][pos // 16], h, pos % 16].numpy(), int(budget[r]), sink, recent)
                assert np.array_equal(got[layer, r, h, :len(want)], want), (layer, r, h)
                assert (got[layer, r, h, len(want):] == -1).all()
    ctx.recg_free()


# ---- move -----------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("flags", POOLS)
@pytest.mark.parametrize("head_dim,nkv", [(64, 2), (128, 8)])
@pytest.mark.parametrize("in_place", [True, False])
def test_move(flags, head_dim, nkv, in_place):
    L, budget = [0, 1, 40, 700, 333, 16, 64, 2100], [4, 0, 17, 123, 332, 16, 1, 1500]
    pt, n_pages = synth.page_tables(list(L) * 2, [1] * 16, 16, seed=6, spare_pages=5)
    src, dst = pt[:8], None if in_place else pt[8:]
    ctx = make((2 * nkv, nkv, head_dim), pt.shape[1], 32, 8, flags, layers=3)
    pool = binding.alloc_kv_pool(ctx, n_pages)
    g = torch.Generator(device="cuda").manual_seed(3)
    ctx_pool = pool.view(torch.uint8)
    ctx_pool.random_(0, 256, generator=g)
    for r in range(8):
        for layer in range(3):
            if L[r]:
                k, v = synth.kv_values(L[r], nkv, head_dim, seed=10 * r + layer, device="cuda")
                ctx.recg_kv_write(pool, n_pages, layer, src[r], 0, k, v)
    w = torch.rand((3, n_pages, nkv, 16), device="cuda")
    before, w_before = ctx_pool.clone(), w.clone()
    rows = [[ctx.recg_kv_read(pool, n_pages, layer, src[r], 0, L[r]) if L[r] else None for layer in range(3)] for r in range(8)]

    ev = binding.Eviction(L, budget, src, pool, n_pages, w, 0, 0, dst, (1, 3))
    keep = torch.empty((2, 8, nkv, 1500), dtype=torch.int32, device="cuda")
    ctx.recg_kv_select(ev, keep)
    ctx.recg_kv_compact(ev, keep)
    ctx.recg_sync()
    lists = keep.cpu().numpy()
    block = before.numel() // (3 * n_pages * nkv)
    changed = (ctx_pool != before).view(3, n_pages, nkv, block).any(-1).cpu().numpy()
    allowed = np.zeros_like(changed)
    for r in range(8):
        n = min(L[r], budget[r])
        to = src[r] if in_place else dst[r]
        allowed[1:, to[:-(-n // 16)]] = True
        for layer in (1, 2):
            if not n:
                continue
            ids = lists[layer - 1, r, :, :n]
            k0, v0 = (t.cpu() for t in rows[r][layer])
            k1, v1 = (t.cpu() for t in ctx.recg_kv_read(pool, n_pages, layer, to, 0, n))
            for h in range(nkv):
                assert torch.equal(k1[:, h], k0[ids[h], h]) and torch.equal(v1[:, h], v0[ids[h], h]), (r, layer, h)
                pos = np.arange(n)
                wh = w[layer, to[pos // 16], h, pos % 16].cpu()
                assert torch.equal(wh, w_before[layer, src[r][ids[h] // 16], h, ids[h] % 16].cpu())
            # slots of the last page behind what stays are left as they were
            for s in range(n, min(-(-n // 16) * 16, L[r] if in_place else n)):
                kb, vb = ctx.recg_kv_read(pool, n_pages, layer, to, s, 1)
                assert torch.equal(kb.cpu()[0], k0[s]) and torch.equal(vb.cpu()[0], v0[s])
    assert not changed[~allowed].any()
    ctx.recg_free()


@pytest.mark.parametrize("flags", POOLS)
def test_lists_that_name_no_position_are_refused_on_the_device(flags):
    pt = np.arange(4)[None]
    ctx = make(TINY, 4, 32, 1, flags)
    pool = binding.alloc_kv_pool(ctx, 8)
    k, v = synth.kv_values(60, 2, 64, seed=3, device="cuda")
    ctx.recg_kv_write(pool, 8, 0, pt[0], 0, k, v)
    held = ctx.recg_kv_read(pool, 8, 0, pt[0], 0, 60)
    ev = binding.Eviction([60], [5], pt, pool, 8, None)
    keep = torch.tensor([3, -1, 60, 1, 59], dtype=torch.int32, device="cuda").expand(1, 1, 2, 5).contiguous()
    ctx.recg_kv_compact(ev, keep)
    with pytest.raises(binding.RecgError, match="out of range"):
        ctx.recg_sync()
    got = ctx.recg_kv_read(pool, 8, 0, pt[0], 0, 60)
    ctx.recg_sync()
    for a, b in zip(got, held):                         # entries 1 (-1), 2 (60) and 3 (1 < 3) are left as they were
        assert torch.equal(a[0], b[3]) and torch.equal(a[4], b[59]) and torch.equal(a[1:4], b[1:4]) and torch.equal(a[5:], b[5:])
    ctx.recg_free()


def test_refusals():
    pt = np.arange(8).reshape(2, 4)
    ctx = make(TINY, 4, 8, 2, 0)
    pool = binding.alloc_kv_pool(ctx, 16)
    w = torch.zeros((2, 16, 2, 16), device="cuda")
    keep = torch.zeros((1, 2, 2, 10), dtype=torch.int32, device="cuda")
    ok = dict(ctx_len=[40, 50], budget=[10, 10], page_table=pt, kv_pool=pool, kv_pool_pages=16, weights=w)

    def refused(text, status=1, both=True, **kw):
        ev = binding.Eviction(**{**ok, **kw})
        for f in ((ctx.recg_kv_select, ctx.recg_kv_compact) if both else (ctx.recg_kv_compact,)):
            with pytest.raises(binding.RecgError, match=text) as e:
                f(ev, keep)
            assert e.value.status == status

    refused("negative", ctx_len=[-1, 5])
    refused("negative", budget=[-1, 5])
    refused("negative n_sink", n_sink=-1)
    refused("budget below", n_sink=6, n_recent=5)
    refused("does not cover", 3, ctx_len=[65, 5])
    refused("page id", page_table=np.where(pt == 2, 16, pt))
    refused("page id", page_table=np.where(pt == 2, -1, pt))
    refused("layer range", layers=(2, 3))
    refused("keep_stride", 3, budget=[11, 10])
    refused("named twice", both=False, page_table=np.where(pt == 2, 5, pt))
    refused("named twice or is a source", both=False, dst_page_table=pt + 4)
    refused("named twice or is a source", both=False, dst_page_table=np.full((2, 4), 9))
    with pytest.raises(binding.RecgError, match="weights is null"):
        ctx.recg_kv_select(binding.Eviction(**{**ok, "weights": None}), keep)
    with pytest.raises(binding.RecgError, match="pool is null"):
        ctx.recg_kv_compact(binding.Eviction(**{**ok, "kv_pool": None}), keep)
    for bad in (keep[:, :1], keep.float(), keep.cpu(), keep[..., ::2]):
        with pytest.raises(ValueError):
            ctx.recg_kv_select(binding.Eviction(**ok), bad)
    with pytest.raises(ValueError):
        binding.Eviction(**{**ok, "budget": [3]})
    # shared source pages are fine where what stays goes elsewhere
    shared = np.array([[0, 1, 2, 3], [0, 1, 4, 5]])
    ev = binding.Eviction(**{**ok, "page_table": shared, "dst_page_table": np.arange(8, 16).reshape(2, 4)})
    ctx.recg_kv_select(ev, keep)
    ctx.recg_kv_compact(ev, keep)
    ctx.recg_sync()
    # gathered weight
    q, lse = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, 4), device="cuda")
    batch = binding.Batch([3, 9], [1, 1], [0, 0], None, pt, pool, 16)
    for decay in (-1.0, float("nan"), float("inf")):
        with pytest.raises(binding.RecgError, match="decay"):
            ctx.recg_kv_weights(batch, 0, q, lse, None, w, decay=decay)
    with pytest.raises(binding.RecgError, match="layer"):
        ctx.recg_kv_weights(batch, 2, q, lse, None, w)
    for kw in (dict(lse=lse[:1]), dict(q=q[:1]), dict(weights_out=w[:1]), dict(row_weight=torch.ones(3, device="cuda")), dict(weights_in=w[:1])):
        with pytest.raises(ValueError):
            ctx.recg_kv_weights(**{**dict(batch=batch, layer=0, q=q, lse=lse, weights_in=None, weights_out=w), **kw})
    assert binding.lib().recg_kv_weights(ctx.h, C.byref(batch.c), 0, q.data_ptr() + 2, lse.data_ptr(), None, 1.0, None, w.data_ptr()) == 1
    ctx.recg_sync()
    ctx.recg_free()


@pytest.mark.parametrize("flags", POOLS)
def test_calls_that_would_collide_or_be_misaligned_are_refused(flags):
    ctx = make(TINY, 4, 8, 2, flags)
    pool = binding.alloc_kv_pool(ctx, 16)
    w = torch.zeros((2 * 16 * 2 * 16 + 4,), device="cuda")
    q, lse = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, 4), device="cuda")
    even, odd = w[:-4], w[1:-3]
    table = np.array([[0, 1, 2, 3], [4, 5, 6, 7]])
    batch = binding.Batch([40, 50], [1, 1], [0, 0], None, table, pool, 16)
    lib = binding.lib()
    for src, dst in ((odd, even), (even, odd), (None, odd)):
        assert lib.recg_kv_weights(ctx.h, C.byref(batch.c), 0, q.data_ptr(), lse.data_ptr(), None, 1.0,
                                   None if src is None else src.data_ptr(), dst.data_ptr()) == 1
        assert b"16-byte" in lib.recg_last_error(ctx.h)
    out = even.view(2, 16, 2, 16)
    for bad in (np.array([[0, 1, 2, 3], [0, 5, 6, 7]]), np.array([[0, 1, 2, 3], [4, 5, 4, 7]])):
        shared = binding.Batch([40, 50], [1, 1], [0, 0], None, bad, pool, 16)
        for given in (shared, None):                                   # (the second: laid out by the call that was refused)
            with pytest.raises(binding.RecgError, match="named twice"):
                ctx.recg_kv_weights(given, 0, q, lse, None, out)
    ctx.recg_kv_weights(binding.Batch([40, 33], [1, 1], [0, 0], None, np.array([[0, 1, 2, 3], [4, 5, 6, 0]]), pool, 16), 0, q, lse, None, out)
    ctx.recg_kv_weights(batch, 0, q, lse, None, out)                   # (a page behind the last position is nobody's)
    rows = torch.zeros((2, 2, 64), dtype=torch.bfloat16, device="cuda")
    off = binding.Batch([3], [2], [0], None, np.arange(4)[None], pool.view(torch.uint8)[2:] if flags else pool[1:], 15)
    with pytest.raises(binding.RecgError, match="16-byte"):
        ctx.recg_kv_append(off, 0, rows, rows)
    with pytest.raises(binding.RecgError, match="beyond"):             # pos0 + n_pos passes 31 bits
        ctx._check(lib.recg_kv_read(ctx.h, pool.data_ptr(), 16, 0, table.astype(np.int32)[0].ctypes.data, 4, 2 ** 31 - 1, 2,
                                    rows.data_ptr(), rows.data_ptr()))
    ctx.recg_sync()
    ctx.recg_free()


@pytest.mark.parametrize("flags", POOLS)
def test_attention_captured_before_its_work_list_was_built(flags):
    """A batch that only rows were read of has no work list; the one that a captured attention builds is there after a replay only."""
    nq, nkv, d = B8
    desc = synth.fixed_descriptor([300, 20], [3, 1], [2, 0], seed=3)
    T = desc.n_tokens
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = make(B8, desc.page_table.shape[1], T, 2, flags)
        pool = binding.alloc_kv_pool(ctx, desc.n_pages)
        for r, n in enumerate(desc.ctx_len + desc.rows):
            k, v = synth.kv_values(int(n), nkv, d, seed=r)
            ctx.recg_kv_write(pool, desc.n_pages, 0, desc.page_table[r], 0, k.cuda(), v.cuda())
        batch = binding.Batch(desc.ctx_len, desc.verify_len, desc.block_size, None, desc.page_table, pool, desc.n_pages)
        other = binding.Batch([3], [2], [0], None, desc.page_table[:1], pool, desc.n_pages)
        q = synth.queries(T, nq, d, seed=8).cuda()
        want, got, again, spare = (torch.zeros_like(q) for _ in range(4))
        w_want, w_got = (torch.zeros((2, desc.n_pages, nkv, 16), device="cuda") for _ in range(2))
        lse = torch.empty((T, nq), device="cuda")
        ctx.recg_attention(batch, 0, q, want, lse)
        ctx.recg_kv_weights(None, 0, q, lse, None, w_want)
        ctx.recg_attention(other, 0, q, spare)
        ctx.recg_kv_rows(batch, 0)
        ctx.recg_sync()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            ctx.recg_attention(None, 0, q, got, lse)
            ctx.recg_kv_weights(None, 0, q, lse, None, w_got)
        ctx.recg_attention(None, 0, q, again)                          # the graph has not run yet
        torch.cuda.synchronize()
        assert torch.equal(again, want) and not got.any()
        for _ in range(2):
            got.zero_(), w_got.zero_()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(got, want) and torch.equal(w_got, w_want)
        del graph
        ctx.recg_sync()
        ctx.recg_free()


def test_eviction_and_shift_are_refused_while_captured():
    """They copy host arrays; what lies around them in the capture is not harmed."""
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = make(TINY, 4, 8, 2, binding.FLAG_KV_4BIT)
        pool = binding.alloc_kv_pool(ctx, 8)
        w = torch.rand((2, 8, 2, 16), device="cuda")
        keep = torch.zeros((1, 2, 2, 10), dtype=torch.int32, device="cuda")
        ev = binding.Eviction([40, 50], [10, 10], np.arange(8).reshape(2, 4), pool, 8, w)
        rows = torch.randn((2, 2, 64), device="cuda").bfloat16()
        ctx.recg_kv_append(binding.Batch([40, 50], [1, 1], [0, 0], None, np.arange(8).reshape(2, 4), pool, 8), 0, rows, rows)
        ctx.recg_sync()
        graph = torch.cuda.CUDAGraph()
        got = torch.zeros((2, 2, 2, 64), dtype=torch.bfloat16, device="cuda")
        with torch.cuda.graph(graph, stream=stream):
            for call in (lambda: ctx.recg_kv_select(ev, keep), lambda: ctx.recg_kv_compact(ev, keep), lambda: ctx.recg_kv_shift([1, 2])):
                with pytest.raises(binding.RecgError, match="captured"):
                    call()
            ctx.recg_kv_rows(None, 0, got[0], got[1])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got[0].cpu(), _kv4.values_bf16(rows.cpu())) and torch.equal(got[0], got[1])
        del graph
        ctx.recg_kv_select(ev, keep)
        ctx.recg_sync()
        ctx.recg_free()
