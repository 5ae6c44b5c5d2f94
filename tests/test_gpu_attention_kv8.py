"""Attention over an 8-bit pool against float64 attention over what the pool stands for, with bounds from the roundings that the kernels
make (tests/_kv8.py)."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2609_34388_b200 import binding, synth
from tests import _kv4, _kv8
from tests._util import f64

pytestmark = pytest.mark.gpu

TINY = (4, 2, 64)
B8 = (32, 8, 128)
B14 = (40, 8, 128)
KV8 = binding.FLAG_KV_8BIT
FLAGS = [KV8, KV8 | binding.FLAG_SIMT_ATTENTION]


def shape_of(heads):
    nq, nkv, d = heads
    return synth.ModelShape(n_layers=2, hidden=64, n_q_heads=nq, n_kv_heads=nkv, head_dim=d, ffn=64, vocab=64)


def run_case(heads, reqs, seed, flags=KV8, corr=None, scale=1.0, offset=0.0, layer=1, window=None, spread=0.0):
    """reqs: (L, v, b); corr: per request the draft indices that branches replace (b masks each); window: (n_sink, window); spread: rows of K and V
    differ by e^(spread x).  Asserts o and lse."""
    nq, nkv, d = heads
    L, v, b = (list(x) for x in zip(*reqs))
    corr = corr or [()] * len(reqs)
    desc = synth.fixed_descriptor(L, v, b, seed=seed, corr=[[(i, 5) for i in c] for c in corr], corr_block=b)
    T = desc.n_tokens
    ctx = binding.Context(binding.make_config(shape_of(heads), len(reqs), T, desc.page_table.shape[1], flags))
    if window:
        ctx.recg_window(*window)
    pool = binding.alloc_kv_pool(ctx, desc.n_pages, fill=None)
    pool.view(torch.uint8).fill_(255)              # whatever nobody writes is NaN
    q = (synth.queries(T, nq, d, seed=seed + 5) * scale).to(torch.bfloat16)
    g = torch.Generator().manual_seed(seed)
    ks, vs = [], []
    for r, n in enumerate(desc.rows):
        k_, v_ = synth.kv_values(L[r] + int(n), nkv, d, seed=seed * 100 + r)
        k_, v_ = ((t.float() * torch.exp(spread * torch.randn((t.shape[0], nkv, 1), generator=g)) + o).to(torch.bfloat16) for t, o in ((k_, offset), (v_, 0.0)))
        ctx.recg_kv_write(pool, desc.n_pages, layer, desc.page_table[r], 0, k_.cuda(), v_.cuda())
        if flags & KV8:
            ks.append(_kv8.Cache(nkv, d).write(0, k_).held)
            vs.append(_kv8.Cache(nkv, d).write(0, v_).held)
        else:
            ks.append(f64(k_))
            vs.append(f64(v_))
    batch = binding.Batch(L, v, b, None, desc.page_table, pool, desc.n_pages, **desc.branch_kwargs())
    o = torch.full((T + 1, nq, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((T + 1, nq), float("nan"), device="cuda")
    ctx.recg_attention(batch, layer, q.cuda(), o[:T], lse[:T])
    again = torch.empty_like(o[:T])
    ctx.recg_attention(None, layer, q.cuda(), again)
    ctx.recg_sync()
    assert torch.equal(again, o[:T])               # the same without the log-sum-exp, and deterministic
    assert torch.isnan(o[T]).all() and torch.isnan(lse[T]).all()
    t = 0
    for r, n in enumerate(desc.rows):
        n = int(n)
        see = _kv4.visible(L[r], v[r], b[r], corr[r], b[r])
        if window:
            see = _kv8.window(see, _kv8.positions(L[r], v[r], b[r], corr[r], b[r]), *window)
        assert see.any(-1).all()
        qr, got, got_lse = f64(q[t:t + n]), f64(o[t:t + n]), f64(lse[t:t + n])
        if flags & KV8:
            _kv8.check(got, got_lse, qr, ks[r], vs[r], see)
        else:                                       # bf16: probabilities rounded to bf16 (2^-8 of a term), everything else as above
            ref, ref_lse = _kv8.attention(qr, ks[r], vs[r], see)
            o_err, lse_err = _kv8.attention_bounds(qr, ks[r], vs[r], see)
            terms, _ = _kv8.attention(qr, ks[r], np.abs(vs[r]), see)
            over = np.abs(got - ref) / (o_err + 2.0 ** -8 * terms + 2.0 ** -8 * (np.abs(ref) + o_err) + 1e-30)
            assert np.isfinite(got).all() and over.max() <= 1.0, (r, over.max())
            assert (np.abs(got_lse - ref_lse) <= lse_err).all(), r
        t += n
    ctx.recg_free()


SHORT = [[(0, 1, 0)], [(0, 0, 1)], [(1, 1, 1)], [(15, 1, 0)], [(16, 2, 2)], [(17, 3, 8)], [(33, 8, 8)], [(63, 1, 1)], [(64, 1, 0)],
         [(65, 0, 8)], [(200, 16, 16)], [(130, 5, 0)], [(127, 1, 0)], [(128, 1, 0)], [(129, 33, 0)],
         [(100, 4, 4), (7, 1, 8), (300, 16, 16), (64, 2, 2), (0, 8, 8)]]
LONG = [(B8, [(4096, 16, 16)]), (B8, [(1000, 33, 31), (5, 40, 0)]), (B8, [(3000, 1, 0)] + [(50 + 37 * i, 1, 0) for i in range(20)]),
        (TINY, [(2500, 40, 30), (100, 70, 0)]), (B14, [(300, 25, 25), (77, 26, 24), (1500, 50, 14), (0, 3, 2), (40, 1, 8)]),
        (B14, [(9000, 1, 0)]), (B8, [(300, 200, 0), (700, 8, 8), (0, 95, 1)]), ((16, 1, 128), [(500, 8, 1), (40, 1, 0)]), ((8, 8, 64), [(333, 1, 0), (90, 4, 5)])]


@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("heads", [TINY, B8])
@pytest.mark.parametrize("reqs", SHORT)
def test_short_contexts(heads, reqs, flags):
    run_case(heads, reqs, seed=11, flags=flags)


@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("heads,reqs", LONG)
def test_long_contexts_many_rows_and_group_sizes(heads, reqs, flags):
    run_case(heads, reqs, seed=21, flags=flags)


@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("heads", [TINY, B8])
def test_branches(heads, flags):
    run_case(heads, [(100, 8, 8), (0, 5, 4), (1030, 16, 7), (31, 2, 0)], seed=31, flags=flags, corr=[(1, 6), (4,), (3, 15), (1,)])


@pytest.mark.parametrize("heads,n,rows", [(B8, 700, (1, 0)), (B8, 260, (3, 1)), (TINY, 900, (2, 0)), (B14, 150, (1, 2))])
def test_many_short_requests(heads, n, rows):
    """More work items than a CTA keeps descriptors of on chip."""
    g = np.random.default_rng(9)
    run_case(heads, [(int(x), *rows) for x in g.integers(0, 100, n)], seed=61)


@pytest.mark.parametrize("flags", FLAGS)
def test_sharp_scores_keys_off_centre_and_rows_of_many_sizes(flags):
    run_case(B8, [(900, 3, 5), (2000, 1, 0)], seed=41, flags=flags, scale=12.0)
    run_case(TINY, [(900, 3, 5)], seed=42, flags=flags, scale=12.0)
    run_case(B8, [(500, 3, 5)], seed=43, flags=flags, offset=20.0)
    run_case(B8, [(700, 3, 5), (300, 1, 0)], seed=44, flags=flags, spread=1.5)
    run_case(TINY, [(700, 3, 5), (300, 1, 0)], seed=45, flags=flags, spread=1.5)


def pool_of(ctx, desc, layer, k, v, flags=KV8):
    pool = binding.alloc_kv_pool(ctx, desc.n_pages, fill=None)
    pool.view(torch.uint8).fill_(255)
    ctx.recg_kv_write(pool, desc.n_pages, layer, desc.page_table[0], 0, k.cuda(), v.cuda())
    return pool


@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("heads", [TINY, B8])
@pytest.mark.parametrize("rows", [(1, 0), (4, 3)])
def test_blocks_of_very_different_sizes(heads, rows, flags):
    """V of blocks that lie 2^30 apart and zeros between them: what a block contributes counts, not how large it is; a row whose larger
    block has next to no probability loses nothing of the others."""
    nq, nkv, d = heads
    desc = synth.fixed_descriptor([400], [rows[0]], [rows[1]], seed=3)
    n = 400 + desc.n_tokens
    ctx = binding.Context(binding.make_config(shape_of(heads), 1, 32, desc.page_table.shape[1], flags))
    k, v = synth.kv_values(n, nkv, d, seed=9)
    q = synth.queries(desc.n_tokens, nq, d, seed=8)
    size = torch.ones(n)
    size[:16], size[16:32], size[32:48], size[100:130] = 2.0 ** 30, 2.0 ** -30, 0.0, 2.0 ** 15
    v = (v.float() * size[:, None, None]).bfloat16()
    k = k.float()
    k[:16] = 0.0                                             # ... the large block: scores far below the others'
    for h in range(nkv):
        k[:16, h] -= 40.0 * torch.nn.functional.normalize(q[0, h * (nq // nkv)].float(), dim=0)
    k = k.bfloat16()
    pool = pool_of(ctx, desc, 0, k, v, flags)
    batch = binding.Batch([400], [rows[0]], [rows[1]], None, desc.page_table, pool, desc.n_pages)
    o = torch.zeros((desc.n_tokens, nq, d), dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros((desc.n_tokens, nq), device="cuda")
    ctx.recg_attention(batch, 0, q.cuda(), o, lse)
    ctx.recg_sync()
    see = _kv4.visible(400, *rows)
    _kv8.check(f64(o), f64(lse), f64(q), _kv8.Cache(nkv, d).write(0, k).held, _kv8.Cache(nkv, d).write(0, v).held, see, 64.0)
    ctx.recg_free()


@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("heads", [TINY, B8])
def test_values_that_no_visible_row_holds_stay_out(heads, flags):
    """NaN in K and infinite V in a branch's rows reach that branch only; of a V alone that is none the log-sum-exp knows nothing."""
    nq, nkv, d = heads
    desc = synth.fixed_descriptor([50], [4], [3], seed=3, corr=[[(2, 5)]], corr_block=[3])
    ctx = binding.Context(binding.make_config(shape_of(heads), 1, 32, desc.page_table.shape[1], flags))
    n = 50 + desc.n_tokens
    k, v = synth.kv_values(n, nkv, d, seed=9)
    k[57:, 0, 5], v[57:, 1, 3] = float("nan"), float("inf")          # positions 57 .. 60: the branch; K of one head, V of another
    q = synth.queries(desc.n_tokens, nq, d, seed=8)
    pool = pool_of(ctx, desc, 0, k, v, flags)
    o = torch.zeros((desc.n_tokens, nq, d), dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros((desc.n_tokens, nq), device="cuda")
    batch = binding.Batch([50], [4], [3], None, desc.page_table, pool, desc.n_pages, **desc.branch_kwargs())
    ctx.recg_attention(batch, 0, q.cuda(), o, lse)
    ctx.recg_sync()
    see = _kv4.visible(50, 4, 3, (2,), 3)
    held_k, held_v = (np.nan_to_num(_kv8.Cache(nkv, d).write(0, t).held) for t in (k, v))
    _kv8.check(f64(o[:7]), f64(lse[:7]), f64(q[:7]), held_k, held_v, see[:7])
    g = nq // nkv
    assert torch.isnan(o[7:, :2 * g]).all() and torch.isnan(lse[7:, :g]).all()
    assert torch.isfinite(lse[7:, g:]).all() and torch.isfinite(o[7:, 2 * g:]).all()
    # a query that is not finite is nobody else's
    q2 = q.clone()
    q2[1, 0, 3], q2[2, 1, 7] = float("inf"), float("nan")
    o2 = torch.zeros_like(o)
    ctx.recg_attention(None, 0, q2.cuda(), o2)
    ctx.recg_sync()
    rest = torch.ones((7, nq), dtype=torch.bool)
    rest[1, 0] = rest[2, 1] = False
    assert torch.equal(o2[:7].cpu()[rest], o[:7].cpu()[rest]) and torch.isnan(o2[2, 1]).all() and torch.isnan(o2[1, 0]).all()
    ctx.recg_free()


def test_refusals():
    ctx = binding.Context(binding.make_config(shape_of(TINY), 1, 8, 4, KV8))
    pool = binding.alloc_kv_pool(ctx, 4)
    batch = binding.Batch([3], [2], [0], None, np.arange(4)[None], pool, 4)
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device="cuda")
    lib = binding.lib()
    b = C.byref(batch.c)
    assert lib.recg_attention(ctx.h, b, 0, q.data_ptr() + 2, q.data_ptr()) == 1 and b"aligned" in lib.recg_last_error(ctx.h)
    assert lib.recg_attention(ctx.h, b, 2, q.data_ptr(), q.data_ptr()) == 1 and b"layer" in lib.recg_last_error(ctx.h)
    off = binding.Batch([3], [2], [0], None, np.arange(4)[None], pool[1:], 4)
    with pytest.raises(binding.RecgError, match="16-byte"):
        ctx.recg_attention(off, 0, q, q)
    ctx.recg_attention(batch, 0, q, torch.empty_like(q))
    ctx.recg_sync()
    ctx.recg_free()
