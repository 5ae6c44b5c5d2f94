"""Attention over a 4-bit pool against float64 attention over what the pool stands for, with bounds from the roundings that the
kernels make (tests/_kv4.py), and the log-sum-exp for both kinds of pool."""
import numpy as np
import pytest
import torch

from paper_2609_34388_b200 import binding, synth
from tests import _kv4
from tests._util import f64

pytestmark = pytest.mark.gpu

TINY = (4, 2, 64)
B8 = (32, 8, 128)
B14 = (40, 8, 128)


def shape_of(heads):
    nq, nkv, d = heads
    return synth.ModelShape(n_layers=2, hidden=64, n_q_heads=nq, n_kv_heads=nkv, head_dim=d, ffn=64, vocab=64)


def run_case(heads, reqs, seed, flags=binding.FLAG_KV_4BIT, corr=None, scale=1.0, offset=0.0, layer=1, check=None):
    """reqs: (L, v, b); corr: per request the draft indices that branches replace (b masks each).  Asserts o and lse."""
    nq, nkv, d = heads
    L, v, b = (list(x) for x in zip(*reqs))
    corr = corr or [()] * len(reqs)
    desc = synth.fixed_descriptor(L, v, b, seed=seed, corr=[[(i, 5) for i in c] for c in corr], corr_block=b)
    T = desc.n_tokens
    ctx = binding.Context(binding.make_config(shape_of(heads), len(reqs), T, desc.page_table.shape[1], flags))
    pool = binding.alloc_kv_pool(ctx, desc.n_pages, fill=None)
    pool.view(torch.uint8).fill_(255)              # steps and minima of slots that nobody writes are NaN, codes 15
    q = (synth.queries(T, nq, d, seed=seed + 5) * scale).to(torch.bfloat16)
    ks, vs = [], []
    for r, n in enumerate(desc.rows):
        k_, v_ = synth.kv_values(L[r] + int(n), nkv, d, seed=seed * 100 + r)
        k_ = (k_ + offset).to(torch.bfloat16)
        ks.append(k_)
        vs.append(v_)
        ctx.recg_kv_write(pool, desc.n_pages, layer, desc.page_table[r], 0, k_.cuda(), v_.cuda())
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
        assert see.any(-1).all()
        qr, got, got_lse = f64(q[t:t + n]), f64(o[t:t + n]), f64(lse[t:t + n])
        if flags & binding.FLAG_KV_4BIT:
            kc, vc = _kv4.codes(ks[r]), _kv4.codes(vs[r])
            ref, ref_lse = _kv4.attention(qr, kc[2] + kc[1] * kc[0], vc[2] + vc[1] * vc[0], see)
            o_err, lse_err = _kv4.attention_bounds(qr, kc, vc, see)
            over = np.abs(got - ref) / (o_err + 2.0 ** -8 * (np.abs(ref) + o_err) + 1e-30)
            assert np.isfinite(got).all() and over.max() <= 1.0, (r, over.max())
        else:
            ref, ref_lse = _kv4.attention(qr, f64(ks[r]), f64(vs[r]), see)
            lse_err = 2.0 ** -19 * (np.abs(qr) @ np.abs(f64(ks[r])).max((0, 1))) / np.sqrt(d) + 2.0 ** -20 * (1 + np.abs(ref_lse))
        over = np.abs(got_lse - ref_lse) / lse_err
        assert np.isfinite(got_lse).all() and over.max() <= 1.0, (r, over.max())
        t += n
    ctx.recg_free()


FLAGS = [binding.FLAG_KV_4BIT, binding.FLAG_KV_4BIT | binding.FLAG_SIMT_ATTENTION]


@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("heads", [TINY, B8])
@pytest.mark.parametrize("reqs", [
    [(0, 1, 0)], [(0, 0, 1)], [(1, 1, 1)], [(15, 1, 0)], [(16, 2, 2)], [(17, 3, 8)], [(33, 8, 8)], [(63, 1, 1)], [(64, 1, 0)],
    [(65, 0, 8)], [(200, 16, 16)], [(130, 5, 0)], [(127, 1, 0)], [(128, 1, 0)], [(129, 33, 0)],
    [(100, 4, 4), (7, 1, 8), (300, 16, 16), (64, 2, 2), (0, 8, 8)]])
def test_short_contexts(heads, reqs, flags):
    run_case(heads, reqs, seed=11, flags=flags)


@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("heads,reqs", [
    (B8, [(4096, 16, 16)]), (B8, [(1000, 33, 31), (5, 40, 0)]), (B8, [(3000, 1, 0)] + [(50 + 37 * i, 1, 0) for i in range(20)]),
    (TINY, [(2500, 40, 30), (100, 70, 0)]), (B14, [(300, 25, 25), (77, 26, 24), (1500, 50, 14), (0, 3, 2), (40, 1, 8)]),
    (B14, [(9000, 1, 0)]), (B8, [(300, 200, 0), (700, 8, 8), (0, 95, 1)]), ((16, 1, 128), [(500, 8, 1), (40, 1, 0)]),
    ((6, 2, 128), [(700, 5, 6), (0, 43, 0)]), ((8, 8, 64), [(333, 1, 0), (90, 4, 5)])])
def test_long_contexts_many_rows_and_group_sizes(heads, reqs, flags):
    if (heads[0] + 2 * heads[1]) * heads[2] % 128:
        pytest.skip("the context asks for a qkv width of whole 128 columns")
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
def test_sharp_scores_and_keys_off_centre(flags):
    """Scores whose maximum moves through the context, and keys that all lie far from zero (their common part only shifts the scores)."""
    run_case(B8, [(900, 3, 5), (2000, 1, 0)], seed=41, flags=flags, scale=12.0)
    run_case(TINY, [(900, 3, 5)], seed=42, flags=flags, scale=12.0)
    run_case(B8, [(500, 3, 5)], seed=43, flags=flags, offset=20.0)


@pytest.mark.parametrize("flags", [0, binding.FLAG_SIMT_ATTENTION])
@pytest.mark.parametrize("heads", [TINY, B8])
def test_log_sum_exp_of_a_bf16_pool(heads, flags):
    run_case(heads, [(0, 1, 0), (40, 4, 4), (700, 16, 16)], seed=51, flags=flags)
    run_case(heads, [(3000, 16, 16)], seed=52, flags=flags)
    run_case(heads, [(30, 1, 0)], seed=53, flags=flags)


@pytest.mark.parametrize("flags", FLAGS)
def test_values_that_no_visible_row_holds_stay_out(flags):
    """NaN in the K and V of a branch's rows reaches that branch only; infinite V in a row that nobody but itself sees likewise."""
    nq, nkv, d = B8
    desc = synth.fixed_descriptor([50], [4], [3], seed=3, corr=[[(2, 5)]], corr_block=[3])
    ctx = binding.Context(binding.make_config(shape_of(B8), 1, 32, desc.page_table.shape[1], flags))
    n = 50 + desc.n_tokens
    k, v = synth.kv_values(n, nkv, d, seed=9)
    clean_k, clean_v = k.clone(), v.clone()
    k[57:], v[57:] = float("nan"), float("inf")                      # positions 57 .. 60: the branch
    q = synth.queries(desc.n_tokens, nq, d, seed=8).cuda()
    outs = []
    for kk, vv in ((k, v), (clean_k, clean_v)):
        pool = binding.alloc_kv_pool(ctx, desc.n_pages)
        ctx.recg_kv_write(pool, desc.n_pages, 0, desc.page_table[0], 0, kk.cuda(), vv.cuda())
        o = torch.zeros_like(q)
        batch = binding.Batch([50], [4], [3], None, desc.page_table, pool, desc.n_pages, **desc.branch_kwargs())
        ctx.recg_attention(batch, 0, q, o)
        outs.append(o)
    ctx.recg_sync()
    assert torch.equal(outs[0][:7], outs[1][:7]) and torch.isnan(outs[0][7:]).all()
    ctx.recg_free()


def test_refusals():
    ctx = binding.Context(binding.make_config(shape_of(TINY), 1, 8, 4, binding.FLAG_KV_4BIT))
    pool = binding.alloc_kv_pool(ctx, 4)
    batch = binding.Batch([3], [2], [0], None, np.arange(4)[None], pool, 4)
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros((2, 4), device="cuda")
    lib = binding.lib()
    assert lib.recg_attention_lse(ctx.h, None, 0, q.data_ptr(), q.data_ptr(), lse.data_ptr()) == 1        # no batch so far
    import ctypes as C
    b = C.byref(batch.c)
    assert lib.recg_attention_lse(ctx.h, b, 0, q.data_ptr(), q.data_ptr(), None) == 1
    assert lib.recg_attention(ctx.h, b, 0, q.data_ptr() + 2, q.data_ptr()) == 1 and b"aligned" in lib.recg_last_error(ctx.h)
    assert lib.recg_attention(ctx.h, b, 2, q.data_ptr(), q.data_ptr()) == 1 and b"layer" in lib.recg_last_error(ctx.h)
    off = binding.Batch([3], [2], [0], None, np.arange(4)[None], pool[1:], 4)
    with pytest.raises(binding.RecgError, match="16-byte"):
        ctx.recg_attention(off, 0, q, q)
    for bad in (lse.double(), lse[:1], lse.cpu(), torch.zeros((4, 2), device="cuda").t()[:, ::1]):
        with pytest.raises(ValueError):
            ctx.recg_attention(batch, 0, q, q, bad)
    ctx.recg_attention(batch, 0, q, torch.empty_like(q), lse)
    ctx.recg_sync()
    ctx.recg_free()


@pytest.mark.parametrize("flags", [0] + FLAGS)
def test_operations_on_rows_and_attention_of_one_batch_in_any_order(flags):
    """Reading rows lays the batch out without attention's work list, which an attention without a batch then has to build."""
    desc = synth.fixed_descriptor([700, 33, 0], [5, 1, 40], [4, 0, 3], seed=3)
    T = desc.n_tokens
    ctx = binding.Context(binding.make_config(shape_of(B8), 3, T, desc.page_table.shape[1], flags))
    pool = binding.alloc_kv_pool(ctx, desc.n_pages)
    for r, n in enumerate(desc.ctx_len + desc.rows):
        k, v = synth.kv_values(int(n), 8, 128, seed=r)
        ctx.recg_kv_write(pool, desc.n_pages, 0, desc.page_table[r], 0, k.cuda(), v.cuda())
    batch = binding.Batch(desc.ctx_len, desc.verify_len, desc.block_size, None, desc.page_table, pool, desc.n_pages)
    q = synth.queries(T, 32, 128, seed=8).cuda()
    want, lse = torch.empty_like(q), torch.empty((T, 32), device="cuda")
    ctx.recg_attention(batch, 0, q, want, lse)
    w_want = torch.zeros((2, desc.n_pages, 8, 16), device="cuda")
    ctx.recg_kv_weights(None, 0, q, lse, None, w_want)
    other = binding.Batch([3], [2], [0], None, desc.page_table[:1], pool, desc.n_pages)
    ctx.recg_attention(other, 0, q, torch.empty_like(q))                # another batch's list stands in the workspace now
    rows = ctx.recg_kv_rows(batch, 0)
    got, got_lse = torch.empty_like(q), torch.empty_like(lse)
    ctx.recg_attention(None, 0, q, got, got_lse)
    assert torch.equal(got, want) and torch.equal(got_lse, lse)
    ctx.recg_attention(other, 0, q, torch.empty_like(q))
    w = torch.zeros_like(w_want)
    ctx.recg_kv_weights(batch, 0, q, lse, None, w)
    ctx.recg_kv_append(None, 0, *rows)
    got.zero_()
    ctx.recg_attention(None, 0, q, got)
    assert torch.equal(w, w_want)
    if not flags:
        assert torch.equal(got, want)                                  # (in 4 bits rows that come back are other values)
    ctx.recg_sync()
    ctx.recg_free()
