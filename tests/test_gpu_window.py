"""Attention that looks back a window, over bf16 and 8-bit pools, against float64 attention with the same mask."""
import numpy as np
import pytest
import torch

from paper_2609_34388_b200 import binding, synth
from tests import _kv4, _kv8
from tests._util import f64
from tests.test_gpu_attention_kv8 import B8, B14, KV8, LONG, TINY, run_case, shape_of

pytestmark = pytest.mark.gpu

FLAGS = [0, KV8, binding.FLAG_SIMT_ATTENTION, KV8 | binding.FLAG_SIMT_ATTENTION]


@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("heads", [TINY, B8])
@pytest.mark.parametrize("window", [(0, 1), (1, 1), (4, 16), (0, 64), (64, 64), (65, 63), (5, 100), (130, 7), (0, 1 << 30), (1 << 30, 1)])
def test_windows_and_first_tokens(heads, window, flags):
    run_case(heads, [(0, 1, 0), (500, 1, 0), (129, 3, 8), (200, 16, 16), (64, 0, 8), (63, 1, 1), (321, 5, 0)], seed=11, flags=flags, window=window)


@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("window", [(4, 200), (100, 33), (0, 1500)])
@pytest.mark.parametrize("heads,reqs", LONG)
def test_long_contexts_many_rows_and_group_sizes(heads, reqs, window, flags):
    run_case(heads, reqs, seed=21, flags=flags, window=window)


@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("heads", [TINY, B8])
@pytest.mark.parametrize("window", [(4, 3), (0, 20), (64, 700)])
def test_branches(heads, window, flags):
    """Rows of branches stand where they hypothesise to, in front of rows that precede them."""
    run_case(heads, [(100, 8, 8), (0, 5, 4), (1030, 16, 7), (31, 2, 0), (2000, 40, 30)], seed=31, flags=flags, corr=[(1, 6), (4,), (3, 15), (1,), (2, 39)],
             window=window)


@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("heads,reqs", [(B8, [(900, 700, 0)]), (B8, [(300 + 7 * i, 40, 0) for i in range(9)]), (B8, [(300 + 7 * i, 1, 0) for i in range(60)]),
                                        (B14, [(500, 1, 0)] * 19 + [(400, 60, 9)] * 7), (TINY, [(500, 300, 0)] * 9), ((16, 1, 128), [(333, 500, 0)] * 5)])
def test_several_whole_tiles_for_a_cta(heads, reqs, flags):
    """More tiles than CTAs, all about as long: pairs of tiles and single ones, a last CTA with fewer."""
    run_case(heads, reqs, seed=71, flags=flags, window=(3, 50))


@pytest.mark.parametrize("flags", FLAGS)
def test_many_short_requests(flags):
    g = np.random.default_rng(9)
    run_case(B8, [(int(x), 1, 0) for x in g.integers(0, 400, 500)], seed=61, flags=flags, window=(3, 50))
    run_case(TINY, [(int(x), 2, 0) for x in g.integers(0, 400, 700)], seed=62, flags=flags, window=(3, 50))


@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("heads", [TINY, B8])
def test_what_no_row_sees_is_not_read(heads, flags):
    """NaN everywhere outside of what the window shows, in whole blocks and in those at its edges."""
    nq, nkv, d = heads
    L, rows, sink, window = 1500, 3, 5, 333
    desc = synth.fixed_descriptor([L], [rows], [0], seed=3)
    ctx = binding.Context(binding.make_config(shape_of(heads), 1, 32, desc.page_table.shape[1], flags))
    ctx.recg_window(sink, window)
    k, v = synth.kv_values(L + rows, nkv, d, seed=9)
    first = L - window + 1
    hidden = torch.zeros(L + rows, dtype=torch.bool)
    hidden[sink:first] = True
    bad = k.clone(), v.clone()
    # (a masked V next to visible ones: in 8 bits any, in bf16 those of blocks that are left out)
    edge = hidden.clone()
    if not flags & KV8:
        edge[:64], edge[first // 64 * 64:] = False, False
    bad[0][edge], bad[1][edge] = float("nan"), float("inf")
    q = synth.queries(rows, nq, d, seed=8)
    o = torch.zeros((rows, nq, d), dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros((rows, nq), device="cuda")
    pool = binding.alloc_kv_pool(ctx, desc.n_pages)
    ctx.recg_kv_write(pool, desc.n_pages, 0, desc.page_table[0], 0, bad[0].cuda(), bad[1].cuda())
    batch = binding.Batch([L], [rows], [0], None, desc.page_table, pool, desc.n_pages)
    ctx.recg_attention(batch, 0, q.cuda(), o, lse)
    ctx.recg_sync()
    assert torch.isfinite(o).all() and torch.isfinite(lse).all()
    see = _kv8.window(_kv4.visible(L, rows, 0), _kv8.positions(L, rows, 0), sink, window)
    if flags & KV8:
        held = [np.nan_to_num(_kv8.Cache(nkv, d).write(0, t).held) for t in bad]
        _kv8.check(f64(o), f64(lse), f64(q), *held, see)
    else:
        ref, ref_lse = _kv8.attention(f64(q), f64(k), f64(v), see)
        assert (np.abs(f64(o) - ref) <= 2.0 ** -7 * _kv8.attention(f64(q), f64(k), np.abs(f64(v)), see)[0] + 2.0 ** -8 * np.abs(ref)).all()
    ctx.recg_free()


@pytest.mark.parametrize("flags", FLAGS[:2])
def test_a_window_that_changes(flags):
    """The batch laid out before is seen through the new window; without one it is as it was, to the bit; captured calls keep theirs."""
    desc = synth.fixed_descriptor([900, 33, 400], [5, 1, 40], [4, 0, 3], seed=3)
    T = desc.n_tokens
    shape = shape_of(B8)
    plain = binding.Context(binding.make_config(shape, 3, T, desc.page_table.shape[1], flags))
    ctx = binding.Context(binding.make_config(shape, 3, T, desc.page_table.shape[1], flags))
    pool = binding.alloc_kv_pool(ctx, desc.n_pages)
    for r, n in enumerate(desc.ctx_len + desc.rows):
        k, v = synth.kv_values(int(n), 8, 128, seed=r)
        ctx.recg_kv_write(pool, desc.n_pages, 0, desc.page_table[r], 0, k.cuda(), v.cuda())
    batch = binding.Batch(desc.ctx_len, desc.verify_len, desc.block_size, None, desc.page_table, pool, desc.n_pages)
    q = synth.queries(T, 32, 128, seed=8).cuda()
    new = lambda: (torch.zeros_like(q), torch.zeros((T, 32), device="cuda"))

    def fresh(window):
        c = binding.Context(binding.make_config(shape, 3, T, desc.page_table.shape[1], flags))
        c.recg_window(*window)
        out = new()
        c.recg_attention(batch, 0, q, *out)
        c.recg_sync()
        c.recg_free()
        return out

    want = new()
    plain.recg_attention(batch, 0, q, *want)
    for window in ((0, 0), (4, 100), (200, 9), (0, 0), (4, 100)):
        ctx.recg_window(*window)
        for b in (batch, None):
            got = new()
            ctx.recg_attention(b, 0, q, *got)
            for a, w in zip(got, want if window == (0, 0) else fresh(window)):
                assert torch.equal(a, w)
    # rows laid the batch out, the window changed behind them
    ctx.recg_kv_rows(batch, 0)
    ctx.recg_window(7, 50)
    got = new()
    ctx.recg_attention(None, 0, q, *got)
    for a, w in zip(got, fresh((7, 50))):
        assert torch.equal(a, w)
    plain.recg_sync()
    ctx.recg_sync()
    plain.recg_free()
    ctx.recg_free()


@pytest.mark.parametrize("flags", FLAGS[:2])
def test_captured(flags):
    """Append and attention with a window, captured into a graph: replays follow what q, k and v hold."""
    desc = synth.fixed_descriptor([900, 33], [5, 1], [4, 0], seed=3)
    T = desc.n_tokens
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        ctx = binding.Context(binding.make_config(shape_of(B8), 2, T, desc.page_table.shape[1], flags))
        pool = binding.alloc_kv_pool(ctx, desc.n_pages)
        for r, n in enumerate(desc.ctx_len):
            k, v = synth.kv_values(int(n), 8, 128, seed=r)
            ctx.recg_kv_write(pool, desc.n_pages, 0, desc.page_table[r], 0, k.cuda(), v.cuda())
        ctx.recg_window(4, 300)
        batch = binding.Batch(desc.ctx_len, desc.verify_len, desc.block_size, None, desc.page_table, pool, desc.n_pages)
        x = torch.randn((T, 48, 128), device="cuda").bfloat16()
        turned, o = torch.empty((T, 32, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((T, 32, 128), dtype=torch.bfloat16, device="cuda")

        def both(b):
            ctx.recg_kv_append_rotary(b, 0, x[:, :32], x[:, 32:40], x[:, 40:], turned)
            ctx.recg_attention(None, 0, turned, o)

        both(batch)
        before = pool.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            both(None)
        for seed in (1, 2):
            x.copy_(torch.randn(x.shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda"))
            both(None)
            want = o.clone(), turned.clone(), pool.clone()
            o.zero_()
            turned.zero_()
            pool.copy_(before)
            graph.replay()
            assert torch.equal(o, want[0]) and torch.equal(turned, want[1]) and torch.equal(pool.view(torch.uint8), want[2].view(torch.uint8))
        ctx.recg_sync()
        del graph
        ctx.recg_free()


def test_refusals():
    shape = shape_of(TINY)
    four = binding.Context(binding.make_config(shape, 1, 8, 4, binding.FLAG_KV_4BIT))
    with pytest.raises(binding.RecgError, match="4 bits"):
        four.recg_window(0, 16)
    four.recg_window(0, 0)
    four.recg_free()
    ctx = binding.Context(binding.make_config(shape, 1, 8, 4, 0))
    for bad in ((-1, 5), (0, -1), ((1 << 30) + 1, 4), (0, (1 << 30) + 1)):
        with pytest.raises(binding.RecgError, match="2\\^30"):
            ctx.recg_window(*bad)
    assert binding.lib().recg_window(None, 0, 0) == 1
    ctx.recg_window(4, 16)
    pool = binding.alloc_kv_pool(ctx, 4)
    batch = binding.Batch([3], [2], [0], None, np.arange(4)[None], pool, 4)
    q, lse = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, 4), device="cuda")
    w = torch.zeros((2, 4, 2, 16), device="cuda")
    with pytest.raises(binding.RecgError, match="window"):
        ctx.recg_kv_weights(batch, 0, q, lse, None, w)
    ctx.recg_window(0, 0)
    ctx.recg_kv_weights(batch, 0, q, lse, None, w)
    ctx.recg_sync()
    ctx.recg_free()


@pytest.mark.parametrize("flags", FLAGS)
@pytest.mark.parametrize("window", [None, (5, 100)])
def test_workspace_regions_are_kept(flags, window):
    """With guard bands behind every region of the workspace, which recg_sync() checks."""
    flags |= binding.FLAG_DEBUG_CHECKS
    run_case(B8, [(900, 33, 8), (3, 1, 0), (0, 64, 0)], seed=81, flags=flags, window=window, corr=[(2, 9), (), (63,)])
    run_case(TINY, [(500, 1, 0)] * 40, seed=82, flags=flags, window=window)


def test_two_contexts_on_two_streams():
    """A pool that two contexts read at once, each with a window of its own."""
    desc = synth.fixed_descriptor([3000], [16], [16], seed=3)
    T = desc.n_tokens
    k, v = synth.kv_values(3000 + T, 8, 128, seed=9)
    q = synth.queries(T, 32, 128, seed=8).cuda()
    torch.cuda.synchronize()
    alone, together = [], []
    contexts = []
    for i, window in enumerate(((0, 0), (4, 500))):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            ctx = binding.Context(binding.make_config(shape_of(B8), 1, T, desc.page_table.shape[1], KV8))
            ctx.recg_window(*window)
            contexts.append((ctx, stream))
    pool = binding.alloc_kv_pool(contexts[0][0], desc.n_pages)
    torch.cuda.synchronize()
    contexts[0][0].recg_kv_write(pool, desc.n_pages, 0, desc.page_table[0], 0, k.cuda(), v.cuda())
    contexts[0][0].recg_sync()
    batch = binding.Batch([3000], [16], [16], None, desc.page_table, pool, desc.n_pages)
    for out, wait in ((alone, True), (together, False)):
        outs = [torch.empty_like(q) for _ in contexts]
        torch.cuda.synchronize()
        for _ in range(20):
            for (ctx, _), o in zip(contexts, outs):
                ctx.recg_attention(batch, 0, q, o)
                if wait:
                    ctx.recg_sync()
        for ctx, _ in contexts:
            ctx.recg_sync()
        out += outs
    assert all(torch.equal(a, b) for a, b in zip(alone, together)) and not torch.equal(alone[0], alone[1])
    for ctx, _ in contexts:
        ctx.recg_free()
