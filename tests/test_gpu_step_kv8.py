"""Whole rounds over a cache in 8 bits, and rounds that look back a window.

The oracle gets the pool's own rows (read back after the round) as its K/V, so that a code which falls on the other side of a rounding
boundary costs nothing; the new rows' codes are checked by themselves: bit by bit in the first layer, whose input both kinds of pool share,
and within a rounding and the round's own tolerance in the others."""
import numpy as np
import pytest
import torch

from oracle import recg_oracle as orc
from paper_2609_34388_b200 import binding, synth
from tests import _kv4, _kv8
from tests._util import f64
from tests.test_gpu_step_kv4 import TOL, fill, model, read

pytestmark = pytest.mark.gpu

EIGHT = binding.FLAG_KV_8BIT
REQS = [[(0, 1, 0)], [(40, 1, 0), (0, 3, 0), (333, 2, 2)], [(63, 1, 8), (40, 8, 8), (17, 3, 4), (0, 37, 0), (5, 0, 8)]]


def check(ctx, shape, ocfg, W64, lg, pool, n_pages, table, L, v, b, ys, window=None, shift=None, eight=True):
    """The round that ctx ran last, against float64, request by request."""
    logits, hidden = f64(ctx.logits_tensor(lg)), f64(ctx.recg_debug_buffer(0))
    t0 = y0 = 0
    for r in range(len(L)):
        n = v[r] + b[r]
        held = read(ctx, pool, n_pages, table[r], L[r] + n, shape.n_layers)
        see = _kv4.visible(L[r], v[r], b[r])
        if window:
            see = _kv8.window(see, _kv8.positions(L[r], v[r], b[r]), *window)
        see = np.concatenate([see, np.zeros((n, n), dtype=bool)], axis=1)
        ids = list(ys[y0:y0 + v[r]]) + [ocfg.mask_id()] * b[r]
        pos = L[r] + np.arange(n) + (0 if shift is None else shift[r])
        want, kv, h = orc.decoder_rows(ocfg, W64, ids, pos, see, held)
        assert np.abs(hidden[t0:t0 + n] - h).max() <= TOL * np.abs(h).max(), r
        assert np.abs(logits[t0:t0 + n] - want).max() <= TOL * np.abs(want).max(), r
        for l, pair in enumerate(kv):
            for got, full in zip(held[l], pair):
                new = full[L[r] + n:]
                # a row within TOL of the largest, and rounded to four digits (2^-4); what a block is too large for is 2^-18 of it
                err = TOL * np.abs(new).max() * (1 + 2.0 ** -4) + 2.0 ** -4 * np.abs(new) + 2.0 ** -18 * np.abs(held[l]).max()
                assert (np.abs(got[L[r]:] - new) <= (err if eight else 2 * TOL * np.abs(new).max())).all(), (l, r)
        t0, y0 = t0 + n, y0 + v[r]


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("flags", [0, binding.FLAG_SIMT_GEMM, binding.FLAG_SIMT_ATTENTION, binding.FLAG_CHAIN, binding.FLAG_FOLD_NORM])
@pytest.mark.parametrize("reqs", REQS)
def test_round(head_dim, flags, reqs):
    shape, W, ocfg, W64 = model(head_dim)
    L, v, b = (list(x) for x in zip(*reqs))
    desc = synth.fixed_descriptor(L, v, b, seed=9)
    ys = synth.token_ids(sum(v), shape.vocab, seed=4).tolist()
    T, nkv = desc.n_tokens, shape.n_kv_heads
    rows = []
    for kind in (0, EIGHT):
        ctx = binding.Context(binding.make_config(shape, 8, 128, desc.page_table.shape[1], flags | kind), W)
        pool = binding.alloc_kv_pool(ctx, desc.n_pages, fill=None)
        pool.view(torch.uint8).fill_(255)                                  # NaN wherever nothing is written
        fill(ctx, pool, desc.n_pages, shape, L, desc.page_table, 11)
        batch = binding.Batch(L, v, b, ys, desc.page_table, pool, desc.n_pages)
        lg = ctx.recg_step(batch)
        ctx.recg_sync()
        k, w = (torch.empty((T, nkv, head_dim), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        ctx.recg_kv_rows(None, 0, k, w)
        rows.append((k.cpu(), w.cpu()))
        if kind:
            check(ctx, shape, ocfg, W64, lg, pool, desc.n_pages, desc.page_table, L, v, b, ys)
            o = torch.empty((T, shape.n_q_heads, head_dim), dtype=torch.bfloat16, device="cuda")
            ctx.recg_attention(None, shape.n_layers - 1, ctx.recg_debug_buffer(2).view_as(o), o)
            assert torch.equal(o.view(T, -1), ctx.recg_debug_buffer(1))   # the round's attention is the operator
        ctx.recg_sync()
        ctx.recg_free()
    t = 0
    for r, n in enumerate(int(x) for x in desc.rows):
        front = synth.kv_values(L[r], nkv, head_dim, seed=11 + 100 * r) if L[r] else (torch.zeros((0, nkv, head_dim)),) * 2
        for plain, coded, f in zip(*rows, front):
            assert torch.equal(coded[t:t + n], _kv8.Cache(nkv, head_dim).write(0, f).write(L[r], plain[t:t + n]).bf16(L[r], n))
        t += n


@pytest.mark.parametrize("eight", [0, EIGHT])
@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("flags", [0, binding.FLAG_SIMT_ATTENTION, binding.FLAG_CHAIN])
@pytest.mark.parametrize("window", [(4, 30), (0, 5), (70, 100)])
def test_round_with_a_window(head_dim, flags, window, eight):
    shape, W, ocfg, W64 = model(head_dim)
    L, v, b = (list(x) for x in zip(*REQS[2]))
    L[1], L[2] = 400, 250
    desc = synth.fixed_descriptor(L, v, b, seed=9)
    ys = synth.token_ids(sum(v), shape.vocab, seed=4).tolist()
    ctx = binding.Context(binding.make_config(shape, 8, 128, desc.page_table.shape[1], flags | eight), W)
    pool = binding.alloc_kv_pool(ctx, desc.n_pages, fill=None)
    pool.view(torch.uint8).fill_(255)
    fill(ctx, pool, desc.n_pages, shape, L, desc.page_table, 11)
    shift = [3, 0, 1000, 0, 1]                            # rotary positions move, what the rows see does not
    ctx.recg_kv_shift(shift)
    ctx.recg_window(*window)
    lg = ctx.recg_step(binding.Batch(L, v, b, ys, desc.page_table, pool, desc.n_pages))
    ctx.recg_sync()
    check(ctx, shape, ocfg, W64, lg, pool, desc.n_pages, desc.page_table, L, v, b, ys, window, shift, eight=bool(eight))
    w = torch.zeros((shape.n_layers, desc.n_pages, shape.n_kv_heads, 16), device="cuda")
    with pytest.raises(binding.RecgError, match="window|8 bits"):
        ctx.recg_kv_track(w)
    if not eight:
        ctx.recg_window(0, 0)
        ctx.recg_kv_track(w)
        with pytest.raises(binding.RecgError, match="gathered"):
            ctx.recg_window(4, 30)
        ctx.recg_window(0, 0)
    ctx.recg_sync()
    ctx.recg_free()


@pytest.mark.parametrize("window", [None, (4, 60)])
@pytest.mark.parametrize("flags", [0, EIGHT])
def test_device_rounds(flags, window):
    """A device-resident round over the same rows: the same K/V and logits as the round that the host lays out, and the next one on top."""
    if not flags and not window:
        pytest.skip("as ever")
    shape, W, ocfg, W64 = model(128)
    L, v, b = [20, 133, 0], [3, 1, 9], [4, 8, 0]
    pt, n_pages = synth.page_tables(L, [60] * 3, 16, seed=5)
    ys = [synth.token_ids(n, shape.vocab, seed=60 + n).tolist() for n in v]
    flat = [t for y in ys for t in y]
    out = []
    for device in (False, True):
        ctx = binding.Context(binding.make_config(shape, 4, 128, pt.shape[1], flags), W)
        pool = binding.alloc_kv_pool(ctx, n_pages, fill=None)
        pool.view(torch.uint8).fill_(255)
        fill(ctx, pool, n_pages, shape, L, pt, 11)
        if window:
            ctx.recg_window(*window)
        if device:
            db = binding.DeviceBatch(L, v, b, ys, 16, pt, pool, n_pages, rows_hint=32)
            lg = ctx.recg_step_device(db)
        else:
            lg = ctx.recg_step(binding.Batch(L, v, b, flat, pt, pool, n_pages))
        ctx.recg_sync()
        if not device:
            check(ctx, shape, ocfg, W64, lg, pool, n_pages, pt, L, v, b, flat, window, eight=bool(flags))
        out.append((f64(ctx.logits_tensor(lg))[:sum(v) + sum(b)], [read(ctx, pool, n_pages, pt[r], L[r] + v[r] + b[r], 1)[0] for r in range(3)]))
        if device:
            ctx.recg_verify_device()
            ctx.recg_next_round(db, 0)
            ctx.recg_sync()
            before = pool.clone()                       # a round that is refused on the device writes nothing
            ctx.recg_step_device(binding.DeviceBatch([20, 10 ** 9, 0], v, b, ys, 16, pt, pool, n_pages, rows_hint=32))
            with pytest.raises(RuntimeError):
                ctx.recg_sync()
            torch.cuda.synchronize()
            assert torch.equal(before.view(torch.uint8), pool.view(torch.uint8))
            lg = ctx.recg_step_device(db)
            ctx.recg_sync()
            L2, v2, b2 = (t.cpu().tolist() for t in (db.ctx_len, db.verify_len, db.block_size))
            ys2 = [db.verify_tokens[r, :v2[r]].cpu().tolist() for r in range(3)]
            check(ctx, shape, ocfg, W64, lg, pool, n_pages, pt, L2, v2, b2, [t for y in ys2 for t in y], window, eight=bool(flags))
        ctx.recg_free()
    (la, ra), (lb, rb) = out
    assert np.abs(la - lb).max() <= TOL * np.abs(la).max()
    for x, y in zip(ra, rb):
        for s, t in zip(x, y):
            assert np.array_equal(s, t)


def test_refusals():
    shape, W, _, _ = model(64)
    ctx = binding.Context(binding.make_config(shape, 2, 32, 8, EIGHT), W)
    pool = binding.alloc_kv_pool(ctx, 8)
    w = torch.zeros((shape.n_layers, 8, 2, 16), device="cuda")
    with pytest.raises(binding.RecgError, match="8 bits"):
        ctx.recg_kv_track(w)
    ctx.recg_kv_track(None)
    with pytest.raises(binding.RecgError, match="16-byte"):
        ctx.recg_step(binding.Batch([0], [1], [0], [3], np.zeros((1, 1)), pool.view(-1)[4:], 7))
    with pytest.raises(binding.RecgError, match="named twice"):        # two requests' rows into one page
        ctx.recg_step(binding.Batch([16, 17], [1, 1], [0, 0], [3, 4], np.array([[0, 2], [1, 2]]), pool, 8))
    ctx.recg_step(binding.Batch([16, 16], [1, 1], [0, 0], [3, 4], np.array([[0, 3], [0, 2]]), pool, 8))      # one that both read
    ctx.recg_sync()
    ctx.recg_free()
