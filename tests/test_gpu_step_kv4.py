"""Whole rounds over a cache in 4 bits, and eviction around rounds: step, gathered weight, choice, move, shift of the rotation, step.

The oracle gets the pool's own rows (read back after the round) as its K/V, so that a code which falls on the other side of a rounding
boundary costs nothing; the new rows' codes are checked by themselves: bit by bit in the first layer, whose input both kinds of pool share,
and within half a step and the round's own tolerance in the others."""
import numpy as np
import pytest
import torch

from oracle import recg_oracle as orc
from paper_2609_34388_b200 import binding, synth
from tests import _kv4
from tests._util import f64, oracle_cfg, oracle_weights

pytestmark = pytest.mark.gpu

TOL = 2e-2      # hidden states, logits and rows against float64, relative to the largest: the tolerance of the rounds over bf16
FOUR = binding.FLAG_KV_4BIT
SHAPES = {64: synth.tiny_shape(),
          128: synth.ModelShape(n_layers=3, hidden=256, n_q_heads=6, n_kv_heads=2, head_dim=128, ffn=512, vocab=1024, rope_base=10000.0)}


def model(head_dim):
    shape = SHAPES[head_dim]
    W = synth.model_weights(shape, seed=0, dtype=torch.bfloat16)
    synth.perturb_norm_gains(W)
    dev = {k: ([t.cuda() for t in v] if isinstance(v, list) else v.cuda()) for k, v in W.items()}
    return shape, dev, oracle_cfg(shape), oracle_weights(W)


def read(ctx, pool, n_pages, table, n, layers):
    return [tuple(f64(t) for t in ctx.recg_kv_read(pool, n_pages, l, table, 0, n)) for l in range(layers)]


def check(ctx, shape, ocfg, W64, lg, pool, n_pages, table, L, v, b, ys, shift=None, four=True):
    """The round that ctx ran last, against float64, request by request."""
    logits, hidden = f64(ctx.logits_tensor(lg)), f64(ctx.recg_debug_buffer(0))
    t0 = y0 = 0
    for r in range(len(L)):
        n = v[r] + b[r]
        held = read(ctx, pool, n_pages, table[r], L[r] + n, shape.n_layers)
        see = np.concatenate([_kv4.visible(L[r], v[r], b[r]), np.zeros((n, n), dtype=bool)], axis=1)
        ids = list(ys[y0:y0 + v[r]]) + [ocfg.mask_id()] * b[r]
        pos = L[r] + np.arange(n) + (0 if shift is None else shift[r])
        want, kv, h = orc.decoder_rows(ocfg, W64, ids, pos, see, held)
        assert np.abs(hidden[t0:t0 + n] - h).max() <= TOL * np.abs(h).max(), r
        assert np.abs(logits[t0:t0 + n] - want).max() <= TOL * np.abs(want).max(), r
        for l, pair in enumerate(kv):
            for got, full in zip(held[l], pair):
                new = full[L[r] + n:]
                # a row within TOL of the largest: its ends move by that, so its step by 2 TOL / 15, and 7.5 steps are half its range;
                # the step and the value read are rounded to bf16 (2^-8 each, of 15 steps and of the value)
                span = new.max(-1, keepdims=True) - new.min(-1, keepdims=True)
                err = 3 * TOL * np.abs(new).max() + span / 30 + 2.0 ** -8 * (span + np.abs(new))
                assert (np.abs(got[L[r]:] - new) <= (err if four else 2 * TOL * np.abs(new).max())).all(), (l, r)
        t0, y0 = t0 + n, y0 + v[r]


def fill(ctx, pool, n_pages, shape, L, table, seed):
    for r, n in enumerate(L):
        for l in range(shape.n_layers):
            if n:
                k, v = synth.kv_values(n, shape.n_kv_heads, shape.head_dim, seed=seed + 100 * r + l)
                ctx.recg_kv_write(pool, n_pages, l, table[r], 0, k.cuda(), v.cuda())


@pytest.mark.parametrize("head_dim", [64, 128])
@pytest.mark.parametrize("flags", [0, binding.FLAG_SIMT_GEMM, binding.FLAG_SIMT_ATTENTION, binding.FLAG_CHAIN, binding.FLAG_FOLD_NORM])
@pytest.mark.parametrize("reqs", [[(0, 1, 0)], [(40, 1, 0), (0, 3, 0), (333, 2, 2)], [(63, 1, 8), (40, 8, 8), (17, 3, 4), (0, 37, 0), (5, 0, 8)]])
def test_round(head_dim, flags, reqs):
    shape, W, ocfg, W64 = model(head_dim)
    L, v, b = (list(x) for x in zip(*reqs))
    desc = synth.fixed_descriptor(L, v, b, seed=9)
    ys = synth.token_ids(sum(v), shape.vocab, seed=4).tolist()
    rows = []
    for kind in (0, FOUR):
        ctx = binding.Context(binding.make_config(shape, 8, 128, desc.page_table.shape[1], flags | kind), W)
        pool = binding.alloc_kv_pool(ctx, desc.n_pages, fill=None)
        pool.view(torch.uint8).fill_(255)                                  # NaN wherever nothing is written
        fill(ctx, pool, desc.n_pages, shape, L, desc.page_table, 11)
        batch = binding.Batch(L, v, b, ys, desc.page_table, pool, desc.n_pages)
        lg = ctx.recg_step(batch)
        ctx.recg_sync()
        T = desc.n_tokens
        k, w = (torch.empty((T, shape.n_kv_heads, shape.head_dim), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        ctx.recg_kv_rows(None, 0, k, w)
        rows.append((k, w))
        if kind:
            check(ctx, shape, ocfg, W64, lg, pool, desc.n_pages, desc.page_table, L, v, b, ys)
            o = torch.empty((T, shape.n_q_heads, shape.head_dim), dtype=torch.bfloat16, device="cuda")
            ctx.recg_attention(None, shape.n_layers - 1, ctx.recg_debug_buffer(2).view_as(o), o)
            assert torch.equal(o.view(T, -1), ctx.recg_debug_buffer(1))   # the round's attention is the operator
        ctx.recg_sync()
        ctx.recg_free()
    for plain, coded in zip(*rows):
        assert torch.equal(coded.cpu(), _kv4.values_bf16(plain.cpu()))


@pytest.mark.parametrize("flags", [0, FOUR])
@pytest.mark.parametrize("head_dim", [64, 128])
def test_rounds_with_eviction(flags, head_dim):
    """Two rounds that gather, one eviction, one round behind it; the third request's pages go to new ones, the others stay in place."""
    shape, W, ocfg, W64 = model(head_dim)
    nl, nkv, group = shape.n_layers, shape.n_kv_heads, shape.n_q_heads // shape.n_kv_heads
    L, room = [0, 90, 250], 150
    pt, n_pages = synth.page_tables(L, [room] * 3, 16, seed=5)
    ctx = binding.Context(binding.make_config(shape, 4, 128, pt.shape[1], flags), W)
    pool = binding.alloc_kv_pool(ctx, n_pages, fill=None)
    pool.view(torch.uint8).fill_(255)
    fill(ctx, pool, n_pages, shape, L, pt, 11)
    weights = torch.zeros((nl, n_pages, nkv, 16), device="cuda")
    decay = 0.5
    ctx.recg_kv_track(weights, decay)
    expect = 0.0
    for number, (v, b) in enumerate([([60, 1, 4], [0, 8, 0]), ([1, 9, 3], [4, 0, 8])]):
        ys = synth.token_ids(sum(v), shape.vocab, seed=40 + number).tolist()
        before = weights.clone()
        lg = ctx.recg_step(binding.Batch(L, v, b, ys, pt, pool, n_pages))
        check(ctx, shape, ocfg, W64, lg, pool, n_pages, pt, L, v, b, ys, four=bool(flags))
        # the last layer's weights are those of the operator on the round's own queries
        q = ctx.recg_debug_buffer(2).view(-1, shape.n_q_heads, head_dim)
        o, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
        ctx.recg_attention(None, nl - 1, q, o, lse)
        row_weight = torch.tensor([x for r in range(3) for x in [1.0] * v[r] + [0.0] * b[r]], device="cuda")
        again = before.clone()
        ctx.recg_kv_weights(None, nl - 1, q, lse, again, again, row_weight, decay)
        ctx.recg_sync()
        assert torch.equal(again[nl - 1], weights[nl - 1])
        # a verify row gives 1 per query head, and what was there is scaled; a probability is off by what _kv4.gathered() allows it
        expect = decay * expect + sum(v) * group
        most = max(np.abs(read(ctx, pool, n_pages, pt[r], L[r] + v[r] + b[r], nl)[nl - 1][0]).max() for r in range(3))
        size = np.abs(f64(q)).sum(-1).max() * most / np.sqrt(head_dim)
        np.testing.assert_allclose(f64(weights[nl - 1].double().sum((0, 2))), expect, rtol=3 * size * 2.0 ** -19 + 2.0 ** -13)
        L = [n + x for n, x in zip(L, v)]                                  # all drafts taken
    ctx.recg_kv_track(None)

    budget = [33, 70, 100]
    keep = torch.empty((nl, 3, nkv, 100), dtype=torch.int32, device="cuda")
    held = [read(ctx, pool, n_pages, pt[r], L[r], nl) for r in range(3)]
    ev = binding.Eviction(L, budget, pt, pool, n_pages, weights, 2, 16, layers=(0, nl))
    ctx.recg_kv_select(ev, keep)
    ctx.recg_kv_compact(ev, keep)
    ctx.recg_sync()
    keep = keep.cpu().numpy()
    for r in range(3):
        for l, (k, w) in enumerate(read(ctx, pool, n_pages, pt[r], budget[r], nl)):
            for h in range(nkv):
                ids = keep[l, r, h, :budget[r]]
                assert np.array_equal(k[:, h], held[r][l][0][ids, h]) and np.array_equal(w[:, h], held[r][l][1][ids, h])
                assert ids[:2].tolist() == [0, 1] and ids[-16:].tolist() == list(range(L[r] - 16, L[r]))
    shift = [n - int(k) for n, k in zip(L, ev.kept)]
    ctx.recg_kv_shift(shift)
    L = [int(x) for x in ev.kept]
    v, b = [1, 5, 2], [8, 0, 3]
    ys = synth.token_ids(sum(v), shape.vocab, seed=50).tolist()
    lg = ctx.recg_step(binding.Batch(L, v, b, ys, pt, pool, n_pages))
    check(ctx, shape, ocfg, W64, lg, pool, n_pages, pt, L, v, b, ys, shift, four=bool(flags))
    # fewer entries than requests: the others are not shifted; none: nothing is
    ctx.recg_kv_shift(shift[:1])
    lg = ctx.recg_step(binding.Batch(L, v, b, ys, pt, pool, n_pages))
    check(ctx, shape, ocfg, W64, lg, pool, n_pages, pt, L, v, b, ys, [shift[0], 0, 0], four=bool(flags))
    ctx.recg_kv_shift([])
    lg = ctx.recg_step(binding.Batch(L, v, b, ys, pt, pool, n_pages))
    check(ctx, shape, ocfg, W64, lg, pool, n_pages, pt, L, v, b, ys, four=bool(flags))
    ctx.recg_free()


@pytest.mark.parametrize("flags", [0, FOUR])
def test_device_rounds(flags):
    """A device-resident round over the same rows: the same K/V, weights and logits as the round that the host lays out."""
    shape, W, ocfg, W64 = model(128)
    nl = shape.n_layers
    L, v, b = [20, 133, 0], [3, 1, 9], [4, 8, 0]
    shift = [0, 700, 5]
    pt, n_pages = synth.page_tables(L, [40] * 3, 16, seed=5)
    ys = [synth.token_ids(n, shape.vocab, seed=60 + n).tolist() for n in v]
    flat = [t for y in ys for t in y]
    out = []
    for device in (False, True):
        ctx = binding.Context(binding.make_config(shape, 4, 128, pt.shape[1], flags), W)
        pool = binding.alloc_kv_pool(ctx, n_pages, fill=None)
        pool.view(torch.uint8).fill_(255)
        fill(ctx, pool, n_pages, shape, L, pt, 11)
        weights = torch.zeros((nl, n_pages, shape.n_kv_heads, 16), device="cuda")
        ctx.recg_kv_track(weights)
        ctx.recg_kv_shift(shift)
        if device:
            lg = ctx.recg_step_device(binding.DeviceBatch(L, v, b, ys, 16, pt, pool, n_pages, rows_hint=32))
        else:
            lg = ctx.recg_step(binding.Batch(L, v, b, flat, pt, pool, n_pages))
        ctx.recg_sync()
        if not device:
            check(ctx, shape, ocfg, W64, lg, pool, n_pages, pt, L, v, b, flat, shift, four=bool(flags))
        out.append((f64(ctx.logits_tensor(lg))[:sum(v) + sum(b)], f64(weights),
                    [read(ctx, pool, n_pages, pt[r], L[r] + v[r] + b[r], 1)[0] for r in range(3)]))
        if device:                                     # a round that is refused on the device gathers nothing
            before = weights.clone()
            bad = binding.DeviceBatch([20, 10 ** 9, 0], v, b, ys, 16, pt, pool, n_pages, rows_hint=32)
            ctx.recg_step_device(bad)
            with pytest.raises(RuntimeError):
                ctx.recg_sync()
            torch.cuda.synchronize()
            assert torch.equal(before, weights)
        ctx.recg_free()
    (la, wa, ra), (lb, wb, rb) = out
    assert np.abs(la - lb).max() <= TOL * np.abs(la).max()
    assert np.abs(wa - wb).max() <= TOL * wa.max()
    for x, y in zip(ra, rb):
        for s, t in zip(x, y):
            assert np.array_equal(s, t)


def test_refusals():
    shape, W, _, _ = model(64)
    ctx = binding.Context(binding.make_config(shape, 2, 32, 8, FOUR), W)
    pool = binding.alloc_kv_pool(ctx, 8)
    w = torch.zeros((shape.n_layers, 8, 2, 16), device="cuda")
    for call in (lambda: ctx.recg_kv_track(w, -1.0), lambda: ctx.recg_kv_track(w, float("nan")), lambda: ctx.recg_kv_track(w, float("inf")),
                 lambda: ctx.recg_kv_track(w.view(-1)[1:]), lambda: ctx.recg_kv_shift([1, 2, 3]), lambda: ctx.recg_kv_shift([-1]),
                 lambda: ctx.recg_kv_shift([2 ** 30 + 1]),
                 lambda: ctx.recg_step(binding.Batch([0], [1], [0], [3], np.zeros((1, 1)), pool.view(-1)[4:], 7))):
        with pytest.raises(RuntimeError):
            call()
    with pytest.raises(RuntimeError):
        bare = binding.Context(binding.make_config(shape, 2, 32, 8, FOUR))
        bare.recg_kv_track(w)
    ctx.recg_kv_track(w)
    with pytest.raises(ValueError, match="batch's pool"):              # weights of another pool
        ctx.recg_step(binding.Batch([0], [1], [0], [3], np.zeros((1, 1)), binding.alloc_kv_pool(ctx, 9), 9))
    for pages in ([[0, 1], [0, 2]], [[0, 0], [1, 2]]):                 # a page that two requests name, or one twice
        with pytest.raises(binding.RecgError, match="named twice"):
            ctx.recg_step(binding.Batch([16, 16], [1, 1], [0, 0], [3, 4], np.array(pages), pool, 8))
    ctx.recg_step(binding.Batch([16, 16], [1, 1], [0, 0], [3, 4], np.array([[0, 3], [1, 2]]), pool, 8))
    ctx.recg_sync()
    ctx.recg_free()
