"""The 4-bit pool: what goes in and comes out, at its borders, against the definition in float64 (bit for bit: both sides round the
same exact value once), and the rows of a batch for both kinds of pool."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2609_34388_b200 import binding, synth
from tests import _kv4

pytestmark = pytest.mark.gpu


def make(n_kv, head_dim, stride, max_tokens=32, max_req=1, flags=binding.FLAG_KV_4BIT, layers=2):
    shape = synth.ModelShape(n_layers=layers, hidden=64, n_q_heads=2 * n_kv, n_kv_heads=n_kv, head_dim=head_dim, ffn=64, vocab=64)
    return binding.Context(binding.make_config(shape, max_req, max_tokens, stride, flags))


def pool_bytes(pool):
    return pool.view(torch.uint8)


@pytest.mark.parametrize("head_dim,n_kv", [(64, 2), (128, 1), (128, 8)])
@pytest.mark.parametrize("pos0,n_pos", [(0, 1), (1, 1), (5, 16), (15, 2), (37, 403), (3, 2000), (7, 14400)])
def test_positions_round_trip(head_dim, n_kv, pos0, n_pos):
    pt, n_pages = synth.page_tables([pos0], [n_pos + 1], 16, seed=n_pos, spare_pages=3)
    ctx = make(n_kv, head_dim, pt.shape[1])
    assert ctx.kv_pool_bytes(n_pages) == 2 * n_pages * n_kv * (16 * head_dim + 128)
    pool = binding.alloc_kv_pool(ctx, n_pages)
    k, v = synth.kv_values(n_pos, n_kv, head_dim, seed=n_pos + 1, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(n_pos)
    pool_bytes(pool).random_(0, 256, generator=g)
    before = pool_bytes(pool).clone()
    ctx.recg_kv_write(pool, n_pages, 1, pt[0], pos0, k, v)
    changed = (pool_bytes(pool) != before).nonzero()[:, 0]
    assert changed.numel() <= n_pos * n_kv * (head_dim + 8) and int(changed.min()) >= before.numel() // 2
    block = 16 * head_dim + 128                                          # ... and in pages of the request only
    pages = set(((changed - before.numel() // 2) // (block * n_kv)).unique().tolist())
    assert pages <= set(pt[0][pos0 // 16:(pos0 + n_pos - 1) // 16 + 1].tolist())
    kb, vb = ctx.recg_kv_read(pool, n_pages, 1, pt[0], pos0, n_pos)
    assert torch.equal(kb.cpu(), _kv4.values_bf16(k)) and torch.equal(vb.cpu(), _kv4.values_bf16(v))
    for i in {0, n_pos // 2, n_pos - 1}:                                 # one position alone, both halves of a token pair
        kb, vb = ctx.recg_kv_read(pool, n_pages, 1, pt[0], pos0 + i, 1)
        assert torch.equal(kb[0].cpu(), _kv4.values_bf16(k[i])) and torch.equal(vb[0].cpu(), _kv4.values_bf16(v[i]))
    # written again one by one (the halves of a pair by different calls): the same bytes
    if n_pos <= 16:
        whole = pool_bytes(pool).clone()
        pool_bytes(pool).copy_(before)
        for i in reversed(range(n_pos)):
            ctx.recg_kv_write(pool, n_pages, 1, pt[0], pos0 + i, k[i:i + 1], v[i:i + 1])
        assert torch.equal(pool_bytes(pool), whole)
    ctx.recg_sync()
    ctx.recg_free()


@pytest.mark.parametrize("pos0,n_pos", [(9, 14336 - 9), (9, 14336), (9, 64000 - 9), (9, 64000), (15, 130000)])
def test_long_ranges(pos0, n_pos):
    """Ranges that take as many page ids as a launch carries, one more, and several launches."""
    pt, n_pages = synth.page_tables([pos0], [n_pos + 1], 16, seed=3, spare_pages=3)
    ctx = make(1, 64, pt.shape[1])
    pool = binding.alloc_kv_pool(ctx, n_pages)
    k, v = synth.kv_values(n_pos, 1, 64, seed=7, device="cuda")
    ctx.recg_kv_write(pool, n_pages, 1, pt[0], pos0, k, v)
    kb, vb = ctx.recg_kv_read(pool, n_pages, 1, pt[0], pos0, n_pos)
    assert torch.equal(kb.cpu(), _kv4.values_bf16(k)) and torch.equal(vb.cpu(), _kv4.values_bf16(v))
    ctx.recg_sync()
    ctx.recg_free()


def special_rows(d):
    """Rows on the format's borders, [rows, d] bf16."""
    bf = lambda t: torch.as_tensor(t, dtype=torch.float64).float().bfloat16()
    i = torch.arange(d, dtype=torch.float64)
    g = torch.Generator().manual_seed(1)
    rows = [torch.zeros(d), torch.full((d,), -3.5), i % 16,                      # constants; the codes themselves
            (i % 31) / 2, (i % 61) / 4 - 7,                                       # ties: half steps
            torch.where(i == d - 1, 1e30, 1.0), torch.where(i == 3, -3e38, 2.0),  # one value far out
            torch.where(i % 2 == 0, 3e38, -3e38),                                 # a range that overflows
            torch.where(i == 5, float("inf"), 1.0), torch.where(i == 6, float("-inf"), 1.0), torch.where(i == 7, float("nan"), 1.0),
            -1.0 + torch.where(i == 0, 0.0, 1.0 + 2.0 ** -20 * (i % 7)),          # tiny values next to one that is not
            torch.where(i % 3 == 0, -1.0, torch.where(i % 3 == 1, 2.0 ** -22, 1.0)),
            1e-37 * i, 1e-30 * i, 100.0 + (i % 4)]
    rows += [torch.randn(d, generator=g, dtype=torch.float64) * 10.0 ** e for e in (-20, -3, 0, 3, 20)]
    rows += [torch.round(torch.randn(d, generator=g, dtype=torch.float64) * 4) / 2 for _ in range(40)]    # coarse grids: many ties
    return torch.stack([bf(r) for r in rows])


@pytest.mark.parametrize("d", [64, 128])
def test_rows_on_the_borders(d):
    rows = special_rows(d)
    n = rows.shape[0]
    pt, n_pages = synth.page_tables([0], [n], 16, seed=5)
    ctx = make(2, d, pt.shape[1])
    pool = binding.alloc_kv_pool(ctx, n_pages)
    k = torch.stack([rows, rows.flip(0)], 1).cuda()
    v = torch.stack([rows.roll(3, 0), rows.roll(7, 0)], 1).cuda()
    ctx.recg_kv_write(pool, n_pages, 0, pt[0], 0, k, v)
    for got, x in zip(ctx.recg_kv_read(pool, n_pages, 0, pt[0], 0, n), (k, v)):
        want = _kv4.values_bf16(x)
        assert torch.equal(torch.isnan(got.cpu()), torch.isnan(want))
        # below the smallest normal number the kernels' arithmetic has zeros
        diff = (got.cpu().double() - want.double()).abs().nan_to_num(0)
        assert float(diff.max()) <= 2.0 ** -126, diff.amax((1, 2))
        held, src = _kv4.values(x), x.cpu().double().numpy()
        _, s, _ = _kv4.codes(x)
        ok = np.isfinite(held)
        # half a step, the rounding of the step (15 s 2^-8 at most where s was rounded down and the top level falls short of the maximum)
        assert (np.abs(held - src)[ok] <= (np.broadcast_to(s, held.shape) * (0.5 + 15 * 2.0 ** -8) + 2.0 ** -114)[ok]).all()
    ctx.recg_sync()
    ctx.recg_free()


@pytest.mark.parametrize("flags", [0, binding.FLAG_KV_4BIT])
@pytest.mark.parametrize("head_dim,n_kv", [(64, 2), (128, 8)])
@pytest.mark.parametrize("reqs", [[(0, 1, 0)], [(31, 1, 0)], [(16, 0, 5), (0, 40, 3), (255, 1, 1)], [(7 * i, 1, 0) for i in range(70)]])
def test_rows_of_a_batch(flags, head_dim, n_kv, reqs):
    """Appended rows lie where a write of their positions puts them, whatever their stride, and come back."""
    L, vl, b = map(list, zip(*reqs))
    desc = synth.fixed_descriptor(L, vl, b, seed=3)
    T = desc.n_tokens
    ctx = make(n_kv, head_dim, desc.page_table.shape[1], max_tokens=T, max_req=len(reqs), flags=flags)
    pool = binding.alloc_kv_pool(ctx, desc.n_pages)
    wide = torch.randn((T, 3 * n_kv + 1, head_dim), device="cuda").bfloat16()
    k, v = wide[:, n_kv:2 * n_kv], wide[:, 2 * n_kv:3 * n_kv]
    batch = binding.Batch(L, vl, b, None, desc.page_table, pool, desc.n_pages)
    ctx.recg_kv_append(batch, 1, k, v)
    other = torch.zeros_like(pool)
    t = 0
    for r, n in enumerate(desc.rows):
        ctx.recg_kv_write(other, desc.n_pages, 1, desc.page_table[r], L[r], k[t:t + n].contiguous(), v[t:t + n].contiguous())
        t += n
    assert torch.equal(pool_bytes(pool), pool_bytes(other))
    out = torch.full_like(wide, 9.0)
    ctx.recg_kv_rows(None, 1, out[:, :n_kv], out[:, n_kv + 1:2 * n_kv + 1])
    want = [_kv4.values_bf16(x) if flags else x.cpu() for x in (k, v)]
    assert torch.equal(out[:, :n_kv].cpu(), want[0]) and torch.equal(out[:, n_kv + 1:2 * n_kv + 1].cpu(), want[1])
    assert (out[:, n_kv] == 9.0).all() and (out[:, 2 * n_kv + 1:] == 9.0).all()
    again = ctx.recg_kv_rows(batch, 1)
    assert torch.equal(again[0].cpu(), want[0]) and torch.equal(again[1].cpu(), want[1])
    ctx.recg_sync()
    ctx.recg_free()


def test_refusals_of_the_row_operations():
    ctx = make(2, 64, 4, max_tokens=8, max_req=2)
    pool = binding.alloc_kv_pool(ctx, 8)
    k = torch.zeros((2, 2, 64), dtype=torch.bfloat16, device="cuda")
    lib = binding.lib()
    with pytest.raises(ValueError):
        ctx.recg_kv_append(None, 0, k, k)                                    # two rows, and no batch before
    assert lib.recg_kv_append(ctx.h, None, 0, k.data_ptr(), k.data_ptr(), 0) == 1 and "laid out before" in lib.recg_last_error(ctx.h).decode()
    pt = np.array([[0, 1, 2, 3], [4, 5, 6, 7]])
    batch = binding.Batch([3, 9], [1, 1], [0, 0], None, pt, pool, 8)
    for layer in (-1, 2):
        with pytest.raises(binding.RecgError, match="layer"):
            ctx.recg_kv_append(batch, layer, k, k)
    bad = binding.Batch([3, 9], [1, 1], [0, 0], None, np.where(pt == 4, 8, pt), pool, 8)
    with pytest.raises(binding.RecgError, match="page id"):
        ctx.recg_kv_append(bad, 0, k, k)
    p = k.data_ptr()
    for kp, vp, stride in ((p + 2, p, 0), (p, p + 8, 0), (p, p, 127), (p, p, 132), (p, p, -128)):
        assert lib.recg_kv_append(ctx.h, C.byref(batch.c), 0, kp, vp, stride) == 1, (kp - p, vp - p, stride)
        assert lib.recg_kv_rows(ctx.h, C.byref(batch.c), 0, kp, vp, stride) == 1
    for t in (k.float(), k[:, :1], k[:1], k.cpu(), k.transpose(0, 1)):
        with pytest.raises(ValueError):
            ctx.recg_kv_append(batch, 0, t, t)
    ctx.recg_kv_append(batch, 0, k, k)
    ctx.recg_sync()
    ctx.recg_free()
