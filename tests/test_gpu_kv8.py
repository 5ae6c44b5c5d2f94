"""The 8-bit pool: what goes in and comes out against the definition in float64, bit for bit (both sides round the same exact value once),
blocks that fill up row by row, and the rows of a batch, rotated on the way or not, for every kind of pool."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2609_34388_b200 import binding, synth
from tests import _kv4, _kv8
from tests._util import f64

pytestmark = pytest.mark.gpu

KINDS = [0, binding.FLAG_KV_8BIT, binding.FLAG_KV_4BIT]
BASE = 500000.0


def make(n_kv, head_dim, stride, max_tokens=32, max_req=1, flags=binding.FLAG_KV_8BIT, layers=2, group=2):
    shape = synth.ModelShape(n_layers=layers, hidden=64, n_q_heads=group * n_kv, n_kv_heads=n_kv, head_dim=head_dim, ffn=64, vocab=64,
                             rope_base=BASE)
    return binding.Context(binding.make_config(shape, max_req, max_tokens, stride, flags))


def dirty_pool(ctx, n_pages, seed=1):
    pool = binding.alloc_kv_pool(ctx, n_pages, fill=None)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    pool.view(torch.uint8).random_(0, 256, generator=g)
    return pool


def same(got, want):
    """Bit for bit, NaN for NaN, -0 for 0."""
    got, want = got.cpu().double(), want.double()
    return torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(0), want.nan_to_num(0))


@pytest.mark.parametrize("head_dim,n_kv", [(64, 2), (128, 1), (128, 8)])
@pytest.mark.parametrize("pos0,n_pos", [(0, 1), (1, 1), (5, 16), (15, 2), (37, 403), (3, 2000), (7, 14400)])
def test_positions_round_trip(head_dim, n_kv, pos0, n_pos):
    pt, n_pages = synth.page_tables([pos0], [n_pos + 1], 16, seed=n_pos, spare_pages=3)
    ctx = make(n_kv, head_dim, pt.shape[1])
    layer = (n_pages * n_kv * (32 * head_dim + 8) + 127) // 128 * 128
    assert ctx.kv_pool_bytes(n_pages) == 2 * layer
    pool = dirty_pool(ctx, n_pages)
    k, v = synth.kv_values(pos0 + n_pos, n_kv, head_dim, seed=n_pos + 1, device="cuda")
    v = v * torch.exp(2 * torch.randn(v.shape[0], n_kv, 1, device="cuda")).to(v.dtype)
    if pos0:
        ctx.recg_kv_write(pool, n_pages, 1, pt[0], 0, k[:pos0], v[:pos0])
    raw = pool.view(torch.uint8)
    before = raw.clone()
    ctx.recg_kv_write(pool, n_pages, 1, pt[0], pos0, k[pos0:], v[pos0:])
    changed = (raw != before).nonzero()[:, 0] - layer
    assert int(changed.min()) >= 0                                       # the other layer stays
    codes = n_pages * n_kv * 32 * head_dim
    pages = set((changed[changed < codes] // (32 * head_dim * n_kv)).unique().tolist()) | \
        set(((changed[changed >= codes] - codes) // (8 * n_kv)).unique().tolist())
    assert pages <= set(pt[0][pos0 // 16:(pos0 + n_pos - 1) // 16 + 1].tolist())
    want = [_kv8.Cache(n_kv, head_dim).write(0, x[:pos0]).write(pos0, x[pos0:]) for x in (k, v)]
    for first, n in [(0, pos0 + n_pos), (pos0 + n_pos - 1, 1), (pos0, 1), (pos0 // 2, (n_pos + 1) // 2)]:
        for got, w in zip(ctx.recg_kv_read(pool, n_pages, 1, pt[0], first, n), want):
            assert same(got, w.bf16(first, n))
    ctx.recg_sync()
    ctx.recg_free()


@pytest.mark.parametrize("head_dim", [64, 128])
def test_a_block_fills_up_row_by_row(head_dim):
    """Rows that are larger, smaller, zero and none come one by one: what is there is rounded again whenever the exponent moves."""
    pt, n_pages = synth.page_tables([0], [40], 16, seed=4)
    ctx = make(2, head_dim, pt.shape[1])
    pool = dirty_pool(ctx, n_pages)
    g = torch.Generator().manual_seed(head_dim)
    x = torch.randn((40, 2, head_dim), generator=g) * torch.tensor([1.0, 300.0, 0.0, 1e-3, 1e5, 1.0, 1e9, 1e-30, 1.0, 1e4]).repeat(4)[:, None, None]
    x[5, 1, 3], x[9, 0, 7], x[33, 0, 1] = float("nan"), float("inf"), float("-inf")
    k, v = x.bfloat16(), x.flip(-1).roll(3, 0).bfloat16()
    want = [_kv8.Cache(2, head_dim), _kv8.Cache(2, head_dim)]
    for i in range(40):
        ctx.recg_kv_write(pool, n_pages, 0, pt[0], i, k[i:i + 1].cuda(), v[i:i + 1].cuda())
        for t, w in zip((k, v), want):
            w.write(i, t[i:i + 1])
        if i % 3 == 0 or i > 36:
            for got, w in zip(ctx.recg_kv_read(pool, n_pages, 0, pt[0], 0, i + 1), want):
                assert same(got, w.bf16(0, i + 1)), i
    # rows that were taken back: the exponent follows those that are left and the new ones
    for pos0, n in ((35, 2), (4, 3), (16, 1), (0, 5)):
        if pos0 > want[0].held.shape[0]:
            continue
        ctx.recg_kv_write(pool, n_pages, 0, pt[0], pos0, k[7:7 + n].cuda(), v[7:7 + n].cuda())
        for t, w in zip((k, v), want):
            w.write(pos0, t[7:7 + n])
        for got, w in zip(ctx.recg_kv_read(pool, n_pages, 0, pt[0], 0, pos0 + n), want):
            assert same(got, w.bf16(0, pos0 + n))
    ctx.recg_sync()
    ctx.recg_free()


@pytest.mark.parametrize("d", [64, 128])
def test_values_on_the_borders(d):
    """Powers of two and 448 times them, ties between codes, the smallest codes, the ends of bf16."""
    i = torch.arange(d, dtype=torch.float64)
    rows = [448.0 * 2.0 ** (i % 2), 450.0 + 0 * i, 1.75 * 2.0 ** (i % 9), (1 + (i % 32) / 32) * 16, torch.where(i == 0, 448.0, 2.0 ** -9 * (i % 17) / 2),
            torch.where(i == 0, 448.0, 2.0 ** -10), torch.where(i == 0, 448.0, 2.0 ** -6 * (1 + (i % 64) / 64)), torch.full((d,), 3.3895313892515355e38),
            torch.where(i == 1, 3.3e38, -2.9e38), 1e-38 * i, 2.0 ** -69 * (i % 5) / 2, 2.0 ** -60 * i, 0 * i, -0.0 * i]
    pt, n_pages = synth.page_tables([0], [16 * len(rows)], 16, seed=5)
    ctx = make(2, d, pt.shape[1])
    pool = dirty_pool(ctx, n_pages)
    x = torch.zeros((16 * len(rows), 2, d), dtype=torch.float64)
    for r, row in enumerate(rows):                       # a block of its own each, and all together in the second head
        x[16 * r, 0], x[16 * r + 15, 0] = row, -row / 2
        x[16 * r:16 * r + 16, 1] = torch.stack([rows[(r + j) % 7] for j in range(16)])
    k = x.float().bfloat16()
    v = k.flip(-1)
    ctx.recg_kv_write(pool, n_pages, 0, pt[0], 0, k.cuda(), v.cuda())
    for got, t in zip(ctx.recg_kv_read(pool, n_pages, 0, pt[0], 0, len(k)), (k, v)):
        want = _kv8.Cache(2, d).write(0, t).bf16(0, len(k))
        assert torch.isfinite(got).all()
        assert same(got, want), [int(r) // 16 for r in (got.cpu() != want).any(-1).any(-1).nonzero()[:, 0]]
    ctx.recg_sync()
    ctx.recg_free()


@pytest.mark.parametrize("pos0,n_pos", [(9, 14336 - 9), (9, 14336), (9, 64000 - 9), (9, 64000), (15, 130000)])
def test_long_ranges(pos0, n_pos):
    """Ranges that take as many page ids as a launch carries, one more, and several launches."""
    pt, n_pages = synth.page_tables([pos0], [n_pos + 1], 16, seed=3, spare_pages=3)
    ctx = make(1, 64, pt.shape[1])
    pool = dirty_pool(ctx, n_pages)
    k, v = synth.kv_values(pos0 + n_pos, 1, 64, seed=7, device="cuda")
    ctx.recg_kv_write(pool, n_pages, 1, pt[0], 0, k[:pos0], v[:pos0])
    ctx.recg_kv_write(pool, n_pages, 1, pt[0], pos0, k[pos0:], v[pos0:])
    for got, x in zip(ctx.recg_kv_read(pool, n_pages, 1, pt[0], pos0, n_pos), (k, v)):
        assert same(got, _kv8.Cache(1, 64).write(0, x[:pos0]).write(pos0, x[pos0:]).bf16(pos0, n_pos))
    ctx.recg_sync()
    ctx.recg_free()


REQS = [[(0, 1, 0)], [(31, 1, 0)], [(16, 0, 5), (0, 40, 3), (255, 1, 1)], [(7 * i, 1, 0) for i in range(70)],
        [(15, 33, 0), (1, 15, 1), (14, 2, 0), (15, 2, 0), (48, 16, 0), (0, 700, 0)], [(100 + i, 1 + i % 3, 0) for i in range(600)]]


@pytest.mark.parametrize("head_dim,n_kv", [(64, 2), (128, 8)])
@pytest.mark.parametrize("reqs", REQS)
def test_rows_of_a_batch(head_dim, n_kv, reqs):
    """Appended rows leave the bytes that a write of their positions leaves, whatever their stride, and come back."""
    L, vl, b = map(list, zip(*reqs))
    desc = synth.fixed_descriptor(L, vl, b, seed=3)
    T = desc.n_tokens
    ctx = make(n_kv, head_dim, desc.page_table.shape[1], max_tokens=T, max_req=len(reqs))
    pool = dirty_pool(ctx, desc.n_pages)
    for r, n in enumerate(L):
        k, v = synth.kv_values(n, n_kv, head_dim, seed=r, device="cuda") if n else (None, None)
        if n:
            ctx.recg_kv_write(pool, desc.n_pages, 1, desc.page_table[r], 0, k, 4 * v)
    other = pool.clone()
    wide = torch.randn((T, 3 * n_kv + 1, head_dim), device="cuda").bfloat16()
    k, v = wide[:, n_kv:2 * n_kv], wide[:, 2 * n_kv:3 * n_kv]
    batch = binding.Batch(L, vl, b, None, desc.page_table, pool, desc.n_pages)
    ctx.recg_kv_append(batch, 1, k, v)
    t = 0
    want = []
    for r, n in enumerate(desc.rows):
        ctx.recg_kv_write(other, desc.n_pages, 1, desc.page_table[r], L[r], k[t:t + n].contiguous(), v[t:t + n].contiguous())
        want.append(ctx.recg_kv_read(other, desc.n_pages, 1, desc.page_table[r], L[r], int(n)))
        t += n
    assert torch.equal(pool.view(torch.uint8), other.view(torch.uint8))
    out = torch.full_like(wide, 9.0)
    ctx.recg_kv_rows(None, 1, out[:, :n_kv], out[:, n_kv + 1:2 * n_kv + 1])
    assert torch.equal(out[:, :n_kv], torch.cat([w[0] for w in want])) and torch.equal(out[:, n_kv + 1:2 * n_kv + 1], torch.cat([w[1] for w in want]))
    assert (out[:, n_kv] == 9.0).all() and (out[:, 2 * n_kv + 1:] == 9.0).all()
    ctx.recg_sync()
    ctx.recg_free()


@pytest.mark.parametrize("flags", KINDS)
@pytest.mark.parametrize("heads", [(4, 2, 64), (32, 8, 128), (40, 8, 128), (6, 2, 64)])
@pytest.mark.parametrize("reqs,corr", [(r, None) for r in REQS[:5]] + [([(100, 8, 8), (0, 5, 4), (190003, 16, 7), (31, 2, 0)], [(1, 6), (4,), (3, 15), (1,)])])
def test_rotated_rows_of_a_batch(heads, flags, reqs, corr):
    """K and V lie where appending the rotated K leaves them, and q is rotated: to within its rounding, and K to the bit."""
    nq, nkv, d = heads
    if (nq + 2 * nkv) * d % 128:
        pytest.skip("the context asks for a qkv width of whole 128 columns")
    L, vl, b = map(list, zip(*reqs))
    corr = corr or [()] * len(reqs)
    desc = synth.fixed_descriptor(L, vl, b, seed=3, corr=[[(i, 5) for i in c] for c in corr], corr_block=b)
    T = desc.n_tokens
    ctx = make(nkv, d, desc.page_table.shape[1], max_tokens=T, max_req=len(reqs), flags=flags, group=nq // nkv)
    pool = dirty_pool(ctx, desc.n_pages)
    for r, n in enumerate(L):
        first = n // 16 * 16
        if n > first:
            k, v = synth.kv_values(n - first, nkv, d, seed=r, device="cuda")
            ctx.recg_kv_write(pool, desc.n_pages, 1, desc.page_table[r], first, k, v)
    other = pool.clone()
    p = np.concatenate([_kv8.positions(*reqs[r], corr[r], b[r]) for r in range(len(reqs))])
    wide = torch.randn((T, nq + 2 * nkv, d), device="cuda").bfloat16()
    q, k, v = wide[:, :nq], wide[:, nq:nq + nkv], wide[:, nq + nkv:]
    batch = binding.Batch(L, vl, b, None, desc.page_table, pool, desc.n_pages, **desc.branch_kwargs())
    out = torch.full((T + 1, nq, d), 9.0, dtype=torch.bfloat16, device="cuda")
    source = wide.clone()
    ctx.recg_kv_append_rotary(batch, 1, q, k, v, out[:T])
    assert torch.equal(wide, source) and (out[T] == 9.0).all()
    again = binding.Batch(L, vl, b, None, desc.page_table, other, desc.n_pages, **desc.branch_kwargs())
    ctx.recg_kv_append(again, 1, _kv8.rotated(k, p, BASE)[0].cuda(), v.contiguous())
    assert torch.equal(pool.view(torch.uint8), other.view(torch.uint8))
    # q: rounded to bf16 once (2^-8 with the tie), and before that sums of two products in 32 bits whose factors are rounded too
    _, want = _kv8.rotated(q, p, BASE)
    size = np.abs(f64(q)[..., :d // 2]) + np.abs(f64(q)[..., d // 2:])
    assert (np.abs(f64(out[:T]) - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -21 * np.concatenate([size, size], -1)).all()
    # q in place, and without q
    dense = q.contiguous()
    ctx.recg_kv_append_rotary(None, 1, dense, k, v, dense) if flags == 0 else ctx.recg_kv_append_rotary(batch, 1, dense, k, v, dense)
    assert torch.equal(dense, out[:T])
    fresh = pool.clone()
    ctx.recg_kv_append_rotary(batch, 1, None, k, v)
    assert torch.equal(pool.view(torch.uint8), fresh.view(torch.uint8))
    ctx.recg_sync()
    ctx.recg_free()


def test_rotation_follows_a_shift():
    """Positions that recg_kv_shift has moved, and angles of positions that are far out."""
    ctx = make(2, 128, 4, max_tokens=8, max_req=2, flags=0)
    pool = binding.alloc_kv_pool(ctx, 8)
    ctx.recg_kv_shift([1000000, 3])
    batch = binding.Batch([3, 20], [2, 1], [0, 1], None, np.arange(8).reshape(2, 4), pool, 8)
    x = torch.randn((4, 8, 128), device="cuda").bfloat16()
    k, v, q = x[:, :2].contiguous(), x[:, 2:4].contiguous(), x[:, 4:].contiguous()
    ctx.recg_kv_append_rotary(batch, 0, q, k, v, q)
    p = np.array([1000003, 1000004, 23, 24])
    assert torch.equal(ctx.recg_kv_rows(None, 0)[0].cpu(), _kv8.rotated(k, p, BASE)[0])
    want = _kv8.rotated(x[:, 4:], p, BASE)[1]
    assert (np.abs(f64(q) - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -20 * np.abs(f64(x)).max()).all()
    ctx.recg_sync()
    ctx.recg_free()


def test_refusals():
    lib = binding.lib()
    with pytest.raises(binding.RecgError, match="not both"):
        make(2, 64, 4, flags=binding.FLAG_KV_8BIT | binding.FLAG_KV_4BIT)
    ctx = make(2, 64, 4, max_tokens=8, max_req=2)
    pool = binding.alloc_kv_pool(ctx, 8)
    k = torch.zeros((2, 2, 64), dtype=torch.bfloat16, device="cuda")
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16, device="cuda")
    p = k.data_ptr()
    assert lib.recg_kv_append_rotary(ctx.h, None, 0, None, 0, None, p, p, 0) == 1 and "laid out before" in lib.recg_last_error(ctx.h).decode()
    pt = np.arange(8).reshape(2, 4)
    batch = binding.Batch([3, 9], [1, 1], [0, 0], None, pt, pool, 8)
    for layer in (-1, 2):
        with pytest.raises(binding.RecgError, match="layer"):
            ctx.recg_kv_append_rotary(batch, layer, q, k, k, q)
    at = q.data_ptr()
    b = C.byref(batch.c)
    for args in ((at, 0, None, p, p, 0), (None, 0, at, p, p, 0), (at, 0, at, None, p, 0), (at, 0, at, p, None, 0), (at + 2, 0, at, p, p, 0),
                 (at, 0, at + 8, p, p, 0), (at, 0, at, p + 2, p, 0), (at, 255, at, p, p, 0), (at, 260, at, p, p, 0), (at, 0, at, p, p, 127),
                 (at, 0, at, p, p, 132), (at, 0, at, p, p, -128), (at, -256, at, p, p, 0)):
        assert lib.recg_kv_append_rotary(ctx.h, b, 0, *args) == 1, args
    for bad in (q.float(), q[:, :2], q[:1], q.cpu(), q.transpose(0, 1)):
        with pytest.raises(ValueError):
            ctx.recg_kv_append_rotary(batch, 0, bad, k, k, q)
        with pytest.raises(ValueError):
            ctx.recg_kv_append_rotary(batch, 0, q, k, k, bad)
    with pytest.raises(ValueError):
        ctx.recg_kv_append_rotary(batch, 0, q, k, k)
    # a page that takes the rows of two requests, in appends of either kind; for reading and for attention it may be shared
    both = binding.Batch([3, 9], [1, 1], [0, 0], None, np.array([[0, 1, 2, 3], [0, 5, 6, 7]]), pool, 8)
    for call in (lambda: ctx.recg_kv_append(both, 0, k, k), lambda: ctx.recg_kv_append_rotary(both, 0, q, k, k, q), lambda: ctx.recg_kv_append(None, 0, k, k)):
        with pytest.raises(binding.RecgError, match="named twice"):
            call()
    ctx.recg_kv_write(pool, 8, 0, pt[0], 0, torch.zeros((10, 2, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((10, 2, 64), dtype=torch.bfloat16, device="cuda"))
    ctx.recg_kv_rows(both, 0)
    ctx.recg_attention(both, 0, q, torch.empty_like(q))
    # what there is not over 8 bits
    w = torch.zeros((2, 8, 2, 16), device="cuda")
    lse = torch.zeros((2, 4), device="cuda")
    with pytest.raises(binding.RecgError, match="8 bits"):
        ctx.recg_kv_weights(batch, 0, q, lse, None, w)
    ev = binding.Eviction([9, 9], [4, 4], pt, pool, 8, w, layers=(0, 2))
    keep = torch.zeros((2, 2, 2, 4), dtype=torch.int32, device="cuda")
    ctx.recg_kv_select(ev, keep)
    with pytest.raises(binding.RecgError, match="8 bits"):
        ctx.recg_kv_compact(ev, keep)
    off = binding.Batch([3, 9], [1, 1], [0, 0], None, pt, pool[4:], 8)
    with pytest.raises(binding.RecgError, match="16-byte"):
        ctx.recg_kv_append(off, 0, k, k)
    ctx.recg_kv_append_rotary(batch, 0, q, k, k, q)
    ctx.recg_sync()
    ctx.recg_free()


def test_pages_behind_four_gigabytes():
    """Every operation on pages whose blocks and headers lie behind 2^32 bytes, in the second layer."""
    n_pages = 140000                                                     # 4.6 GB a layer
    ctx = make(8, 128, 8, max_tokens=64, max_req=2, group=4)
    assert ctx.kv_pool_bytes(n_pages) // 2 > 2 ** 32
    pool = binding.alloc_kv_pool(ctx, n_pages, fill=None)
    pt = n_pages - 1 - np.arange(16).reshape(2, 8) * 3
    L = [70, 33]
    caches = []
    for r, n in enumerate(L):
        k, v = synth.kv_values(n, 8, 128, seed=r)
        ctx.recg_kv_write(pool, n_pages, 1, pt[r], 0, k.cuda(), v.cuda())
        caches.append([_kv8.Cache(8, 128).write(0, k), _kv8.Cache(8, 128).write(0, v)])
    batch = binding.Batch(L, [5, 1], [12, 0], None, pt, pool, n_pages)
    x = torch.randn((18, 48, 128), device="cuda").bfloat16()
    q, k, v = x[:, :32], x[:, 32:40], x[:, 40:]
    turned, o, lse = torch.empty((18, 32, 128), dtype=torch.bfloat16, device="cuda"), torch.empty((18, 32, 128), dtype=torch.bfloat16, device="cuda"), \
        torch.empty((18, 32), device="cuda")
    ctx.recg_kv_append_rotary(batch, 1, q, k, v, turned)
    p = np.concatenate([np.arange(70, 87), [33]])
    rk = _kv8.rotated(k, p, BASE)[0]
    got = ctx.recg_kv_rows(None, 1)
    for r, (t, n) in enumerate(((0, 17), (17, 1))):
        caches[r][0].write(L[r], rk[t:t + n])
        caches[r][1].write(L[r], v[t:t + n])
        assert same(got[0][t:t + n], caches[r][0].bf16(L[r], n)) and same(got[1][t:t + n], caches[r][1].bf16(L[r], n))
        for held, c in zip(ctx.recg_kv_read(pool, n_pages, 1, pt[r], 0, L[r] + n), caches[r]):
            assert same(held, c.bf16(0, L[r] + n))
    for rows in (2, 1):                                                  # the kernel of many rows, and that of few
        if rows == 1:
            batch = binding.Batch([87, 34], [1, 1], [0, 0], None, pt, pool, n_pages)
            ctx.recg_kv_append(batch, 1, k[:2].contiguous(), v[:2].contiguous())
            caches = [[c[i].write(n, t[r:r + 1]) for i, t in enumerate((k, v))] for r, (c, n) in enumerate(zip(caches, (87, 34)))]
        n = 18 if rows == 2 else 2
        ctx.recg_attention(batch, 1, turned[:n], o[:n], lse[:n])
        ctx.recg_sync()
        for r, (t, m, see) in enumerate(((0, 17, _kv4.visible(70, 5, 12)), (17, 1, _kv4.visible(33, 1, 0))) if rows == 2 else
                                        ((0, 1, _kv4.visible(87, 1, 0)), (1, 1, _kv4.visible(34, 1, 0)))):
            _kv8.check(f64(o[t:t + m]), f64(lse[t:t + m]), f64(turned[t:t + m]), caches[r][0].held, caches[r][1].held, see)
    ctx.recg_free()
