"""The pool's operations at the edges of what they are given: contexts without layers."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2609_34388_b200 import binding, synth
from tests import _kv4

pytestmark = pytest.mark.gpu

POOLS = [0, binding.FLAG_KV_4BIT]


def make(layers, flags, heads=(4, 2, 64), max_req=2, max_tokens=32, stride=4):
    nq, nkv, d = heads
    shape = synth.ModelShape(n_layers=layers, hidden=64, n_q_heads=nq, n_kv_heads=nkv, head_dim=d, ffn=64, vocab=64)
    return binding.Context(binding.make_config(shape, max_req, max_tokens, stride, flags))


@pytest.mark.parametrize("flags", POOLS)
def test_a_context_without_layers_has_a_pool_of_one(flags):
    ctx, one = make(0, flags), make(1, flags)
    pool, table = binding.alloc_kv_pool(one, 4), np.arange(4)[None]
    k = torch.randn((60, 2, 64), device="cuda").bfloat16()
    held = _kv4.values_bf16(k) if flags else k.cpu()
    ctx.recg_kv_write(pool, 4, 0, table[0], 0, k, k)
    batch = binding.Batch([55], [5], [0], None, table, pool, 4)
    q = torch.randn((5, 4, 64), device="cuda").bfloat16()
    w = torch.zeros((1, 4, 2, 16), device="cuda")
    lib, rows = binding.lib(), k[:5].clone()
    o, lse, want, lse_want = torch.empty_like(q), torch.empty((5, 4), device="cuda"), torch.empty_like(q), torch.empty((5, 4), device="cuda")
    one.recg_attention(batch, 0, q, want, lse_want)
    # the second layer: refused by every operation, before anything is launched
    calls = [lambda l: ctx.recg_kv_write(pool, 4, l, table[0], 0, k, k), lambda l: ctx.recg_kv_read(pool, 4, l, table[0], 0, 60),
             lambda l: ctx.recg_kv_append(batch, l, rows, rows), lambda l: ctx.recg_kv_rows(batch, l), lambda l: ctx.recg_attention(batch, l, q, o, lse),
             lambda l: ctx.recg_attention(batch, l, q, o), lambda l: ctx.recg_kv_weights(batch, l, q, lse_want, None, w)]
    for call in calls:
        for layer in (1, 2 ** 31 - 1, -1):
            with pytest.raises(binding.RecgError, match="layer"):
                call(layer)
    # the first: as a context of one layer
    ctx.recg_attention(batch, 0, q, o, lse)
    assert torch.equal(o, want) and torch.equal(lse, lse_want)
    for x in ctx.recg_kv_rows(batch, 0):
        assert torch.equal(x.cpu(), held[55:])
    ctx.recg_kv_weights(batch, 0, q, lse, None, w)
    w_one = torch.zeros_like(w)
    one.recg_kv_weights(batch, 0, q, lse, None, w_one)
    assert torch.equal(w, w_one) and float(w.sum()) > 1
    with pytest.raises(ValueError):
        ctx.recg_kv_weights(batch, 0, q, lse, None, w.repeat(2, 1, 1, 1))
    keep = torch.empty((1, 1, 2, 20), dtype=torch.int32, device="cuda")
    ev = binding.Eviction([60], [20], table, pool, 4, w, 2, 3)
    ctx.recg_kv_select(ev, keep)
    ctx.recg_kv_compact(ev, keep)
    got = ctx.recg_kv_read(pool, 4, 0, table[0], 0, 20)[0].cpu()
    for h in range(2):
        assert torch.equal(got[:, h], held[keep[0, 0, h].cpu().long(), h])
    assert lib.recg_kv_select(ctx.h, C.byref(binding.Eviction([60], [20], table, pool, 4, w, layers=(0, 2)).c), keep.data_ptr(), 20) == 1
    for c in (ctx, one):
        c.recg_sync()
        c.recg_free()


@pytest.mark.parametrize("flags", POOLS)
@pytest.mark.parametrize("head_dim", [64, 128])
def test_in_place_lists_of_requests_that_are_not_cut(flags, head_dim):
    """keep may be any list with keep[i] >= i, also where as many positions stay as there are; an entry that is not one is reported."""
    ctx = make(1, flags, heads=(4, 2, head_dim), stride=16)
    n, table = [5, 200], np.arange(32).reshape(2, 16)
    pool, w = binding.alloc_kv_pool(ctx, 32), torch.rand((1, 32, 2, 16), device="cuda")
    before = w.clone()
    rows = []
    for r in range(2):
        k, v = synth.kv_values(n[r], 2, head_dim, seed=r, device="cuda")
        ctx.recg_kv_write(pool, 32, 0, table[r], 0, k, v)
        rows.append([t.cpu() for t in ctx.recg_kv_read(pool, 32, 0, table[r], 0, n[r])])
    g = np.random.default_rng(4)
    lists = np.full((1, 2, 2, 200), -1, dtype=np.int32)
    for h in range(2):
        lists[0, 0, h, :5] = [1, 1, 3, 3, 4]
        lists[0, 1, h] = [g.integers(i, 200) for i in range(200)]
    lists[0, 1, 0, 30:180] = np.arange(30, 180)                      # whole pages that stay where they are, behind and before some that do not
    keep = torch.from_numpy(lists).cuda()
    ev = binding.Eviction(n, [5, 1000], table, pool, 32, w)
    ctx.recg_kv_compact(ev, keep)
    ctx.recg_sync()

    def check(lists):
        for r in range(2):
            for got, had in zip(ctx.recg_kv_read(pool, 32, 0, table[r], 0, n[r]), rows[r]):
                for h in range(2):
                    assert torch.equal(got.cpu()[:, h], had[lists[0, r, h, :n[r]].astype(np.int64), h]), (r, h)
            pos = np.arange(n[r])
            for h in range(2):
                src = lists[0, r, h, :n[r]]
                assert torch.equal(w[0, table[r][pos // 16], h, pos % 16], before[0, table[r][src // 16], h, src % 16]), (r, h)

    check(lists)
    # the identity changes nothing
    same = np.broadcast_to(np.arange(200, dtype=np.int32), (1, 2, 2, 200)).copy()
    bytes_before = pool.view(torch.uint8).clone()
    ctx.recg_kv_compact(ev, torch.from_numpy(same).cuda())
    ctx.recg_sync()
    assert torch.equal(pool.view(torch.uint8), bytes_before)
    # entries that name no position, or one in front: reported, and their positions are left as they were
    same[0, 0, 1, 4], same[0, 1, 0, 7], same[0, 1, 1, 199] = 5, 6, -1
    ctx.recg_kv_compact(ev, torch.from_numpy(same).cuda())
    with pytest.raises(binding.RecgError, match="out of range"):
        ctx.recg_sync()
    assert torch.equal(pool.view(torch.uint8), bytes_before)
    ctx.recg_free()


@pytest.mark.parametrize("flags,far", [(0, 45000), (binding.FLAG_KV_4BIT, 160000)])
def test_pages_behind_four_gigabytes(flags, far):
    """The last pages of a pool of two layers that takes more than 2^32 bytes: what every operation gives for the first pages of a small one."""
    nq, nkv, d, L, n = 32, 8, 128, 300, 3
    got = []
    for n_pages in (64, far):
        ctx = make(2, flags, heads=(nq, nkv, d), stride=20, max_req=1, max_tokens=64)
        assert n_pages == 64 or ctx.kv_pool_bytes(n_pages) > 2 ** 32 + 2 ** 30
        pool, w = binding.alloc_kv_pool(ctx, n_pages, fill=None), torch.zeros((2, n_pages, nkv, 16), device="cuda")
        table, other = (n_pages - 1 - np.arange(20))[None], (n_pages - 21 - np.arange(20))[None]
        k, v = (t.cuda() for t in synth.kv_values(L + n, nkv, d, seed=3))
        ctx.recg_kv_write(pool, n_pages, 1, table[0], 0, k, v)
        batch = binding.Batch([L], [n], [0], None, table, pool, n_pages)
        ctx.recg_kv_append(batch, 1, k[:n], v[:n])
        out = list(ctx.recg_kv_rows(None, 1)) + list(ctx.recg_kv_read(pool, n_pages, 1, table[0], 0, L + n))
        for rows in (n, 40):                                           # both attention kernels of a 4-bit pool
            few = binding.Batch([L + n - rows], [rows], [0], None, table, pool, n_pages)
            q = synth.queries(rows, nq, d, seed=5).cuda()
            o, lse = torch.empty_like(q), torch.empty((rows, nq), device="cuda")
            ctx.recg_attention(few, 1, q, o, lse)
            ctx.recg_kv_weights(few, 1, q, lse, w, w)
            out += [o, lse]
        keep = torch.empty((1, 1, nkv, 100), dtype=torch.int32, device="cuda")
        for dst in (other, None):
            ev = binding.Eviction([L], [100], table, pool, n_pages, w, 4, 16, dst, (1, 2))
            ctx.recg_kv_select(ev, keep)
            ctx.recg_kv_compact(ev, keep)
            to = torch.from_numpy((table if dst is None else dst)[0, :7].copy()).cuda()
            out += [keep.clone(), w[1, to]] + list(ctx.recg_kv_read(pool, n_pages, 1, to.cpu().numpy(), 0, 100))
        ctx.recg_sync()
        ctx.recg_free()
        got.append([t.cpu() for t in out])
        del pool, w
        torch.cuda.empty_cache()
    for i, (a, b) in enumerate(zip(*got)):
        assert torch.equal(a, b), i
