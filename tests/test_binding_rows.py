"""Calls with batch=None are sized by the batch that the library has laid out last, whatever the calls in between were.

On the CPU the library is a stand-in that keeps count of layouts as the library does (an upload lays out; a refusal in front of it leaves
what was there); on the GPU it is the library itself."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2609_34388_b200 import binding, synth
from tests import _kv4

NKV, D = 2, 64
SHAPE = synth.ModelShape(n_layers=2, hidden=64, n_q_heads=4, n_kv_heads=NKV, head_dim=D, ffn=64, vocab=64)


class Library:
    """Remembers the rows and pages of the batch laid out last, and what a call with batch=None was given room for."""

    def __init__(self):
        self.rows = self.pages = 0
        self.seen = []

    def lay_out(self, b):
        if b is None:
            return 0 if self.rows else 1
        c = b._obj
        n = sum((C.c_int32 * c.n_req).from_address(c.verify_len)) + sum((C.c_int32 * c.n_req).from_address(c.block_size))
        self.rows, self.pages = n, c.kv_pool_pages
        return 0

    def recg_init(self, out, cfg, w, stream):
        return 0

    def recg_last_error(self, h):
        return b"refused"

    def recg_layout_info(self, h, rows, pages):
        C.c_int32.from_address(rows).value = self.rows
        C.c_int64.from_address(pages).value = self.pages
        return 0

    def recg_verify(self, h, b, logits, dtype, out):
        return self.lay_out(b) if logits else 0

    def recg_kv_rows(self, h, b, layer, k, v, stride):
        if layer < 0 or layer >= 2:
            return 1
        status = self.lay_out(b)
        self.seen.append((v - k) // (2 * NKV * D))          # rows that fit in front of v (both in one allocation)
        return status


@pytest.fixture
def library(monkeypatch):
    fake = Library()
    monkeypatch.setattr(binding, "lib", lambda: fake)
    monkeypatch.setattr(binding, "_CUDA", torch.device("cpu"))
    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    return fake


def batch_of(rows, n_pages=8, page0=0, pool=None):
    pool = torch.zeros(8) if pool is None else pool
    return binding.Batch([3], [rows], [0], [1] * rows, page0 + np.arange(4)[None], pool, n_pages)


@pytest.mark.parametrize("between", ["layer", "shape", "dtype", "verify", "step of other weights", "nothing"])
def test_room_of_a_call_without_a_batch(library, between):
    ctx = binding.Context(binding.make_config(SHAPE, 2, 64, 4, 0), stream=1)
    small, large = batch_of(2), batch_of(40)
    ctx.recg_kv_rows(large if between != "verify" else small, 0)
    if between == "layer":
        with pytest.raises(binding.RecgError):
            ctx.recg_kv_rows(small, 7)
    elif between in ("shape", "dtype"):
        k = torch.zeros((3, NKV, D), dtype=torch.bfloat16) if between == "shape" else torch.zeros((2, NKV, D))
        with pytest.raises(ValueError):
            ctx.recg_kv_append(small, 0, k, k)
    elif between == "verify":
        ctx.recg_verify(large, torch.zeros((40, 64)))
    elif between == "step of other weights":
        ctx._track = torch.zeros(5)
        with pytest.raises(ValueError):
            ctx.recg_step(small)
    k, v = ctx.recg_kv_rows(None, 0)
    assert library.rows == 40 and library.seen[-1] == 40 and k.shape == v.shape == (40, NKV, D)


def test_no_batch_so_far(library):
    ctx = binding.Context(binding.make_config(SHAPE, 2, 64, 4, 0), stream=1)
    with pytest.raises(binding.RecgError):
        ctx.recg_kv_rows(None, 0)
    assert library.seen == [0]


@pytest.mark.gpu
@pytest.mark.parametrize("flags", [0, binding.FLAG_KV_4BIT])
@pytest.mark.parametrize("between", ["layer", "shape", "lse", "decay", "pool", "verify", "step", "capacity"])
def test_operations_without_a_batch_behind_refused_calls(flags, between):
    """A batch of 40 rows, a call that is refused with (or a verification that lays out) another one, then every operation with None."""
    W = synth.model_weights(SHAPE, seed=0, dtype=torch.bfloat16)
    W = {k: ([t.cuda() for t in v] if isinstance(v, list) else v.cuda()) for k, v in W.items()}
    ctx = binding.Context(binding.make_config(SHAPE, 2, 64, 4, flags), W)
    n_pages = 9
    pool, w = binding.alloc_kv_pool(ctx, n_pages), torch.zeros((2, n_pages, NKV, 16), device="cuda")
    k = torch.randn((43, NKV, D), device="cuda").bfloat16()
    small, large = batch_of(2, n_pages, 4, pool), batch_of(40, n_pages, 0, pool)
    for b in (small, large):
        ctx.recg_kv_write(pool, n_pages, 0, b.page_table[0], 0, k, k)
    q = torch.randn((40, 4, D), device="cuda").bfloat16()
    lse, o, o_want = torch.zeros((40, 4), device="cuda"), torch.empty_like(q), torch.empty_like(q)
    rows, pages = C.c_int32(), C.c_int64()
    info = lambda: (binding.lib().recg_layout_info(ctx.h, C.addressof(rows), C.addressof(pages)), rows.value, pages.value)
    assert info() == (0, 0, 0) and binding.lib().recg_layout_info(ctx.h, None, C.addressof(pages)) == 1
    ctx.recg_attention(large, 0, q, o_want, lse)
    if between == "verify":
        ctx.recg_kv_rows(small, 0)
        assert info() == (0, 2, n_pages)
        ctx.recg_verify(large, torch.randn((40, 64), device="cuda"))
    else:
        call = {"layer": lambda: ctx.recg_kv_rows(small, 7), "shape": lambda: ctx.recg_kv_append(small, 0, k[:3], k[:3]),
                "lse": lambda: ctx.recg_attention(small, 0, q[:2], o, lse), "decay": lambda: ctx.recg_kv_weights(small, 0, q[:2], lse[:2], None, w, decay=-1.0),
                "pool": lambda: ctx.recg_kv_weights(small, 0, q[:2], lse[:2], None, w[:1]),
                "step": lambda: (ctx.recg_kv_track(w[:1].clone()), ctx.recg_step(small)),
                "capacity": lambda: ctx.recg_kv_rows(batch_of(65, n_pages, 4, pool), 0)}[between]
        with pytest.raises((ValueError, binding.RecgError)):
            call()
    if between == "capacity":                                  # (refused in the course of the upload: there is no batch now)
        assert info() == (0, 0, 0)
        with pytest.raises(binding.RecgError, match="no batch"):
            ctx.recg_kv_rows(None, 0)
        ctx.recg_kv_rows(large, 0)
    assert info() == (0, 40, n_pages)
    kb, vb = ctx.recg_kv_rows(None, 0)
    want = (_kv4.values_bf16(k) if flags else k.cpu())[3:]
    assert torch.equal(kb.cpu(), want) and torch.equal(vb.cpu(), want)
    ctx.recg_attention(None, 0, q, o, lse)
    assert torch.equal(o, o_want)
    ctx.recg_kv_weights(None, 0, q, lse, None, w)
    for bad in (lambda: ctx.recg_attention(None, 0, q, o, lse[:2]), lambda: ctx.recg_kv_weights(None, 0, q[:2], lse[:2], None, w),
                lambda: ctx.recg_kv_weights(None, 0, q, lse, None, w[:1]), lambda: ctx.recg_kv_weights(None, 0, q, lse, None, w, torch.ones(2, device="cuda")),
                lambda: ctx.recg_kv_append(None, 0, k[:2], k[:2]), lambda: ctx.recg_kv_rows(None, 0, k[:2], k[:2])):
        with pytest.raises(ValueError):
            bad()
    ctx.recg_kv_append(None, 0, kb, vb)
    ctx.recg_sync()
    ctx.recg_free()
