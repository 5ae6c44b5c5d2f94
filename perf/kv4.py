"""Times around the 4-bit KV pool that are not operator cases: whole rounds over either kind of pool, and attention batches on both sides of
the line between its two kernels.  Run from the repository's root: python perf/kv4.py [rounds] [device] [rows] [moves]

  rounds  eight layers of the 8B class: bf16 pool, 4 bits, 4 bits with the weights gathered
  device  the same with the lengths on the device (recg_step_device)
  rows    attention of one layer, the kernel that the batch's largest row tile chooses and the one of few rows (RECG_FLAG_SIMT_ATTENTION)
  moves   choice and move of an eviction in place and to other pages, eight layers

CUDA events around 20 passes behind 5, inputs as they are left by the pass before (larger than L2 but for the smallest)."""
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2609_34388_b200 import binding, synth  # noqa: E402

FOUR, SIMT = binding.FLAG_KV_4BIT, binding.FLAG_SIMT_ATTENTION


def timed(f, n=20):
    for _ in range(5):
        f()
    a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    torch.cuda.synchronize()
    a.record()
    for _ in range(n):
        f()
    b.record()
    torch.cuda.synchronize()
    return a.elapsed_time(b) / n * 1e3


def contexts(n_req, lo, hi):
    return np.random.default_rng(3).integers(lo, hi + 1, n_req)


def filled_pool(ctx, L, table, n_pages, layers):
    pool = binding.alloc_kv_pool(ctx, n_pages, fill=None)
    g = torch.Generator(device="cuda").manual_seed(1)
    for r, n in enumerate(L):
        k, v = (torch.randn((int(n), ctx.cfg.n_kv_heads, ctx.cfg.head_dim), device="cuda", generator=g).bfloat16() for _ in range(2))
        for layer in range(layers):
            ctx.recg_kv_write(pool, n_pages, layer, table[r], 0, k, v)
    return pool


def rounds(device):
    shape = synth.llama8b_shape(8)
    W = synth.model_weights(shape, seed=0, device="cuda")
    for name, n_req, v, b, lo, hi in (("16 requests, a token each", 16, 1, 0, 512, 8192), ("64 requests, a token each", 64, 1, 0, 512, 8192),
                                      ("16 requests, 16 + 16 rows", 16, 16, 16, 512, 8192), ("1 request, a token behind 131072", 1, 1, 0, 131072, 131072)):
        L = contexts(n_req, lo, hi)
        table, n_pages = synth.page_tables(L, [v + b] * n_req, 16, seed=5)
        ids = np.random.default_rng(4).integers(0, 1000, (n_req, v))
        out = []
        for flags, track in ((0, False), (FOUR, False), (FOUR, True)):
            ctx = binding.Context(binding.make_config(shape, n_req, n_req * (v + b), table.shape[1], flags), W)
            pool = filled_pool(ctx, L, table, n_pages, shape.n_layers)
            if track:
                ctx.recg_kv_track(torch.zeros((shape.n_layers, n_pages, shape.n_kv_heads, 16), device="cuda"))
            if device:
                batch = binding.DeviceBatch(L, [v] * n_req, [b] * n_req, ids.tolist(), max(v, 1), table, pool, n_pages, rows_hint=n_req * (v + b))
                out.append(timed(lambda: ctx.recg_step_device(batch)))
            else:
                batch = binding.Batch(L, [v] * n_req, [b] * n_req, ids.reshape(-1), table, pool, n_pages)
                out.append(timed(lambda: ctx.recg_step(batch)))
            ctx.recg_sync()
            ctx.recg_free()
            del pool
        print(f"{'device round' if device else 'round'}: {name}: bf16 {out[0]:.0f}, 4 bits {out[1]:.0f}, gathered {out[2]:.0f} us", flush=True)


def rows():
    shape = synth.llama8b_shape(1)
    mixed = [1] * 15 + [16]
    for name, L, v, b in ([(f"16 requests, {4 * n} rows a kv head", contexts(16, 512, 8192), [n] * 16, [0] * 16) for n in (1, 2, 3, 8)]
                          + [(f"1 request of 4096, {4 * n} rows a kv head", [4096], [n], [0]) for n in (1, 2, 3, 8)]
                          + [("15 requests of one row, one of 16 + 16", contexts(16, 512, 8192), mixed, [0] * 15 + [16]),
                             ("63 requests of one row, one of 16 + 16", contexts(64, 512, 8192), [1] * 63 + [16], [0] * 63 + [16])]):
        table, n_pages = synth.page_tables(L, [x + y for x, y in zip(v, b)], 16, seed=5)
        T = sum(v) + sum(b)
        out = []
        for flags in (0, FOUR, FOUR | SIMT):
            ctx = binding.Context(binding.make_config(shape, len(L), T, table.shape[1], flags))
            pool = filled_pool(ctx, np.asarray(L) + v + b, table, n_pages, 1)
            q = synth.queries(T, shape.n_q_heads, shape.head_dim, device="cuda")
            o = torch.empty_like(q)
            ctx.recg_attention(binding.Batch(L, v, b, None, table, pool, n_pages), 0, q, o)
            out.append(timed(lambda: ctx.recg_attention(None, 0, q, o), 50))
            ctx.recg_sync()
            ctx.recg_free()
            del pool
        print(f"attention: {name}: bf16 {out[0]:.1f}, 4 bits {out[1]:.1f}, 4 bits by the kernel of few rows {out[2]:.1f} us", flush=True)


def moves():
    shape = synth.llama8b_shape(8)
    for n_req, lo, hi in ((1, 4096, 4096), (4, 8192, 16384), (16, 2048, 8192)):
        L = contexts(n_req, lo, hi)
        both, n_pages = synth.page_tables(list(L) * 2, [1] * (2 * n_req), 16, seed=5)
        budget = (L * 0.33).astype(np.int32)
        for flags, kind in ((0, "bf16"), (FOUR, "4 bits")):
            ctx = binding.Context(binding.make_config(shape, n_req, 32, both.shape[1], flags))
            pool = filled_pool(ctx, L, both, n_pages, shape.n_layers)
            w = torch.rand((shape.n_layers, n_pages, shape.n_kv_heads, 16), device="cuda")
            keep = torch.empty((shape.n_layers, n_req, shape.n_kv_heads, int(budget.max())), dtype=torch.int32, device="cuda")
            out = []
            for dst in (both[n_req:], None):
                ev = binding.Eviction(L, budget, both[:n_req], pool, n_pages, w, 4, 256, dst, (0, shape.n_layers))
                ctx.recg_kv_select(ev, keep)
                if dst is not None:
                    out.append(timed(lambda: ctx.recg_kv_select(ev, keep)))
                # (in place the same list is good again: what it moves then is not what was chosen, but as many bytes)
                out.append(timed(lambda: ctx.recg_kv_compact(ev, keep)))
            moved = float(budget.sum()) * shape.n_layers * shape.n_kv_heads * 2 * (136 if flags else 512) / 6449e3
            print(f"eviction: {n_req} requests of {lo} to {hi} to a third, {kind}: choice {out[0]:.1f}, move to other pages {out[1]:.1f}, "
                  f"in place {out[2]:.1f} us (bytes moved: {moved:.1f})", flush=True)
            ctx.recg_sync()
            ctx.recg_free()
            del pool


if __name__ == "__main__":
    what = sys.argv[1:] or ["rounds", "device", "rows", "moves"]
    for name, f in (("rounds", lambda: rounds(False)), ("device", lambda: rounds(True)), ("rows", rows), ("moves", moves)):
        if name in what:
            f()
