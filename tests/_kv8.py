"""Plain float64 forms of the 8-bit cache, used by the tests: what blocks of it stand for, how they change as rows come in, attention
over that, and rotation."""
import math

import numpy as np
import torch


def block(x):
    """x float64 [rows <= 16, heads, d], NaN or infinite where a row is none -> (what the cache stands for, exponents [heads])."""
    bad = ~np.isfinite(x).all(-1)                                        # [rows, heads]
    a = np.where(bad[..., None], 0.0, x)
    most = np.abs(a).max((0, 2))
    e = np.zeros(len(most), dtype=int)
    for h, m in enumerate(most):
        if m > 0:
            e[h] = max(-60, min(120, math.ceil(math.log2(m / 448.0)) - 2))
            while e[h] < 120 and m > 448.0 * 2.0 ** e[h]:
                e[h] += 1
    unit = 2.0 ** e.astype(np.float64)[None, :, None]
    y = a / unit
    with np.errstate(divide="ignore"):
        step = 2.0 ** (np.maximum(np.floor(np.log2(np.where(y == 0, 1.0, np.abs(y)))), -6) - 3)
    end = np.where(e == 120, 240.0, 448.0)[None, :, None]
    held = np.clip(np.rint(y / step) * step, -end, end) * unit
    return np.where(bad[..., None], np.nan, held), e


class Cache:
    """One request's positions as the cache stands for them."""

    def __init__(self, heads, d):
        self.held = np.zeros((0, heads, d))
        self.e = np.zeros((0, heads), dtype=int)          # per position: its block's exponent

    def write(self, pos0, x):
        """x [n, heads, d] (a torch tensor in bf16) for positions pos0 ..; what stood from pos0 on is gone."""
        if x.shape[0] == 0:
            return self
        start = pos0 // 16 * 16
        rows = np.concatenate([self.held[start:pos0], x.detach().cpu().double().numpy()])
        assert len(rows) == pos0 + x.shape[0] - start, "a request is written front to back"
        parts, es = [self.held[:start]], [self.e[:start]]
        for i in range(0, len(rows), 16):
            held, e = block(rows[i:i + 16])
            parts.append(held)
            es.append(np.broadcast_to(e, held.shape[:2]))
        self.held, self.e = np.concatenate(parts), np.concatenate(es)
        return self

    def bf16(self, pos0, n):
        return torch.from_numpy(self.held[pos0:pos0 + n]).float().bfloat16()


def attention(q, k, v, see):
    """q [n, nq, d], k and v [L, nkv, d] float64, see [n, L] bool -> (o [n, nq, d], lse [n, nq]).  Rows that are none reach those that see
    them only."""
    n, nq, d = q.shape
    g = nq // k.shape[1]
    o, lse = np.zeros((n, nq, d)), np.full((n, nq), -np.inf)
    for h in range(nq):
        with np.errstate(all="ignore"):
            z = np.where(see, q[:, h] @ k[:, h // g].T / math.sqrt(d), -np.inf)
            top = z.max(-1, keepdims=True)
            p = np.exp(z - top)
            vh = v[:, h // g]
            none = np.isnan(vh).any(-1)
            o[:, h] = (p / p.sum(-1, keepdims=True)) @ np.where(none[:, None], 0.0, vh)
            o[:, h] = np.where((see & none)[:, :].any(-1)[:, None], np.nan, o[:, h])
            lse[:, h] = (top + np.log(p.sum(-1, keepdims=True)))[:, 0]
    return o, lse


def attention_bounds(q, k, v, see, size_of_exponents=16.0):
    """How far kernels may be from `attention` (o before its own rounding, and lse).

    o: codes are exact operands, probabilities are rounded to fp16, half a step being 2^-11: 2^-11 of every term p |v|.  Everything else is
    fp32: a score's sum of exact products takes eight or nine steps in an accumulator that drops what is below 2^-22 of its largest term;
    the exponent of V's block is added to it (`size_of_exponents`), 2^x and its argument are good to 2^-21 of the exponents, sums over
    tokens to 2^-17."""
    n, nq, d = q.shape
    g = nq // k.shape[1]
    o_err, lse_err = np.zeros((n, nq, d)), np.zeros((n, nq))
    for h in range(nq):
        kh, vh = k[:, h // g], v[:, h // g]
        size = np.abs(q[:, h]) @ np.abs(kh).T / math.sqrt(d)
        score = np.where(see, size * 2.0 ** -19 + size_of_exponents * 2.0 ** -23, 0.0).max(-1)
        z = np.where(see, q[:, h] @ kh.T / math.sqrt(d), -np.inf)
        top = z.max(-1, keepdims=True)
        p = np.exp(z - top)
        p /= p.sum(-1, keepdims=True)
        terms = p @ np.abs(vh)
        o_err[:, h] = (2.0 ** -11 + 2.0 ** -17 + 4 * score)[:, None] * terms
        lse_err[:, h] = score + 2.0 ** -20 * (1 + np.abs(top[:, 0]) + math.log(see.shape[1]))
    return o_err, lse_err


def check(got, got_lse, q, k, v, see, size_of_exponents=16.0):
    """Asserts o [n, nq, d] and lse [n, nq] of a request against float64, the result's rounding to bf16 (2^-8) counted."""
    o, lse = attention(q, k, v, see)
    o_err, lse_err = attention_bounds(q, k, v, see, size_of_exponents)
    over = np.abs(got - o) / (o_err + 2.0 ** -8 * (np.abs(o) + o_err) + 1e-30)
    assert np.isfinite(got).all() and over.max() <= 1.0, ("o", over.max())
    over = np.abs(got_lse - lse) / lse_err
    assert np.isfinite(got_lse).all() and over.max() <= 1.0, ("lse", over.max())


def positions(L, v, b, corr=(), bc=0):
    """Position of each new row of a request; a branch's rows stand where they hypothesise to."""
    p = list(range(L, L + v + b))
    for i in corr:
        p += range(L + i, L + i + 1 + bc)
    return np.array(p)


def window(see, p, n_sink, window):
    """see [n, L] further restricted: position j below n_sink, or above p - window."""
    j = np.arange(see.shape[1])
    return see & ((j < n_sink) | (j > p[:, None] - window))


def rotated(x, p, base):
    """x [n, heads, d] (bf16) at positions p [n], rounded once."""
    a = x.detach().cpu().double().numpy()
    h = a.shape[-1] // 2
    angle = p[:, None].astype(np.float64) * np.float64(np.float32(base)) ** (-np.arange(h) / h)
    c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
    y = np.concatenate([a[..., :h] * c - a[..., h:] * s, a[..., h:] * c + a[..., :h] * s], -1)
    return torch.from_numpy(y).float().bfloat16(), y
