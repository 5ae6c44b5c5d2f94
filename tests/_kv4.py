"""Plain float64 forms of the 4-bit cache, used by the tests: what a row of it stands for, and attention over that."""
import math

import numpy as np
import torch


def codes(x):
    """x: bf16 tensor [..., d] -> (codes, step, minimum) as float64 arrays, from the definition."""
    a = x.detach().cpu().double().numpy()
    m = a.min(-1, keepdims=True)
    with np.errstate(all="ignore"):
        span = (a.max(-1, keepdims=True).astype(np.float32) - m.astype(np.float32)) / np.float32(15)
        s = torch.from_numpy(span).bfloat16().double().numpy()
        bad = ~np.isfinite(a).all(-1, keepdims=True) | ~np.isfinite(s)
        s = np.where(bad, np.nan, np.where(s < 2.0 ** -119, 0.0, s))
        c = np.where(s > 0, np.clip(np.rint((a - m) / np.where(s > 0, s, 1.0)), 0, 15), 0.0)
    return c, s, m


def values(x):
    """What the cache stands for, in float64."""
    c, s, m = codes(x)
    with np.errstate(all="ignore"):
        return m + s * c


def values_bf16(x):
    """... and as the pool is read: rounded once."""
    return torch.from_numpy(values(x)).float().bfloat16()


def attention(q, k, v, see):
    """q [n, nq, d], k and v [L, nkv, d] float64, see [n, L] bool -> (o [n, nq, d], lse [n, nq])."""
    n, nq, d = q.shape
    g = nq // k.shape[1]
    o, lse = np.zeros((n, nq, d)), np.full((n, nq), -np.inf)
    for h in range(nq):
        z = np.where(see, q[:, h] @ k[:, h // g].T / math.sqrt(d), -np.inf)
        top = z.max(-1, keepdims=True)
        p = np.exp(z - top)
        o[:, h] = (p / p.sum(-1, keepdims=True)) @ np.where(see.any(0)[:, None], v[:, h // g], 0.0)
        lse[:, h] = (top + np.log(p.sum(-1, keepdims=True)))[:, 0]
    return o, lse


def visible(L, v, b, corr=(), bc=0):
    """[n, L + n] bool: what each new row of a request sees (corr: draft indices its branches replace, bc masks each)."""
    n = v + b + len(corr) * (1 + bc)
    see = np.zeros((n, L + n), dtype=bool)
    for i in range(v):
        see[i, :L + i + 1] = True
    see[v:v + b, :L + v + b] = True
    for k, i in enumerate(corr):
        first = v + b + k * (1 + bc)
        see[first:first + 1 + bc, :L + i] = True
        see[first, L + first] = True
        see[first + 1:first + 1 + bc, L + first:L + first + 1 + bc] = True
    return see


def attention_bounds(q, k_codes, v_codes, see):
    """How far kernels may be from `attention` (o before its own rounding, and lse).

    o: both kernels round to fp16, half a step being 2^-11.  One multiplies p s, rounded, with the code c: 2^-11 of every term p s c.
    The other rounds p and m + s c: 2 x 2^-11 of every term p |m + s c|.  Everything else is fp32: a score's sum of exact products takes
    eight or nine steps in an accumulator that drops what is below 2^-22 of its largest term, 2^x and its argument are good to 2^-21 of the
    exponents, and sums over tokens to 2^-17."""
    (ck, sk, mk), (cv, sv, mv) = k_codes, v_codes
    n, nq, d = q.shape
    g = nq // ck.shape[1]
    o_err, lse_err = np.zeros((n, nq, d)), np.zeros((n, nq))
    for h in range(nq):
        kh = h // g
        size = (np.abs(q[:, h]) @ (sk[:, kh] * np.abs(ck[:, kh] - 8)).T
                + np.abs(q[:, h]).sum(-1, keepdims=True) * np.abs(mk[:, kh] + 8 * sk[:, kh]).T) / math.sqrt(d)
        score = np.where(see, size * 2.0 ** -19 + 2.0 ** -21, 0.0).max(-1)               # absolute error of any visible score
        z = np.where(see, q[:, h] @ (mk[:, kh] + sk[:, kh] * ck[:, kh]).T / math.sqrt(d), -np.inf)
        top = z.max(-1, keepdims=True)
        p = np.exp(z - top)
        p /= p.sum(-1, keepdims=True)
        some = see.any(0)[:, None]
        coded, held = p @ np.where(some, sv[:, kh] * cv[:, kh], 0.0), p @ np.where(some, np.abs(mv[:, kh] + sv[:, kh] * cv[:, kh]), 0.0)
        low = p @ np.where(some, np.abs(mv[:, kh]), 0.0)
        o_err[:, h] = 2.0 ** -11 * np.maximum(coded, 2 * held) + (2.0 ** -17 + 4 * score)[:, None] * (coded + low)
        lse_err[:, h] = score + 2.0 ** -20 * (1 + np.abs(top[:, 0]) + math.log(see.shape[1]))
    return o_err, lse_err


def gathered(q, k, see, lse, row_weight):
    """Weight that every position receives, [nkv, L], and how far kernels may be from it: a probability is 2^(score - lse) with both
    in fp32 (a score's sum: see attention_bounds), and at most n * group of them are added up."""
    n, nq, d = q.shape
    nkv = k.shape[1]
    g = nq // nkv
    out, err = np.zeros((nkv, k.shape[0])), np.zeros((nkv, k.shape[0]))
    for h in range(nq):
        with np.errstate(all="ignore"):
            z = q[:, h] @ k[:, h // g].T / math.sqrt(d)
            size = np.abs(q[:, h]) @ np.abs(k[:, h // g]).T / math.sqrt(d)
            use = see & (row_weight != 0)[:, None]
            p = np.where(use, np.exp(z - lse[:, h:h + 1]) * row_weight[:, None], 0.0)
            rel = np.where(use, 3 * size * 2.0 ** -19 + 2.0 ** -20 * (1 + np.abs(z) + np.abs(lse[:, h:h + 1])), 0.0)
        out[h // g] += p.sum(0)
        err[h // g] += (np.abs(p) * (rel + n * g * 2.0 ** -23)).sum(0)
    return out, err
