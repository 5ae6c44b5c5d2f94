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
