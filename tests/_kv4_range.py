"""How far the kernels over a 4-bit pool may be off where values differ by many powers of two: their operands are fp16 numbers, on scales that
neighbours share.

fp16 rounds by 2^-11 of a value down to 2^-14 and by 2^-25 below.  With x = m + s c for a row of K or V:
many rows  (the tcgen05 kernel)
    scales: K and V of 32 tokens 2^e, e a multiple of 8 that brings the largest |end of a row| (K: |m + 8 s| and 8 s) to [1, 2^8), or, where
    some token's own is lower by 16 or more, of every token its own; a row of Q likewise by itself; e is not below -56
    V     s, m and m + s c are rounded: 2^-11 |x|, and (15 + 1 + 1) 2^-25 2^e
    P     stands as 2^7 p 2^(e_j - e), e the largest e_j that the row has seen: 2^-11 p, and 2^-25 of it, which is 2^-32 2^(e - e_j) of p
          (twice where tokens have scales of their own: it is rounded before that is applied, and behind)
    K     s (c - 8), of a rounded s, and the second term of m + 8 s: (8 + 1 + 1) 2^-25 2^e a value (of sum |q|)
    Q     2^-25 2^e a value (of sum |s (c - 8)|), and 2^-25 2^e for the second term of its sum (of |m + 8 s|)
few rows, and gathered weights
    Q     a row's largest, or (few rows) one at most 2^8 as large, in [2^8, 2^9) 2^e, half of the values divided by 16 besides: 2^-21 2^e
          a value
    P s   stands as 2^7 p s / s_top, s_top a power of two above the largest step that the row has seen so far, at most twice the largest:
          2^-11 p s, and 2^-32 s_top

Everything else is fp32: a score's sum takes eight or nine steps in an accumulator that drops what is below 2^-22 of its largest term (2^-19
of the terms' sum, which is taken with c - 8 by many rows and with c by few), 2^x and its argument are good to 2^-21, sums over tokens to 2^-17."""
import numpy as np


def scale_exp(top):
    """Multiples of eight E with 2^-E top in [1, 2^8)."""
    e = np.floor(np.log2(np.maximum(top, 1e-300)))
    return np.clip(np.floor(e / 8) * 8, -56, 120)


def token_scales(top):
    """The scale on which the kernel of many rows has every token, and whether it is the token's own.  top [L]: a token's largest value."""
    L = len(top)
    own = np.concatenate([scale_exp(top), np.full(-L % 32, -56.0)]).reshape(-1, 32)
    held = np.concatenate([top > 0, np.zeros(-L % 32, dtype=bool)]).reshape(-1, 32)
    most = own.max(-1, keepdims=True)
    apart = (held & (own + 8 < most)).any(-1, keepdims=True)
    return np.where(apart, own, most).reshape(-1)[:L], np.broadcast_to(apart, own.shape).reshape(-1)[:L]


def score_bounds(q, ck, sk, mk, many, top_q):
    """|error| of every score in nats, [n, L].  q [n, d] of a head; ck [L, d], sk and mk [L] of its kv head; top_q: largest |q| on whose scale a
    row stands (few rows), [n] or one for all."""
    d = q.shape[1]
    aq = np.abs(q)
    if many:
        c8, mid = sk[:, None] * np.abs(ck - 8), np.abs(mk + 8 * sk)
        size = aq @ c8.T + np.abs(q.sum(-1))[:, None] * mid[None]
        ek, eq = token_scales(np.maximum(mid, 8 * sk))[0], scale_exp(aq.max(-1))
        lost = 10 * 2.0 ** -25 * aq.sum(-1)[:, None] * 2.0 ** ek + 2.0 ** -25 * 2.0 ** eq[:, None] * (c8.sum(-1) + mid)[None]
    else:
        sc = sk[:, None] * ck
        size = aq @ sc.T + np.abs(q.sum(-1))[:, None] * np.abs(mk)[None]
        lost = 2.0 ** -29 * 2.0 ** np.floor(np.log2(np.reshape(top_q, (-1, 1)))) * sc.sum(-1)[None]
    return (size * 2.0 ** -19 + lost) / np.sqrt(d) + 2.0 ** -21


def attention(q, k_codes, v_codes, see, many):
    """o, lse in float64 and the bounds of both (o before its own rounding)."""
    (ck, sk, mk), (cv, sv, mv) = k_codes, v_codes
    n, nq, d = q.shape
    g = nq // ck.shape[1]
    o, o_err, lse, lse_err = np.zeros((n, nq, d)), np.zeros((n, nq, d)), np.zeros((n, nq)), np.zeros((n, nq))
    for h in range(nq):
        kh = h // g
        s_k, m_k, s_v, m_v = (x[:, kh, 0] for x in (sk, mk, sv, mv))
        z = np.where(see, q[:, h] @ (mk[:, kh] + sk[:, kh] * ck[:, kh]).T / np.sqrt(d), -np.inf)
        top = z.max(-1, keepdims=True)
        p = np.exp(z - top)
        total = p.sum(-1, keepdims=True)
        p /= total
        x = m_v[:, None] + s_v[:, None] * cv[:, kh]
        o[:, h], lse[:, h] = p @ x, (top + np.log(total))[:, 0]
        off = np.where(see, score_bounds(q[:, h], ck[:, kh], s_k, m_k, many, np.minimum(np.abs(q).max(), 2.0 ** 8 * np.abs(q[:, h]).max(-1))), 0.0)
        pd = p * off
        # (where the largest score is ahead of all others by more than any two can be off, its position is all of the result)
        second = np.sort(z, -1)[:, -2] if z.shape[1] > 1 else np.full(n, -np.inf)
        pd_o = np.where((top[:, 0] - second > 2 * off.max(-1) + 30)[:, None], 0.0, pd)
        coded, held, low = p @ (s_v[:, None] * cv[:, kh]), p @ np.abs(x), p @ np.abs(m_v)[:, None]
        if many:
            ev, apart = token_scales(np.maximum(np.abs(m_v), np.abs(m_v + 15 * s_v)))
            seen = np.where(see, ev, -1000.0).max(-1, keepdims=True)
            # (a row's reference is a whole number next to its largest score so far: the sum is at least 2^-.5)
            lost = np.sqrt(2) / total * (np.where(see, (1 + apart) * 2.0 ** -32 * 2.0 ** np.maximum(seen - ev, 0), 0.0) @ np.abs(x)) + 17 * 2.0 ** -25 * p @ (2.0 ** ev)[:, None]
            rounded = 2 * 2.0 ** -11 * held
        else:
            lost = see.sum(-1, keepdims=True) / total * 15 * 2.0 ** -32 * 2 * np.where(see, s_v, 0.0).max(-1, keepdims=True)
            rounded = 2.0 ** -11 * coded
        o_err[:, h] = rounded + lost + 2.0 ** -17 * (coded + low) + 1.1 * (pd_o @ np.abs(x) + np.abs(o[:, h]) * pd_o.sum(-1, keepdims=True))
        lse_err[:, h] = 1.1 * pd.sum(-1) + 2.0 ** -20 * (1 + np.abs(top[:, 0]) + np.log(see.shape[1]))
    return o, lse, o_err, lse_err


def gathered(q, k_codes, see, lse, row_weight):
    """Weight that every position receives, [nkv, L], and its bound.  A probability is 2^(score - lse) in fp32."""
    ck, sk, mk = k_codes
    n, nq, d = q.shape
    nkv = ck.shape[1]
    g = nq // nkv
    out, err = np.zeros((nkv, ck.shape[0])), np.zeros((nkv, ck.shape[0]))
    for h in range(nq):
        kh = h // g
        z = q[:, h] @ (mk[:, kh] + sk[:, kh] * ck[:, kh]).T / np.sqrt(d)
        off = score_bounds(q[:, h], ck[:, kh], sk[:, kh, 0], mk[:, kh, 0], False, np.abs(q[:, h]).max(-1)) + 2.0 ** -20 * (1 + np.abs(z) + np.abs(lse[:, h:h + 1]))
        p = np.exp(np.where(see, z - lse[:, h:h + 1], -np.inf)) * row_weight[:, None]
        out[kh] += p.sum(0)
        err[kh] += (p * (1.1 * np.where(see, off, 0.0) + n * g * 2.0 ** -23)).sum(0)
    return out, err
