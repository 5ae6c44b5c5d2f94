"""Operators around a KV cache in 8 bits and attention that looks back over a bounded distance, as measurable cases.

  append   the q, k and v rows of a batch as a projection leaves them: q and k are rotated to their positions, K and V go into the
           paged pool, bf16, 8 or 4 bits (`recg_kv_append_rotary`), and come back as the values that it holds (`recg_kv_rows`)
  attend   hybrid-mask paged attention over a pool in 8 bits, with the log-sum-exp of every row (`recg_attention`)
  window   the same over a bf16 pool or one in 8 bits, where a row sees the first few tokens and those at most a window away
           (`recg_window`, `recg_attention`)

Rotation, of a row at position p and for i < d / 2, a = p base^(-2 i / d):  y_i = x_i cos a - x_(i + d/2) sin a,
y_(i + d/2) = x_(i + d/2) cos a + x_i sin a, rounded once to bf16.

The 8-bit format, per block of 16 tokens (a page), kv head and K or V: e = the least whole number for which no value of the block
exceeds 448 2^e (within -60 .. 120; 0 where all are 0), a value x is held as the e4m3 number nearest to x 2^-e.  Rows that come into a
block which has some already take them along: e follows all of them, and what was held is rounded again.

Mask of Eq. 1: a row sees the positions <= limit and those in [lo, hi); with a window w and n first tokens a row at position p sees,
of these, the positions below n and those above p - w.

Shapes, block sizes and context ranges are those of the package's configurations, tests and benchmark.  The lengths of a
batch follow from the case alone (`batch` seeds them), every tensor from `prepare`'s seed.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
BASE = 500000.0

# (query heads, kv heads, head_dim): the 2-layer test model, the 8B class, the 14B class with five query heads per kv head
_HEADS = {"tiny": (4, 2, 64), "8b": (32, 8, 128), "14b": (40, 8, 128)}


def listed():
    return [
        # one token of one user: launches and latency are all there is
        {"name": "append_one_token", "op": "append", "model": "8b", "bits": 8, "n_req": 1, "rows": 1, "ctx_lo": 500, "ctx_hi": 500,
         "batch": 3},
        # one token of each of 64 decoding requests, most of which continue a block
        {"name": "append_decode_64", "op": "append", "model": "8b", "bits": 8, "n_req": 64, "rows": 1, "ctx_lo": 512, "ctx_hi": 8192,
         "batch": 3},
        # a chunk of prompt of the larger model far into its context, bf16 pool
        {"name": "append_chunk_14b", "op": "append", "model": "14b", "bits": 16, "n_req": 1, "rows": 2001, "ctx_lo": 100003,
         "ctx_hi": 100003, "batch": 3},
        # a long prompt at once, behind nine tokens that are there already
        {"name": "append_prompt", "op": "append", "model": "8b", "bits": 8, "n_req": 1, "rows": 16001, "ctx_lo": 9, "ctx_hi": 9,
         "batch": 3},
        # the smallest attention: three short requests of the test model, head_dim 64
        {"name": "attend_tiny_3", "op": "attend", "model": "tiny", "bits": 8, "n_req": 3, "blocks": "4,8", "verify": "block",
         "ctx_lo": 20, "ctx_hi": 200, "branches": 0, "batch": 3},
        # plain decoding: one token of each of sixteen requests
        {"name": "attend_decode_16", "op": "attend", "model": "8b", "bits": 8, "n_req": 16, "blocks": "0", "verify": "1",
         "ctx_lo": 512, "ctx_hi": 8192, "branches": 0, "batch": 3},
        # the ordinary serving batch, with one correction branch each
        {"name": "attend_8b_16", "op": "attend", "model": "8b", "bits": 8, "n_req": 16, "blocks": "4,8,16,32", "verify": "block",
         "ctx_lo": 512, "ctx_hi": 8192, "branches": 1, "batch": 3},
        # one token far into a very long context
        {"name": "attend_decode_long", "op": "attend", "model": "8b", "bits": 8, "n_req": 1, "blocks": "0", "verify": "1",
         "ctx_lo": 131071, "ctx_hi": 131071, "branches": 0, "batch": 3},
        # a chunk of prompt of the larger model, six thousand tokens into its context
        {"name": "attend_14b_chunk", "op": "attend", "model": "14b", "bits": 8, "n_req": 1, "blocks": "0", "verify": "1001",
         "ctx_lo": 6000, "ctx_hi": 6000, "branches": 0, "batch": 3},
        # one user's round over a bf16 pool that looks back a thousand tokens
        {"name": "window_round_1", "op": "window", "model": "8b", "bits": 16, "n_req": 1, "blocks": "16", "verify": "block",
         "ctx_lo": 8192, "ctx_hi": 8192, "branches": 0, "sink": 4, "window": 1024, "batch": 3},
        # sixteen decoding requests of long contexts, 8 bits, a window of two thousand tokens that is no multiple of anything
        {"name": "window_decode_16", "op": "window", "model": "8b", "bits": 8, "n_req": 16, "blocks": "0", "verify": "1",
         "ctx_lo": 2000, "ctx_hi": 16384, "branches": 0, "sink": 4, "window": 2001, "batch": 3},
        # a chunk of prompt behind sixteen thousand tokens, of which the first hundred and the last thousand count
        {"name": "window_chunk", "op": "window", "model": "8b", "bits": 16, "n_req": 1, "blocks": "0", "verify": "1001",
         "ctx_lo": 16000, "ctx_hi": 16000, "branches": 0, "sink": 100, "window": 1000, "batch": 3},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "append", "attend", "attend", "attend", "window", "window"])
    batch = rng.randrange(1, 1 << 20)
    model = rng.choice(["tiny", "8b", "8b", "14b"])
    if op == "append":
        n_req = _log_int(rng, 1, 64)
        ctx_hi = _log_int(rng, 1, 200000)
        return {"op": op, "model": model, "bits": rng.choice([8, 8, 16, 4]), "n_req": n_req,
                "rows": _log_int(rng, 1, (12000 if model == "14b" else 16000) // n_req), "ctx_lo": rng.randrange(0, ctx_hi),
                "ctx_hi": ctx_hi, "batch": batch}
    kind = rng.choice(["decode", "round", "round", "chunk"])
    if kind == "decode":
        n_req = _log_int(rng, 1, 64)
        blocks, verify, ctx_hi = "0", "1", _log_int(rng, 16, min(100000, 160000 // n_req))
    elif kind == "round":
        n_req = _log_int(rng, 1, 24)
        blocks, verify, ctx_hi = rng.choice(["4,8,16,32", "2,4,8,16", "8,16", "16", "32", "8"]), "block", _log_int(rng, 16, 8192)
    else:
        n_req = 1
        blocks, verify, ctx_hi = "0", str(_log_int(rng, 33, 1000)), _log_int(rng, 16, 6000)
    c = {"op": op, "model": model, "bits": 8, "n_req": n_req, "blocks": blocks, "verify": verify,
         "ctx_lo": rng.randrange(0, ctx_hi // 2), "ctx_hi": ctx_hi,
         "branches": rng.choice([0, 0, 1, 2]) if kind == "round" and n_req <= 8 else 0, "batch": batch}
    if op == "window":
        c.update(bits=rng.choice([8, 16]), sink=rng.choice([0, 1, 4, 64, 100]), window=_log_int(rng, 1, 5000))
    return c


# ---- lengths and masks --------------------------------------------------------------------------------------------------
def _lengths(case):
    """Per request: committed tokens, verify rows, mask rows, branches (their draft index, and masks per branch)."""
    rng = np.random.default_rng(case["batch"])
    n = case["n_req"]
    ctx = rng.integers(case["ctx_lo"], case["ctx_hi"] + 1, size=n)
    if case["op"] == "append":
        return ctx, np.full(n, case["rows"]), np.zeros(n, dtype=int), [[]] * n
    block = rng.choice([int(b) for b in case["blocks"].split(",")], size=n)
    verify = block.copy() if case["verify"] == "block" else np.full(n, int(case["verify"]))
    corr = []
    for v in verify:
        k = min(case["branches"], int(v) - 1)
        corr.append(sorted(rng.choice(np.arange(1, int(v)), size=k, replace=False).tolist()) if k > 0 else [])
    return ctx, verify, block, corr


def _plan(case):
    """The rows of the batch (request, position, and what each sees: positions <= limit and positions in [lo, hi)) and the
    scattered pages."""
    ctx, verify, block, corr = _lengths(case)
    req, at, limit, lo, hi, rows = [], [], [], [], [], []
    for r, (L, v, b, cs) in enumerate(zip(ctx, verify, block, corr)):
        L, v, b = int(L), int(v), int(b)
        n = v + b + len(cs) * (1 + b)
        rows.append(n)
        req += [r] * n
        at += range(L, L + v + b)
        limit += list(range(L, L + v)) + [L + v - 1] * b
        lo += [0] * v + [L + v] * b
        hi += [0] * v + [L + v + b] * b
        for k, i in enumerate(cs):
            first = L + v + b + k * (1 + b)
            at += range(L + i, L + i + 1 + b)
            limit += [L + i - 1] * (1 + b)
            lo += [first] * (1 + b)
            hi += [first + 1] + [first + 1 + b] * b
    rows = np.array(rows)
    kv_len = ctx + rows
    need = -(-kv_len // PAGE)
    # (pages in front of the new rows are neither read nor written by an append: one page stands for all of them)
    first = ctx // PAGE if case["op"] == "append" else np.zeros(len(ctx), dtype=int)
    n_pages = int((need - first).sum()) + 1
    perm = np.random.default_rng(case["batch"] + 1).permutation(n_pages)
    table = np.full((len(ctx), int(need.max())), -1, dtype=np.int32)
    taken = 1
    for r in range(len(ctx)):
        table[r, :first[r]] = perm[0]
        table[r, first[r]:need[r]] = perm[taken:taken + need[r] - first[r]]
        taken += need[r] - first[r]
    return {"ctx": ctx, "verify": verify, "block": block, "corr": corr, "rows": rows, "kv_len": kv_len, "table": table,
            "n_pages": n_pages, "req": np.array(req), "at": np.array(at), "limit": np.array(limit), "lo": np.array(lo),
            "hi": np.array(hi)}


def _inputs(case, seed):
    """The tensors of a case from its seed.  append: q, k, v rows of the batch and, padded to sixteen, what stands in front of them in
    their first block.  Otherwise: K and V of every request, padded to the longest, and rotated queries.

    Values as attention meets them: unit variance, with one channel of K in 32 that is large and off centre, and rows of V that
    differ in size."""
    nq, nkv, d = _HEADS[case["model"]]
    plan = _plan(case)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rand = lambda *shape: torch.randn(shape, generator=g, device="cuda")

    def kv(*shape):
        k = rand(*shape, nkv, d)
        k[..., ::32] = 3.0 * k[..., ::32] + 4.0
        return k.bfloat16(), (rand(*shape, nkv, d) * torch.exp(0.5 * rand(*shape, nkv, 1))).bfloat16()

    C, T = len(plan["ctx"]), int(plan["rows"].sum())
    x = {"plan": plan, "q": rand(T, nq, d).bfloat16()}
    if case["op"] == "append":
        x["k"], x["v"] = kv(T)
        x["front_k"], x["front_v"] = kv(C, PAGE)
    else:
        x["k"], x["v"] = kv(C, int(plan["kv_len"].max()))
    return x


# ---- the plain form ------------------------------------------------------------------------------------------------------
def _quantise8(x, there):
    """The values that 8 bits hold: x [C, n, kv head, d], n a multiple of 16; there [C, n]: the rows that exist."""
    C, n, nkv, d = x.shape
    b = torch.where(there[..., None, None], x.float(), 0.0).reshape(C, n // PAGE, PAGE, nkv, d)
    m, e = torch.frexp(b.abs().amax((2, 4), keepdim=True))                      # largest value = m 2^e, m in [.5, 1)
    e = torch.where(m == 0, 0, torch.clamp(torch.where(m <= 0.875, e - 9, e - 8), -60, 120))
    code = torch.ldexp(b, -e).to(torch.float8_e4m3fn).float()
    return torch.ldexp(code, e).reshape(C, n, nkv, d)


def _quantise4(x):
    """The values that 4 bits hold, sixteen levels of each row; the quotient in 64 bits, since values next to a border decide."""
    x = x.float()
    m = x.amin(-1, keepdim=True)
    s = ((x.amax(-1, keepdim=True) - m) / 15.0).bfloat16().float()
    return m + s * torch.where(s > 0, torch.round((x.double() - m.double()) / s.double()), 0.0).clamp(0, 15).float()


def _rotate(x, cos, sin):
    """x [T, heads, d], cos and sin [T, 1, d / 2], in the type of these."""
    a, b = x.to(cos.dtype).chunk(2, -1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1).bfloat16()


def _scores(q, k, s):
    """Scaled scores [C, kv head, row, query head of the group, position], -inf where the row does not see the position."""
    C, n = s["rows"].shape
    nkv, d = k.shape[2], k.shape[3]
    qp = q[s["rows"].clamp(min=0)].float().reshape(C, n, nkv, -1, d)
    S = torch.matmul(qp.permute(0, 2, 1, 3, 4).reshape(C, nkv, -1, d), k.permute(0, 2, 3, 1)) * (1.0 / math.sqrt(d))
    pos = torch.arange(k.shape[1], device=q.device)
    see = (pos <= s["limit"][..., None]) | ((pos >= s["lo"][..., None]) & (pos < s["hi"][..., None]))            # [C, n, position]
    if s["op"] == "window":
        see &= (pos < s["case"]["sink"]) | (pos > s["p"][..., None] - s["case"]["window"])
    return S.reshape(C, nkv, n, -1, k.shape[1]).masked_fill(~see[:, None, :, None, :], -math.inf)


def _padded(plan):
    """Row numbers of every request, padded with -1, and the rows' positions and masks in the same places (a place without a row
    stands at position 0 and sees that)."""
    C, n = len(plan["ctx"]), int(plan["rows"].max())
    at = np.full((C, n), -1, dtype=np.int64)
    first = np.concatenate([[0], np.cumsum(plan["rows"])])
    for r in range(C):
        at[r, :plan["rows"][r]] = np.arange(first[r], first[r + 1])
    pick = lambda a: np.where(at >= 0, a[np.maximum(at, 0)], 0)
    names = ("rows", "p", "limit", "lo", "hi")
    return dict(zip(names, (torch.as_tensor(a, device="cuda") for a in (at, *(pick(plan[k]) for k in ("at", "limit", "lo", "hi"))))))


def prepare(case, seed):
    op = case["op"]
    nq, nkv, d = _HEADS[case["model"]]
    x = _inputs(case, seed)
    plan = x["plan"]
    C, T = len(plan["ctx"]), x["q"].shape[0]
    s = {"op": op, "case": case, "q": x["q"], "k": x["k"], "v": x["v"], "heads": (nq, nkv, d), **_padded(plan)}
    if op == "append":
        s["position"] = torch.as_tensor(plan["at"], device="cuda")
        # the rows that stand in front of the new ones in their block, as the pool holds them, and where the new ones go
        front = torch.as_tensor(plan["ctx"] % PAGE, device="cuda")
        there = torch.arange(PAGE, device="cuda") < front[:, None]
        s["front"] = [_quantise8(x[t], there) for t in ("front_k", "front_v")]
        s["n_front"], s["front_there"] = front, there
    elif case["bits"] == 8:
        there = torch.arange(x["k"].shape[1], device="cuda") < torch.as_tensor(plan["kv_len"], device="cuda")[:, None]
        pad = -x["k"].shape[1] % PAGE
        full = lambda t: torch.nn.functional.pad(t, (0, 0, 0, 0, 0, pad))
        there = torch.nn.functional.pad(there, (0, pad))
        s["k"], s["v"] = (_quantise8(full(t), there)[:, :x["k"].shape[1]].contiguous() for t in (x["k"], x["v"]))
    if own:
        from paper_2609_34388_b200 import binding, synth

        shape = synth.ModelShape(n_layers=1, hidden=64, n_q_heads=nq, n_kv_heads=nkv, head_dim=d, ffn=64, vocab=64, rope_base=BASE)
        flags = {16: 0, 8: binding.FLAG_KV_8BIT, 4: binding.FLAG_KV_4BIT}[case["bits"]]
        ctx = binding.Context(binding.make_config(shape, C, max(T, 32), plan["table"].shape[1], flags))
        pool = binding.alloc_kv_pool(ctx, plan["n_pages"])
        s.update(ctx=ctx, pool=pool)
        for r in range(C):
            pos0 = int(plan["ctx"][r]) // PAGE * PAGE if op == "append" else 0
            n = int(plan["ctx"][r]) - pos0 if op == "append" else int(plan["kv_len"][r])
            k, v = (x["front_k"][r, :n], x["front_v"][r, :n]) if op == "append" else (x["k"][r, :n], x["v"][r, :n])
            if n:
                ctx.recg_kv_write(pool, plan["n_pages"], 0, plan["table"][r], pos0, k.contiguous(), v.contiguous())
        corr = {}
        if any(plan["corr"]):
            corr = {"n_corr": [len(c) for c in plan["corr"]], "corr_index": [(c + [0, 0])[:2] for c in plan["corr"]],
                    "corr_token": np.zeros((C, 2)), "corr_block": plan["block"]}
        s["batch"] = binding.Batch(plan["ctx"], plan["verify"], plan["block"], None, plan["table"], pool, plan["n_pages"], **corr)
        s["o"] = torch.empty_like(x["q"])
        # the first layer of a batch lays it out, the further ones find it there
        if op == "append":
            ctx.recg_kv_append_rotary(s["batch"], 0, x["q"], x["k"], x["v"], s["o"])
        else:
            if op == "window":
                ctx.recg_window(case["sink"], case["window"])
            s["lse"] = torch.empty((T, nq), device="cuda")
            ctx.recg_attention(s["batch"], 0, x["q"], s["o"], s["lse"])
    return s


def run(s):
    case = s["case"]
    nq, nkv, d = s["heads"]
    if s["op"] == "append":
        if own:
            s["ctx"].recg_kv_append_rotary(None, 0, s["q"], s["k"], s["v"], s["o"])
            return s["o"], *s["ctx"].recg_kv_rows(None, 0)
        # angles in 64 bits (far positions); K, whose rounding decides between two codes, in 64 too
        angle = s["position"][:, None, None] * BASE ** (torch.arange(d // 2, device="cuda", dtype=torch.float64) * (-2.0 / d))
        cos, sin = torch.cos(angle), torch.sin(angle)
        q, k, v = _rotate(s["q"], cos.float(), sin.float()), _rotate(s["k"], cos, sin), s["v"]
        if case["bits"] == 4:
            k, v = _quantise4(k).bfloat16(), _quantise4(v).bfloat16()
        elif case["bits"] == 8:
            C, n = s["rows"].shape
            size = (n + 2 * PAGE - 2) // PAGE * PAGE                             # from the start of the first block to the end of the last
            place = s["n_front"][:, None] + torch.arange(n, device="cuda")
            there = torch.arange(size, device="cuda") < s["n_front"][:, None] + n
            out = []
            for t, front in ((k, s["front"][0]), (v, s["front"][1])):
                buf = torch.zeros((C, max(size, PAGE), nkv, d), device="cuda")
                buf[:, :PAGE] = torch.where(s["front_there"][..., None, None], front, 0.0)
                index = place[..., None, None].expand(-1, -1, nkv, d)
                buf.scatter_(1, index, t.reshape(C, n, nkv, d).float())
                out.append(torch.gather(_quantise8(buf, there), 1, index).reshape(-1, nkv, d).bfloat16())
            k, v = out
        return q, k, v
    if own:
        s["ctx"].recg_attention(None, 0, s["q"], s["o"], s["lse"])
        return s["o"], s["lse"]
    S = _scores(s["q"], s["k"].float(), s)                                                    # [C, kv, n, g, Lk]
    C, _, n, g, Lk = S.shape
    top = S.amax(-1, keepdim=True)
    p = S.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.reshape(C, nkv, n * g, Lk), s["v"].float().permute(0, 2, 1, 3)).reshape(C, nkv, n, g, d) / total
    lse = (top + total.log())[..., 0]
    here = s["rows"] >= 0
    return (o.permute(0, 2, 1, 3, 4).reshape(C, n, nq, d)[here].bfloat16(), lse.permute(0, 2, 1, 3).reshape(C, n, nq)[here].contiguous())


# ---- what a pass cannot do without --------------------------------------------------------------------------------------
def _held_bytes(case):
    """K and V of a token and kv head in the pool."""
    d = _HEADS[case["model"]][2]
    return {16: 4.0 * d, 8: 2.0 * d + 2.0 / PAGE, 4: d + 8.0}[case["bits"]]


def work(case):
    nq, nkv, d = _HEADS[case["model"]]
    p = _plan(case)
    T = float(p["rows"].sum())
    if case["op"] == "append":      # rows in, q out, K and V into the pool and back out of it, as bf16 again
        return {"bytes": T * (4.0 * nq * d + 8.0 * nkv * d + 2 * nkv * _held_bytes(case)), "flops": 3.0 * T * (nq + nkv) * d}
    if case["op"] == "window":      # tokens that some row of the request sees, and those that each row does
        reach = np.array([p["at"][p["req"] == r].min() for r in range(len(p["ctx"]))]) - case["window"]
        kv = float(np.sum(p["kv_len"] - np.maximum(0, reach + 1 - case["sink"])))
        low = np.maximum(p["at"] - case["window"] + 1, 0)
        ahead = np.minimum(low, case["sink"])
        seen = ahead + np.maximum(0, p["limit"] + 1 - low) + np.maximum(0, p["hi"] - np.maximum(p["lo"], low))
    else:
        kv, seen = float(p["kv_len"].sum()), p["limit"] + 1 + p["hi"] - p["lo"]
    return {"bytes": kv * nkv * _held_bytes(case) + 4.0 * T * nq * d + 4.0 * T * nq, "flops": 4.0 * d * nq * float(np.sum(seen))}


# ---- the definition in 64 bits ------------------------------------------------------------------------------------------
def _held(block):
    """What 8 bits hold of one block [rows, heads, d], in 64 bits: numbers of four digits, and of fewer below 2^-6, times 2^e."""
    x = block.double()
    most = x.abs().amax(dim=(0, 2)).cpu().numpy()
    e = np.zeros(len(most))
    for h, a in enumerate(most):
        if a > 0:
            while e[h] > -60 and a <= 448.0 * 2.0 ** (e[h] - 1):
                e[h] -= 1
            while e[h] < 120 and a > 448.0 * 2.0 ** e[h]:
                e[h] += 1
    unit = torch.as_tensor(2.0 ** e, device=x.device)[None, :, None]
    y = x / unit
    step = torch.exp2(torch.clamp(torch.floor(torch.log2(torch.where(y == 0, torch.ones_like(y), y.abs()))), min=-6.0) - 3.0)
    return torch.round(y / step) * step * unit


def _held_rows(x):
    """The same of [n, heads, d], sixteen rows after the other."""
    return torch.cat([_held(x[i:i + PAGE]) for i in range(0, len(x), PAGE)])


def exact(case, seed):
    nq, nkv, d = _HEADS[case["model"]]
    g = nq // nkv
    x = _inputs(case, seed)
    plan = x["plan"]
    start = np.concatenate([[0], np.cumsum(plan["rows"])])
    if case["op"] == "append":
        turn = torch.as_tensor(plan["at"], device="cuda").double()[:, None] * torch.exp(
            torch.arange(d // 2, device="cuda").double() * (-2.0 / d * math.log(BASE)))
        unit = torch.polar(torch.ones_like(turn), turn)[:, None]
        rotated = []
        for t in (x["q"], x["k"]):
            z = torch.complex(t[..., :d // 2].double(), t[..., d // 2:].double()) * unit
            rotated.append(torch.cat([z.real, z.imag], -1))
        q, k, v = rotated[0], rotated[1].bfloat16(), x["v"]
        if case["bits"] == 16:
            return q, rotated[1], v.double()
        out = []
        for t, front in ((k, x["front_k"]), (v, x["front_v"])):
            if case["bits"] == 4:
                a = t.double()
                low = a.min(dim=-1, keepdim=True)[0]
                step = ((a.max(dim=-1, keepdim=True)[0] - low).float() / 15).to(torch.bfloat16).double()
                level = torch.clamp(((a - low) / torch.where(step == 0, 1.0, step)).round(), 0, 15)
                out.append(low + step * torch.where(step == 0, torch.zeros_like(a), level))
                continue
            parts = []
            for r, L in enumerate(plan["ctx"]):
                f = int(L) % PAGE
                rows = t[int(start[r]):int(start[r + 1])].double()
                if f:
                    rows = torch.cat([_held(front[r, :f]), rows])
                parts.append(_held_rows(rows)[f:])
            out.append(torch.cat(parts))
        return q, out[0], out[1]
    o = torch.empty((len(plan["req"]), nq, d), dtype=torch.float64, device="cuda")
    total = torch.empty((len(plan["req"]), nq), dtype=torch.float64, device="cuda")
    for r in range(len(plan["ctx"])):
        n = int(plan["kv_len"][r])
        K, V = x["k"][r, :n], x["v"][r, :n]
        K, V = (_held_rows(K), _held_rows(V)) if case["bits"] == 8 else (K.double(), V.double())
        a, b = int(start[r]), int(start[r + 1])
        cols = np.arange(n)
        see = (cols <= plan["limit"][a:b, None]) | ((cols >= plan["lo"][a:b, None]) & (cols < plan["hi"][a:b, None]))
        if case["op"] == "window":
            see = see & ((cols < case["sink"]) | (plan["at"][a:b, None] - cols < case["window"]))
        hide = torch.as_tensor(~see, device="cuda")
        for hq in range(nq):
            z = (x["q"][a:b, hq].double() @ K[:, hq // g].T) / math.sqrt(d)
            z[hide] = -math.inf
            total[a:b, hq] = torch.logsumexp(z, -1)
            o[a:b, hq] = torch.softmax(z, -1) @ V[:, hq // g]
    return o, total
