"""The operators around a small KV cache, as measurable cases: a cache held in 4 bits and the attention that reads it, and
the eviction of cached tokens by the attention weight that they have gathered.

  store    K and V rows go into a 4-bit pool and come back as the values that it holds: rows of a batch (`recg_kv_append`,
           `recg_kv_rows`) or the prefix of one request (`recg_kv_write`, `recg_kv_read`)
  attend   hybrid-mask paged attention over a 4-bit pool, with the log-sum-exp of every row (`recg_attention`)
  weights  the attention weight that every cached token receives from the rows of a batch, added up over the rounds
           (`recg_kv_weights`)
  evict    which tokens every kv head keeps, and the move of their K, V and weights to other pages (`recg_kv_select`,
           `recg_kv_compact`)

The 4-bit format, per token, kv head and K or V: m = min x, s = bf16((max x - m) / 15), c = the nearest whole number to
(x - m) / s (ties to even, 0 where s is 0); the pool stands for m + s c.

Shapes, block sizes and context ranges are those of the package's configurations, tests and benchmark.  The lengths of a
batch follow from the case alone (`batch` seeds them), every tensor from `prepare`'s seed.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16

# (query heads, kv heads, head_dim): the 2-layer test model, the 8B class, the 14B class with five query heads per kv head
_HEADS = {"tiny": (4, 2, 64), "8b": (32, 8, 128), "14b": (40, 8, 128)}


def listed():
    return [
        # one token of one user goes into the cache: launches and latency are all there is
        {"name": "store_one_token", "op": "store", "model": "8b", "how": "rows", "n_req": 1, "rows": 1, "ctx": 500, "batch": 3},
        # the prefix of one request computed elsewhere comes into the pool, behind nine tokens that are there already
        {"name": "store_prefix", "op": "store", "model": "8b", "how": "prefix", "n_req": 1, "rows": 16001, "ctx": 9, "batch": 3},
        # the smallest attention: three short requests of the test model, head_dim 64
        {"name": "attend_tiny_3", "op": "attend", "model": "tiny", "n_req": 3, "blocks": "4,8", "verify": "block", "ctx_lo": 20,
         "ctx_hi": 200, "branches": 0, "batch": 3},
        # one user, low latency: 16 verify rows and 16 mask rows over 4096 tokens
        {"name": "attend_8b_1", "op": "attend", "model": "8b", "n_req": 1, "blocks": "16", "verify": "block", "ctx_lo": 4096,
         "ctx_hi": 4096, "branches": 0, "batch": 3},
        # plain decoding: one token of each of sixteen requests
        {"name": "attend_decode_16", "op": "attend", "model": "8b", "n_req": 16, "blocks": "0", "verify": "1", "ctx_lo": 512,
         "ctx_hi": 8192, "branches": 0, "batch": 3},
        # the ordinary serving batch, with one correction branch each
        {"name": "attend_8b_16", "op": "attend", "model": "8b", "n_req": 16, "blocks": "4,8,16,32", "verify": "block",
         "ctx_lo": 512, "ctx_hi": 8192, "branches": 1, "batch": 3},
        # one token far into a very long context
        {"name": "attend_decode_long", "op": "attend", "model": "8b", "n_req": 1, "blocks": "0", "verify": "1", "ctx_lo": 131071,
         "ctx_hi": 131071, "branches": 0, "batch": 3},
        # a chunk of prompt of the larger model, six thousand tokens into its context
        {"name": "attend_14b_chunk", "op": "attend", "model": "14b", "n_req": 1, "blocks": "0", "verify": "1001", "ctx_lo": 6000,
         "ctx_hi": 6000, "branches": 0, "batch": 3},
        # the weights of sixteen decoding requests, 4-bit keys
        {"name": "weights_decode_16", "op": "weights", "model": "8b", "bits": 4, "n_req": 16, "blocks": "0", "verify": "1",
         "ctx_lo": 512, "ctx_hi": 8192, "branches": 0, "decay": 1.0, "batch": 3},
        # the weights of a serving batch, bf16 keys; only verify rows count, and old weight fades
        {"name": "weights_8b_16", "op": "weights", "model": "8b", "bits": 16, "n_req": 16, "blocks": "4,8,16,32",
         "verify": "block", "ctx_lo": 512, "ctx_hi": 8192, "branches": 0, "decay": 0.98, "batch": 3},
        # one request is cut to a quarter, one layer of a bf16 pool
        {"name": "evict_1", "op": "evict", "model": "8b", "bits": 16, "layers": 1, "n_req": 1, "ctx_lo": 4096, "ctx_hi": 4096,
         "keep": 0.25, "sink": 4, "recent": 64, "batch": 3},
        # four long requests are cut to a third, eight layers of a 4-bit pool at once
        {"name": "evict_4_long", "op": "evict", "model": "8b", "bits": 4, "layers": 8, "n_req": 4, "ctx_lo": 8192, "ctx_hi": 16384,
         "keep": 0.33, "sink": 4, "recent": 256, "batch": 3},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["store", "attend", "attend", "attend", "weights", "weights", "evict"])
    batch = rng.randrange(1, 1 << 20)
    if op == "store":
        how = rng.choice(["rows", "prefix"])
        n_req = _log_int(rng, 1, 64) if how == "rows" else 1
        return {"op": op, "model": rng.choice(["tiny", "8b", "8b"]), "how": how, "n_req": n_req,
                "rows": _log_int(rng, 1, 2000 // n_req if how == "rows" else 16000), "ctx": rng.randrange(0, 2000), "batch": batch}
    if op == "evict":
        n_req = rng.choice([1, 1, 2, 3, 4])
        ctx_hi = _log_int(rng, 200, 16384)
        return {"op": op, "model": rng.choice(["8b", "8b", "tiny"]), "bits": rng.choice([4, 16]), "layers": rng.choice([1, 2, 4]),
                "n_req": n_req, "ctx_lo": ctx_hi // 2, "ctx_hi": ctx_hi, "keep": round(rng.uniform(0.1, 0.95), 2),
                "sink": rng.choice([0, 4, 16]), "recent": rng.choice([0, 1, 16, 61]), "batch": batch}
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
    c = {"op": op, "model": rng.choice(["tiny", "8b", "8b", "14b"]), "n_req": n_req, "blocks": blocks, "verify": verify,
         "ctx_lo": rng.randrange(0, ctx_hi // 2), "ctx_hi": ctx_hi,
         "branches": rng.choice([0, 0, 1, 2]) if kind == "round" and n_req <= 8 else 0, "batch": batch}
    if op == "weights":
        c.update(bits=rng.choice([4, 16]), decay=rng.choice([1.0, 0.98, 0.5]))
    return c


# ---- lengths and masks --------------------------------------------------------------------------------------------------
def _lengths(case):
    """Per request: committed tokens, verify rows, mask rows, branches (their draft index, and masks per branch)."""
    rng = np.random.default_rng(case["batch"])
    n = case["n_req"]
    if case["op"] == "store":
        ctx = rng.integers(0, case["ctx"] + 1, size=n) if n > 1 else np.array([case["ctx"]])
        return ctx, np.full(n, case["rows"]), np.zeros(n, dtype=int), [[]] * n
    ctx = rng.integers(case["ctx_lo"], case["ctx_hi"] + 1, size=n)
    if case["op"] == "evict":
        return ctx, np.ones(n, dtype=int), np.zeros(n, dtype=int), [[]] * n
    block = rng.choice([int(b) for b in case["blocks"].split(",")], size=n)
    verify = block.copy() if case["verify"] == "block" else np.full(n, int(case["verify"]))
    corr = []
    for v in verify:
        k = min(case["branches"], int(v) - 1)
        corr.append(sorted(rng.choice(np.arange(1, int(v)), size=k, replace=False).tolist()) if k > 0 else [])
    return ctx, verify, block, corr


def _plan(case):
    """The rows of the batch (request, and what each sees: positions <= limit and positions in [lo, hi)) and the scattered pages."""
    ctx, verify, block, corr = _lengths(case)
    req, limit, lo, hi, is_verify = [], [], [], [], []
    rows = []
    for r, (L, v, b, cs) in enumerate(zip(ctx, verify, block, corr)):
        L, v, b = int(L), int(v), int(b)
        n = v + b + len(cs) * (1 + b)
        rows.append(n)
        req += [r] * n
        limit += list(range(L, L + v)) + [L + v - 1] * b
        lo += [0] * v + [L + v] * b
        hi += [0] * v + [L + v + b] * b
        for k, i in enumerate(cs):
            first = L + v + b + k * (1 + b)
            limit += [L + i - 1] * (1 + b)
            lo += [first] * (1 + b)
            hi += [first + 1] + [first + 1 + b] * b
        is_verify += [1.0] * v + [0.0] * (n - v)
    rows = np.array(rows)
    kv_len = ctx + rows
    need = -(-kv_len // PAGE)
    perm = np.random.default_rng(case["batch"] + 1).permutation(2 * int(need.sum()))
    table = np.full((len(ctx), int(need.max())), -1, dtype=np.int32)
    other = table.copy()                                       # pages to which an eviction moves what it keeps
    at = np.concatenate([[0], np.cumsum(need)])
    for r in range(len(ctx)):
        table[r, :need[r]] = perm[at[r]:at[r + 1]]
        other[r, :need[r]] = perm[at[-1] + at[r]:at[-1] + at[r + 1]]
    return {"ctx": ctx, "verify": verify, "block": block, "corr": corr, "rows": rows, "kv_len": kv_len, "table": table,
            "other": other, "n_pages": 2 * int(need.sum()), "req": np.array(req), "limit": np.array(limit), "lo": np.array(lo),
            "hi": np.array(hi), "is_verify": np.array(is_verify, dtype=np.float32)}


def _budget(case, ctx):
    return np.minimum(ctx, np.maximum((ctx * case["keep"]).astype(int), case["sink"] + case["recent"] + 1))


def _inputs(case, seed):
    """The tensors of a case from its seed: K and V of every request, padded to the longest, queries, gathered weights.

    Values as attention meets them: unit variance, with one channel of K in 32 that is large and off centre; weights spread over
    several powers of e, one in ten tokens without any (their order is a tie)."""
    nq, nkv, d = _HEADS[case["model"]]
    plan = _plan(case)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    rand = lambda *shape: torch.randn(shape, generator=g, device="cuda")
    C, Lk, T = len(plan["ctx"]), int(plan["kv_len"].max()), int(plan["rows"].sum())
    layers = case.get("layers", 1)
    k = rand(layers, C, Lk, nkv, d)
    k[..., ::32] = 3.0 * k[..., ::32] + 4.0
    x = {"plan": plan, "k": k.bfloat16(), "v": rand(layers, C, Lk, nkv, d).bfloat16(), "q": rand(T, nq, d).bfloat16()}
    if case["op"] in ("weights", "evict"):
        w = torch.exp(2.0 * rand(layers, plan["n_pages"], nkv, PAGE))
        x["w"] = torch.where(torch.rand(w.shape, generator=g, device="cuda") < 0.1, torch.zeros_like(w), w)
    return x


# ---- the plain form ------------------------------------------------------------------------------------------------------
def _quantise(x):
    """codes, scale and minimum of the last axis; the quotient in 64 bits, since values next to a border decide."""
    x = x.float()
    m = x.amin(-1, keepdim=True)
    s = ((x.amax(-1, keepdim=True) - m) / 15.0).bfloat16().float()
    c = torch.where(s > 0, torch.round((x.double() - m.double()) / s.double()), 0.0).clamp(0, 15)
    return c.to(torch.uint8), s, m


def _value(code):
    c, s, m = code
    return m + s * c.float()


def _slots(table, n):
    """Slot (page * 16 + offset) of positions 0 .. n-1 of every request; -1 behind its pages."""
    pos = torch.arange(n, device=table.device)
    return torch.where(table[:, pos // PAGE] >= 0, table[:, pos // PAGE] * PAGE + pos % PAGE, -1)


def _scores(q, k, at, limit, lo, hi):
    """Scaled scores [C, kv head, row, query head of the group, position], -inf where the row does not see the position."""
    C, n = at.shape
    nkv, d = k.shape[2], k.shape[3]
    qp = q[at.clamp(min=0)].float().reshape(C, n, nkv, -1, d)
    s = torch.matmul(qp.permute(0, 2, 1, 3, 4).reshape(C, nkv, -1, d), k.permute(0, 2, 3, 1)) * (1.0 / math.sqrt(d))
    pos = torch.arange(k.shape[1], device=q.device)
    see = (pos <= limit[..., None]) | ((pos >= lo[..., None]) & (pos < hi[..., None]))            # [C, n, position]
    return s.reshape(C, nkv, n, -1, k.shape[1]).masked_fill(~see[:, None, :, None, :], -math.inf)


def _padded(plan):
    """Row numbers of every request, padded with -1, and the rows' masks in the same places (a place without a row sees
    position 0)."""
    C, n = len(plan["ctx"]), int(plan["rows"].max())
    at = np.full((C, n), -1, dtype=np.int64)
    first = np.concatenate([[0], np.cumsum(plan["rows"])])
    for r in range(C):
        at[r, :plan["rows"][r]] = np.arange(first[r], first[r + 1])
    pick = lambda a, none: np.where(at >= 0, a[np.maximum(at, 0)], none)
    return [torch.as_tensor(a, device="cuda") for a in (at, pick(plan["limit"], 0), pick(plan["lo"], 0), pick(plan["hi"], 0))]


def prepare(case, seed):
    op = case["op"]
    nq, nkv, d = _HEADS[case["model"]]
    x = _inputs(case, seed)
    plan = x["plan"]
    s = {"op": op, "case": case, "plan": plan, "q": x["q"], "heads": (nq, nkv, d)}
    C, Lk, T = len(plan["ctx"]), x["k"].shape[2], x["q"].shape[0]
    s["table"], s["other"] = (torch.as_tensor(plan[t], device="cuda").long() for t in ("table", "other"))
    s["at"], s["limit"], s["lo"], s["hi"] = _padded(plan)
    s["row_req"] = torch.as_tensor(plan["req"], device="cuda")
    start = np.concatenate([[0], np.cumsum(plan["rows"])[:-1]])
    s["row_pos"] = torch.as_tensor(plan["ctx"][plan["req"]] + np.arange(T) - start[plan["req"]], device="cuda")
    if op == "store":
        s["k"], s["v"] = (t[0][s["row_req"], s["row_pos"]].contiguous() for t in (x["k"], x["v"]))
    elif case.get("bits", 4) == 4:
        s["k"], s["v"] = [_quantise(x["k"]), _quantise(x["v"])]
    else:
        s["k"], s["v"] = x["k"], x["v"]
    if op in ("weights", "evict"):
        s["w"], s["w_out"] = x["w"], x["w"].clone()
        s["n_ctx"] = torch.as_tensor(plan["ctx"], device="cuda")
    if op == "weights":
        s["row_weight"] = torch.as_tensor(plan["is_verify"], device="cuda")
        k = _value([t[0] for t in s["k"]]) if case["bits"] == 4 else s["k"][0].float()
        lse = torch.logsumexp(_scores(x["q"], k, s["at"], s["limit"], s["lo"], s["hi"]), -1)      # [C, kv head, row, head]
        s["lse"] = torch.empty((T, nq), device="cuda")
        s["lse"][s["at"][s["at"] >= 0]] = lse.permute(0, 2, 1, 3).reshape(C, -1, nq)[s["at"] >= 0]
        del lse, k
    if op == "evict":
        s["budget"] = _budget(case, plan["ctx"])
        s["n_keep"] = torch.as_tensor(s["budget"], device="cuda")
    if own:
        from paper_2609_34388_b200 import binding, synth

        shape = synth.ModelShape(n_layers=case.get("layers", 1), hidden=64, n_q_heads=nq, n_kv_heads=nkv, head_dim=d, ffn=64, vocab=64)
        kept = int(s["budget"].sum()) if op == "evict" else 0
        four = case.get("bits", 4) == 4
        cfg = binding.make_config(shape, C, max(T, kept, 32), plan["table"].shape[1], binding.FLAG_KV_4BIT if four else 0)
        ctx = binding.Context(cfg)
        pool = binding.alloc_kv_pool(ctx, plan["n_pages"])
        s.update(ctx=ctx, pool=pool)
        if op != "store":
            for layer in range(shape.n_layers):
                for r in range(C):
                    n = int(plan["kv_len"][r])
                    ctx.recg_kv_write(pool, plan["n_pages"], layer, plan["table"][r], 0, x["k"][layer, r, :n].contiguous(),
                                      x["v"][layer, r, :n].contiguous())
        corr = {}
        if any(plan["corr"]):
            corr = {"n_corr": [len(c) for c in plan["corr"]], "corr_index": [(c + [0, 0])[:2] for c in plan["corr"]],
                    "corr_token": np.zeros((C, 2)), "corr_block": plan["block"]}
        s["batch"] = binding.Batch(plan["ctx"], plan["verify"], plan["block"], None, plan["table"], pool, plan["n_pages"], **corr)
        if op == "attend":
            s["o"] = torch.empty_like(x["q"])
            s["lse"] = torch.empty((T, nq), device="cuda")
            ctx.recg_attention(s["batch"], 0, x["q"], s["o"], s["lse"])      # lays the batch out, as the first layer does
        if op == "weights":
            ctx.recg_kv_weights(s["batch"], 0, s["q"], s["lse"], s["w"], s["w_out"], s["row_weight"], case["decay"])
        if op == "evict":
            s["eviction"] = binding.Eviction(plan["ctx"], s["budget"], plan["table"], pool, plan["n_pages"], s["w_out"],
                                             n_sink=case["sink"], n_recent=case["recent"], dst_page_table=plan["other"],
                                             layers=(0, shape.n_layers))
            s["kept"] = binding.Batch([0] * C, s["budget"], [0] * C, None, plan["other"], pool, plan["n_pages"])
    return s


def run(s):
    op, case, plan = s["op"], s["case"], s["plan"]
    nq, nkv, d = s["heads"]
    if op == "store":
        if own:
            if case["how"] == "rows":
                s["ctx"].recg_kv_append(s["batch"], 0, s["k"], s["v"])
                return s["ctx"].recg_kv_rows(None, 0)
            s["ctx"].recg_kv_write(s["pool"], plan["n_pages"], 0, plan["table"][0], case["ctx"], s["k"], s["v"])
            return s["ctx"].recg_kv_read(s["pool"], plan["n_pages"], 0, plan["table"][0], case["ctx"], case["rows"])
        return _value(_quantise(s["k"])).bfloat16(), _value(_quantise(s["v"])).bfloat16()
    if op == "attend":
        if own:
            s["ctx"].recg_attention(None, 0, s["q"], s["o"], s["lse"])
            return s["o"], s["lse"]
        k, v = _value([t[0] for t in s["k"]]), _value([t[0] for t in s["v"]])
        S = _scores(s["q"], k, s["at"], s["limit"], s["lo"], s["hi"])                             # [C, kv, n, g, Lk]
        C, _, n, g, Lk = S.shape
        top = S.amax(-1, keepdim=True)
        p = S.sub_(top).exp_()
        total = p.sum(-1, keepdim=True)
        o = torch.matmul(p.reshape(C, nkv, n * g, Lk), v.permute(0, 2, 1, 3)).reshape(C, nkv, n, g, d) / total
        lse = (top + total.log())[..., 0]
        here = s["at"] >= 0
        return (o.permute(0, 2, 1, 3, 4).reshape(C, n, nq, d)[here].bfloat16(),
                lse.permute(0, 2, 1, 3).reshape(C, n, nq)[here].contiguous())
    if op == "weights":
        if own:
            s["ctx"].recg_kv_weights(None, 0, s["q"], s["lse"], s["w"], s["w_out"], s["row_weight"], case["decay"])
            return s["w_out"]
        k = _value([t[0] for t in s["k"]]) if case["bits"] == 4 else s["k"][0].float()
        S = _scores(s["q"], k, s["at"], s["limit"], s["lo"], s["hi"])
        C, _, n, g, Lk = S.shape
        at = s["at"].clamp(min=0)
        lse = s["lse"][at].reshape(C, n, nkv, g).permute(0, 2, 1, 3)
        rw = torch.where(s["at"] >= 0, s["row_weight"][at], 0.0)
        got = (S.sub_(lse[..., None]).exp_() * rw[:, None, :, None, None]).sum((2, 3))            # [C, kv, Lk]
        slot, pos = _slots(s["table"], Lk), torch.arange(Lk, device=S.device)
        c, p = torch.nonzero(pos < torch.as_tensor(plan["kv_len"], device=S.device)[:, None], as_tuple=True)
        page, off = slot[c, p] // PAGE, slot[c, p] % PAGE
        out = s["w_out"]
        before = torch.where((p < s["n_ctx"][c])[:, None], case["decay"] * s["w"][0, page, :, off], 0.0)
        out[0, page, :, off] = before + got[c, :, p]
        return out
    # evict: the slots that stay, per layer, request and kv head; then K, V and weights of them
    if own:
        keep = torch.empty((case["layers"], len(plan["ctx"]), nkv, int(s["budget"].max())), dtype=torch.int32, device="cuda")
        s["ctx"].recg_kv_select(s["eviction"], keep)
        s["ctx"].recg_kv_compact(s["eviction"], keep)
        return keep, s["w_out"], [s["ctx"].recg_kv_rows(None if layer else s["kept"], layer) for layer in range(case["layers"])]
    L = int(plan["ctx"].max())
    slot, pos = _slots(s["table"], L), torch.arange(L, device="cuda")
    page, off = slot.clamp(min=0) // PAGE, slot.clamp(min=0) % PAGE
    w = s["w"][:, page, :, off].permute(2, 0, 3, 1).float()                                       # [layers, C, kv, L]
    n_ctx = s["n_ctx"][:, None]
    forced = (pos < case["sink"]) | (pos >= n_ctx - case["recent"])
    key = torch.where(forced[:, None], math.inf, w)
    key = torch.where((pos < n_ctx)[:, None], key, -math.inf)
    order = torch.sort(key, dim=-1, descending=True, stable=True).indices
    most = int(s["budget"].max())
    order = torch.where((pos < s["n_keep"][:, None])[:, None], order, L)[..., :most].sort(-1).values
    keep = torch.where(order < L, order, -1).to(torch.int32)
    layer, c, h, i = torch.nonzero(keep >= 0, as_tuple=True)
    src = keep[layer, c, h, i].long()
    to = _slots(s["other"], most)[c, i]
    out = s["w_out"]
    out[layer, to // PAGE, h, to % PAGE] = s["w"][layer, slot[c, src] // PAGE, h, slot[c, src] % PAGE]
    there = torch.nonzero(torch.arange(most, device="cuda") < s["n_keep"][:, None], as_tuple=True)
    kv = [(_value(t) if case["bits"] == 4 else t.float()) for t in (s["k"], s["v"])]              # [layers, C, Lk, kv, d]
    at = keep.clamp(min=0).long().permute(0, 1, 3, 2)[..., None].expand(-1, -1, -1, -1, d)
    kept = [torch.gather(t, 2, at)[:, there[0], there[1]].bfloat16() for t in kv]
    return keep, out, list(zip(kept[0].unbind(0), kept[1].unbind(0)))


# ---- what a pass cannot do without --------------------------------------------------------------------------------------
def work(case):
    nq, nkv, d = _HEADS[case["model"]]
    p = _plan(case)
    T, kv = float(p["rows"].sum()), float(p["kv_len"].sum())
    row4 = d / 2 + 4.0                                  # a row of one head in 4 bits
    row = row4 if case.get("bits", 4) == 4 else 2.0 * d
    first = p["ctx"][p["req"]]
    seen = float(np.sum(p["limit"] + 1 + p["hi"] - p["lo"]))
    if case["op"] == "store":                           # bf16 in, 4 bits out and in again, bf16 out
        return {"bytes": 2 * T * nkv * (4.0 * d + 2 * row4), "flops": 6.0 * T * nkv * d}
    if case["op"] == "attend":
        return {"bytes": 2 * kv * nkv * row4 + 4.0 * T * nq * d + 4.0 * T * nq, "flops": 4.0 * d * nq * seen}
    if case["op"] == "weights":                         # rows without a weight cost nothing
        counted = float(np.sum((p["limit"] + 1 + p["hi"] - p["lo"]) * p["is_verify"]))
        return {"bytes": kv * nkv * (row + 8.0) + 2.0 * T * nq * d + 4.0 * T * nq, "flops": 2.0 * d * nq * counted}
    n = float(_budget(case, p["ctx"]).sum())            # weights in; list out; what is kept in, out, and as bf16 values
    return {"bytes": case["layers"] * nkv * (4.0 * float(first.sum()) + n * (4.0 + 8.0 + 6 * row + 4.0 * d)), "flops": 0.0}


# ---- the definition in 64 bits ------------------------------------------------------------------------------------------
def _held(x):
    """What the 4-bit cache stands for, in 64 bits: nearest of the sixteen values between the extremes."""
    a = x.double()
    low, high = a.min(dim=-1, keepdim=True)[0], a.max(dim=-1, keepdim=True)[0]
    step = ((high - low).float() / 15).to(torch.bfloat16).double()
    level = torch.where(step == 0, torch.zeros_like(a), torch.clamp(((a - low) / torch.where(step == 0, 1.0, step)).round(), 0, 15))
    return low + step * level


def exact(case, seed):
    op = case["op"]
    nq, nkv, d = _HEADS[case["model"]]
    g = nq // nkv
    x = _inputs(case, seed)
    plan = x["plan"]
    held = _held if case.get("bits", 4) == 4 else (lambda t: t.double())
    start = np.concatenate([[0], np.cumsum(plan["rows"])])
    if op == "store":
        out = []
        for t in (x["k"], x["v"]):
            rows = [t[0, r, plan["ctx"][r]:plan["kv_len"][r]] for r in range(len(plan["ctx"]))]
            out.append(held(torch.cat(rows)))
        return tuple(out)
    if op == "evict":
        lists = []
        out = x["w"].double()
        kv = [[[], []] for _ in range(case["layers"])]
        budget = _budget(case, plan["ctx"])
        most = int(budget.max())
        for layer in range(case["layers"]):
            for r, L in enumerate(plan["ctx"]):
                slot = (plan["table"][r][np.arange(L) // PAGE] * PAGE + np.arange(L) % PAGE)
                to = (plan["other"][r][np.arange(budget[r]) // PAGE] * PAGE + np.arange(budget[r]) % PAGE)
                heads = []
                for h in range(nkv):
                    w = x["w"][layer, :, h].reshape(-1)[torch.as_tensor(slot, device="cuda")].cpu().numpy()
                    forced = (np.arange(L) < case["sink"]) | (np.arange(L) >= L - case["recent"])
                    ranked = np.lexsort((np.arange(L), -w, ~forced))[:budget[r]]
                    ids = np.sort(ranked)
                    heads.append(ids)
                    out[layer, torch.as_tensor(to // PAGE, device="cuda"), h, torch.as_tensor(to % PAGE, device="cuda")] = \
                        torch.as_tensor(w[ids], device="cuda").double()
                lists += [np.pad(i, (0, most - len(i)), constant_values=-1) for i in heads]
                for t, into in ((x["k"], kv[layer][0]), (x["v"], kv[layer][1])):
                    into.append(torch.stack([held(t[layer, r, torch.as_tensor(i, device="cuda"), h]) for h, i in enumerate(heads)], 1))
        keep = np.stack(lists).reshape(case["layers"], len(plan["ctx"]), nkv, most).astype(np.int32)
        return keep, out, [(torch.cat(a), torch.cat(b)) for a, b in kv]
    if op == "weights":
        lse = prepare(case, seed)["lse"].double()      # an input
        out = x["w"].double()
    o = torch.empty((len(plan["req"]), nq, d), dtype=torch.float64, device="cuda")
    total = torch.empty((len(plan["req"]), nq), dtype=torch.float64, device="cuda")
    for r in range(len(plan["ctx"])):
        n = int(plan["kv_len"][r])
        K, V = held(x["k"][0, r, :n]), held(x["v"][0, r, :n])
        a, b = int(start[r]), int(start[r + 1])
        cols = np.arange(n)
        see = (cols <= plan["limit"][a:b, None]) | ((cols >= plan["lo"][a:b, None]) & (cols < plan["hi"][a:b, None]))
        hide = torch.as_tensor(~see, device="cuda")
        for h in range(nkv):
            received = torch.zeros(n, dtype=torch.float64, device="cuda")
            for hq in range(h * g, (h + 1) * g):
                z = (x["q"][a:b, hq].double() @ K[:, h].T) / math.sqrt(d)
                z[hide] = -math.inf
                if op == "weights":
                    received += torch.as_tensor(plan["is_verify"][a:b], device="cuda").double() @ torch.exp(z - lse[a:b, hq, None])
                else:
                    total[a:b, hq] = torch.logsumexp(z, -1)
                    o[a:b, hq] = torch.softmax(z, -1) @ V[:, h]
            if op == "weights":
                page = torch.as_tensor(plan["table"][r][cols // PAGE], device="cuda").long()
                off = torch.as_tensor(cols % PAGE, device="cuda")
                old = torch.where(torch.as_tensor(cols < plan["ctx"][r], device="cuda"), case["decay"] * x["w"][0, page, h, off].double(), 0.0)
                out[0, page, h, off] = old + received
    return out if op == "weights" else (o, total)
