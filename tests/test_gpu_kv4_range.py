"""Attention and gathered weight over a 4-bit pool whose rows differ by many powers of two, by position, by row and by branch."""
import numpy as np
import pytest
import torch

from paper_2609_34388_b200 import binding, synth
from tests import _kv4, _kv4_range
from tests._util import f64

pytestmark = pytest.mark.gpu

FOUR = binding.FLAG_KV_4BIT
TINY, B8, B14 = (4, 2, 64), (32, 8, 128), (40, 8, 128)
# heads, (L, v, b) of every request, flags, whether the kernel of many rows takes it
PATHS = {
    "many rows": (B8, [(700, 9, 7), (45, 20, 0)], FOUR, True),
    "many rows, five heads": (B14, [(333, 26, 4)], FOUR, True),
    "many rows, split": (B8, [(5000, 4, 4)], FOUR, True),
    "one row": (B8, [(700, 1, 0), (45, 1, 0), (3, 0, 1)], FOUR, False),
    "one row, split": (B8, [(9000, 1, 1)], FOUR, False),
    "row groups": (B8, [(700, 9, 7), (45, 20, 0)], FOUR | binding.FLAG_SIMT_ATTENTION, False),
    "head_dim 64": (TINY, [(700, 2, 2), (45, 1, 0)], FOUR, False),
    "head_dim 64, row groups": (TINY, [(700, 9, 7), (45, 20, 0)], FOUR, False),
}


def exponents(pattern, n, most):
    """An exponent per position, from -most to most."""
    i = np.arange(n)
    return {"rising": np.rint(-most + 2 * most * i / max(n - 1, 1)), "falling": np.rint(most - 2 * most * i / max(n - 1, 1)),
            "alternating": np.where(i % 2, -most, most), "by 32": np.where(i // 32 % 2, -most, most), "by 128": np.where(i // 128 % 2, most, -most),
            "scattered": np.random.default_rng(n).integers(-most, most + 1, n), "one": np.where(i == n // 3, most, -most),
            "none": np.zeros(n)}[pattern].astype(np.float64)


def times(x, e, dim=0):
    """x 2^e, exactly (bf16 has the exponents)."""
    shape = [1] * x.ndim
    shape[dim] = -1
    return (x.double() * torch.from_numpy(2.0 ** np.asarray(e, dtype=np.float64)).view(shape)).bfloat16()


def run(path, seed, k_of, v_of, q_of, corr=None, layer=1, weights=True):
    """k_of, v_of(r, x [L + n, nkv, d]) and q_of(q [T, nq, d]) change the inputs.  Returns the outputs' distances over their bounds."""
    (nq, nkv, d), reqs, flags, many = PATHS[path]
    L, v, b = (list(x) for x in zip(*reqs))
    corr = corr or [()] * len(reqs)
    desc = synth.fixed_descriptor(L, v, b, seed=seed, corr=[[(i, 5) for i in c] for c in corr], corr_block=b)
    T = desc.n_tokens
    shape = synth.ModelShape(n_layers=2, hidden=64, n_q_heads=nq, n_kv_heads=nkv, head_dim=d, ffn=64, vocab=64)
    ctx = binding.Context(binding.make_config(shape, len(reqs), T, desc.page_table.shape[1], flags))
    pool = binding.alloc_kv_pool(ctx, desc.n_pages, fill=None)
    pool.view(torch.uint8).fill_(255)
    q = q_of(synth.queries(T, nq, d, seed=seed + 5))
    ks, vs = [], []
    for r, n in enumerate(desc.rows):
        k_, v_ = synth.kv_values(L[r] + int(n), nkv, d, seed=seed * 100 + r)
        ks.append(k_of(r, k_))
        vs.append(v_of(r, v_))
        ctx.recg_kv_write(pool, desc.n_pages, layer, desc.page_table[r], 0, ks[r].cuda(), vs[r].cuda())
    batch = binding.Batch(L, v, b, None, desc.page_table, pool, desc.n_pages, **desc.branch_kwargs())
    o, lse = torch.empty((T, nq, d), dtype=torch.bfloat16, device="cuda"), torch.empty((T, nq), device="cuda")
    ctx.recg_attention(batch, layer, q.cuda(), o, lse)
    w = torch.zeros((2, desc.n_pages, nkv, 16), device="cuda")
    if weights:
        ctx.recg_kv_weights(None, layer, q.cuda(), lse, None, w)
    ctx.recg_sync()
    w = f64(w)
    t, worst = 0, [0.0, 0.0, 0.0]
    for r, n in enumerate(desc.rows):
        n = int(n)
        see = _kv4.visible(L[r], v[r], b[r], corr[r], b[r])
        qr, got, got_lse = f64(q[t:t + n]), f64(o[t:t + n]), f64(lse[t:t + n])
        kc, vc = _kv4.codes(ks[r]), _kv4.codes(vs[r])
        want, want_lse, o_err, lse_err = _kv4_range.attention(qr, kc, vc, see, many)
        pos = np.arange(L[r] + n)
        gw, gw_err = _kv4_range.gathered(qr, kc, see, got_lse, np.ones(n)) if weights else (np.zeros((nkv, len(pos))),) * 2
        got_w = w[layer, desc.page_table[r][pos // 16], :, pos % 16].T
        over = (np.abs(got - want) / (o_err + 2.0 ** -8 * (np.abs(want) + o_err)), np.abs(got_lse - want_lse) / lse_err,
                np.abs(got_w - gw) / (gw_err + 2.0 ** -22 * gw + 1e-30))
        for i, x in enumerate(over):
            assert np.isfinite(x).all()
            worst[i] = max(worst[i], float(x.max()))
        t += n
    ctx.recg_free()
    print(path, "o, lse, weights over their bounds: %.3f %.3f %.3f" % tuple(worst))
    assert max(worst) <= 1.0, worst


@pytest.mark.parametrize("most", [9, 40])
@pytest.mark.parametrize("pattern", ["rising", "falling", "alternating", "by 32", "by 128", "scattered", "one"])
@pytest.mark.parametrize("path", PATHS)
def test_values(path, pattern, most):
    """V from 2^-most to 2^most: every scale of 32 tokens, and sums that are scaled down as larger ones come."""
    run(path, 3, lambda r, k: k, lambda r, v: times(v, exponents(pattern, len(v), most)), lambda q: q)


@pytest.mark.parametrize("pattern", ["rising", "falling", "alternating", "by 32", "by 128", "scattered", "one"])
@pytest.mark.parametrize("path", PATHS)
def test_keys(path, pattern):
    """K from 2^-10 to 2^10 and Q of about 2^-10: scores of order one at one end, nothing at the other."""
    run(path, 4, lambda r, k: times(k, exponents(pattern, len(k), 10)), lambda r, v: v, lambda q: times(q, np.full(len(q), -10)))


@pytest.mark.parametrize("path", PATHS)
def test_small_and_large_together(path):
    """K of 2^60 and Q of 2^-60, and the reverse."""
    for e in (60, -60):
        run(path, 5, lambda r, k: times(k, np.full(len(k), e)), lambda r, v: times(v, np.full(len(v), e)), lambda q: times(q, np.full(len(q), -e)))


@pytest.mark.parametrize("path", PATHS)
def test_queries(path):
    """Rows and heads of Q from 2^-14 to 2^2: a row's scores do not depend on its neighbours' beyond the bound."""
    def scaled(q):
        nq = q.shape[1]
        return times(times(q, np.arange(len(q)) * 5 % 17 - 14), np.where(np.arange(nq) % 3 == 1, -3, 0), 1)

    run(path, 6, lambda r, k: k, lambda r, v: v, scaled)
    run(path, 7, lambda r, k: times(k, exponents("scattered", len(k), 3)), lambda r, v: times(v, exponents("by 32", len(v), 8)), scaled)


@pytest.mark.parametrize("path,gap", [(p, g) for p in PATHS for g in (12, 16, 24, 60) if g < 60 or not PATHS[p][3]])
def test_queries_next_to_enormous_ones(path, gap):
    """Every third row and every second head is 2^gap times as large, whose attention is one position (of many rows up to the scores of which
    the attention over a bf16 pool makes sense too: it has them relative to a reference rounded as coarsely as they are)."""
    def scaled(q):
        large = (np.arange(len(q)) % 3 == 1)[:, None] | (np.arange(q.shape[1]) % 2 == 1)[None]
        return (q.double() * torch.from_numpy(np.where(large, 2.0 ** gap, 1.0))[:, :, None]).bfloat16()

    run(path, 10, lambda r, k: k, lambda r, v: v, scaled, weights=gap <= 16)      # (beyond, fp32 has no lse that a score could be compared with)


@pytest.mark.parametrize("gap", [8, 12])
@pytest.mark.parametrize("path", PATHS)
def test_large_values_that_hardly_count(path, gap):
    """V of 2^gap at positions whose scores are 40 below the others': what the others hold has to stay."""
    d = PATHS[path][0][2]
    far = lambda n: np.random.default_rng(n).random(n) < 0.1

    def keys(r, k):
        k = k.clone()
        k[:, :, 0] = torch.where(torch.from_numpy(far(len(k)))[:, None], -40 * d ** 0.5 / 8, 0.0).bfloat16()
        return k

    def queries(q):
        q = q.clone()
        q[:, :, 0] = 8.0
        return q

    run(path, 8, keys, lambda r, v: times(v, np.where(far(len(v)), gap, 0)), queries)


@pytest.mark.parametrize("path,k_gap", [("many rows", 3), ("many rows", 20), ("row groups", 3), ("row groups", 100), ("head_dim 64, row groups", 3),
                                        ("head_dim 64, row groups", 100)])
@pytest.mark.parametrize("gap", [8, 12, 30, 100])
def test_large_values_that_others_see(path, gap, k_gap):
    """The rows of a branch hold V of 2^gap and K of 2^k_gap, which the rows outside of it do not see."""
    L, v, b = PATHS[path][1][0]

    def scaled(e):
        return lambda r, x: times(x, np.where((r == 0) & (np.arange(len(x)) >= L + v + b), e, 0))

    run(path, 9, scaled(k_gap), scaled(gap), lambda q: q, corr=[(2, 5), ()], weights=k_gap == 3)


@pytest.mark.parametrize("before", [0, 5, 31])
@pytest.mark.parametrize("path", ["many rows", "many rows, five heads", "row groups", "head_dim 64, row groups"])
def test_rows_that_grow(path, before):
    """The causal rows of a chunk hold V that grows by 2^4 and K that grows by 2 a position, to 2^100 and 2^20."""
    def grown(by, most):
        return lambda r, x: times(x, np.clip((np.arange(len(x)) - (PATHS[path][1][r][0] - before)) * by, 0, most))

    run(path, 11, grown(1, 20), grown(4, 100), lambda q: q, weights=False)
