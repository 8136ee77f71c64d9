"""How exactly the row operators multiply and add: inputs on which what a product or a rounding leaves out is all
there is to see.  Bounds count roundings as rows_ref.py does (u = 2^-24; v = 2^-8 for one rounding to bf16)."""
import numpy as np
import pytest

import rows_parts as parts
import rows_ref as ref
from gpu_util import note

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def X():
    import paper_2608_00977_amd as tsid
    t = tsid.Tsid(0)
    yield t
    t.close()


def _gpu(a, dtype=np.float32):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype)).cuda()


def _table(g, rows, k, prec):
    import torch
    x = torch.from_numpy(g.standard_normal((rows, k)).astype(np.float32))
    x = (x.bfloat16() if prec == "bf16" else x).cuda()
    return x, x.double().cpu().numpy()


# ------------------------------------------- gradients' sums that cancel

# What is left out of a weight dz by the products of a gradient: two bf16 parts leave v^2 of it for
# probabilities up to 2^-6, three v^3 = u for larger ones and for fp32 factors.
def _left_out(prec, p):
    return ref.V ** 2 if prec == "bf16" and p <= 2.0 ** -6 else ref.U


@pytest.mark.parametrize("prec", ["fp32", "bf16"])
@pytest.mark.parametrize("k,T,n", [(8, 5, 100), (64, 130, 100), (128, 40, 3000), (32, 33, 40)])
def test_rows_gradient_over_equal_items(X, prec, k, T, n):
    """Every item has the same row f: dH_t = scale sum_j a_tj (f - sum_i p_ti f) = 0."""
    g = np.random.default_rng(k + n)
    f, fd = _table(g, 1, k, prec)
    F = f.expand(n, k).contiguous()
    H, _ = _table(g, T, k, prec)
    H[::2] = 0.0
    ids, a = g.integers(0, n, (T, 2)), g.standard_normal((T, 2)).astype(np.float32)
    scale = 2.0 ** -10
    note(f"equal items {prec} k={k} T={T} n={n}")
    lse = X.score(H, F, scale=scale).lse
    dH, _ = X.score_grad(H, F, lse, ids=_gpu(ids, np.int32), dlogp=_gpu(a), scale=scale, want_F=False)
    # a probability: twice the scores' error and the log sum's (lse = z + log n here); the sums' n + 2 additions
    Hd = H.double().cpu().numpy()
    z = scale * Hd @ fd[0]
    zb = ref.z_bound(Hd, np.broadcast_to(fd, (n, k)), np.zeros(n, bool), scale, 1.0, None)
    rel = 2 * zb + ref.lse_bound(zb, z + np.log(n), n) + (8 + 2 * (n + 2)) * ref.U + _left_out(prec, 1.0 / n)
    bound = scale * (np.abs(a.astype(np.float64)).sum(1) * rel)[:, None] * np.abs(fd)
    got = np.abs(dH.double().cpu().numpy())
    assert np.all(got <= bound * (1 + ref.V)), float((got / bound).max())


@pytest.mark.parametrize("prec", ["fp32", "bf16"])
@pytest.mark.parametrize("k,T,n", [(16, 8, 100), (64, 132, 300), (128, 40, 3001)])
def test_items_gradient_of_opposite_rows(X, prec, k, T, n):
    """Rows in fours, h, h, h and -h, with weights a, a, a and 3 a and scores that differ by 2^-16 at most: but for
    that dF_i = scale sum_t dz_ti h_t = 0."""
    g = np.random.default_rng(k + T)
    F, Fd = _table(g, n, k, prec)
    h, _ = _table(g, T // 4, k, prec)
    H = h.repeat_interleave(4, 0)
    H[3::4] *= -1
    a = np.repeat(g.standard_normal(T // 4).astype(np.float32), 4)
    a[3::4] *= 3
    ids = np.repeat(g.integers(0, n, T // 4), 4)
    scale = 2.0 ** -24
    note(f"opposite rows {prec} k={k} T={T} n={n}")
    lse = X.score(H, F, scale=scale).lse
    _, dF = X.score_grad(H, F, lse, ids=_gpu(ids[:, None], np.int32), dlogp=_gpu(a[:, None]), scale=scale, want_H=False)
    Hd = H.double().cpu().numpy()
    dz, _ = ref.dz_score(Hd, Fd, ids[:, None], a[:, None], None, scale, None)
    want = scale * dz.T @ Hd
    zb = ref.z_bound(Hd, Fd, np.zeros(n, bool), scale, 1.0, None)
    rel = 2 * zb + ref.lse_bound(zb, np.full(T, np.log(n)), n) + (8 + 2 * T) * ref.U + _left_out(prec, 1.0 / n)
    # the dense terms, and the listed ones (exact products, T additions)
    w = np.abs(a.astype(np.float64))
    dense = ((w * rel)[:, None] * np.abs(Hd)).sum(0)[None, :] / n
    listed = np.zeros((n, k))
    np.add.at(listed, ids, w[:, None] * np.abs(Hd) * 2 * T * ref.U)
    bound = scale * (dense + listed)
    off = np.abs(dF.double().cpu().numpy() - want)
    bound = bound + (ref.V if prec == "bf16" else 2 * ref.U) * (np.abs(want) + bound)
    assert np.all(off <= bound), float((off / bound).max())


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("k", [8, 64, 128])
def test_rows_beside_none_take_the_same_products(X, k, bias):
    """A row's gradient is the same bits whether the rows that share its wave are there or not: those beyond the last
    one hold no large probability, for which a third part would be multiplied."""
    import torch
    g = np.random.default_rng(k)
    n, T = 100, 128
    F = _table(g, 1, k, "bf16")[0].expand(n, k).contiguous()  # equal items: all that is seen is what is left out
    H, _ = _table(g, T, k, "bf16")
    b = torch.full((n,), 3.0, device="cuda") if bias else None
    ids, a = _gpu(g.integers(0, n, (T, 1)), np.int32), _gpu(g.standard_normal((T, 1)))
    lse = X.score(H, F, scale=0.01, bias=b).lse
    call = lambda t: X.score_grad(H[:t], F, lse[:t].contiguous(), ids=ids[:t].contiguous(), dlogp=a[:t].contiguous(),  # noqa: E731
                                  scale=0.01, bias=b, want_F=False)[0]
    note(f"rows beside none k={k} bias={bias}")
    whole = call(T)
    assert torch.count_nonzero(whole) > 0
    for t in (1, 31, 33, 100, 127):
        assert torch.equal(call(t), whole[:t]), t


# ------------------------------------- the products of three bf16 parts

@pytest.mark.parametrize("many", [False, True])
@pytest.mark.parametrize("k", [8, 16, 32, 64, 128])
def test_scores_multiply_all_parts_of_fp32_factors(X, k, many):
    """One item, and rows with one factor each: a log sum is one product of factors, nothing is added to it."""
    import torch
    x, y = parts.three_parts()
    T = max(k, 40) if many else min(k, 32)
    H = torch.zeros((T, k), device="cuda")
    at = torch.arange(T, device="cuda")
    H[at, (at + (k - 32 if k > 32 and not many else 0)) % k] = float(x)
    F = torch.full((1, k), float(y), device="cuda")
    note(f"products of parts k={k} many={many}")
    for scale in (1.0, -1.0):
        lse = X.score(H, F, scale=scale).lse.double().cpu().numpy()
        # the six products, the exponent's constant, the exponential of what its rounding leaves (2 u), the result
        bound = (parts.PARTS + 1 + 2 + 1) * ref.U * float(x) * float(y)
        assert np.all(np.abs(lse - scale * float(x) * float(y)) <= bound)


@pytest.mark.parametrize("k", [8, 16, 32, 64, 128])
def test_gradients_multiply_all_parts_of_fp32_factors(X, k):
    """Three items of equal scores, one listed, p = 1 / 3: a gradient's entries are one product of p and a factor."""
    import torch
    _, y = parts.three_parts()
    rows = torch.full((1, k), float(y), device="cuda")
    one = torch.ones((1, 1), device="cuda")
    ids = torch.zeros((1, 1), dtype=torch.int32, device="cuda")
    # p: the log sum's correction, the exponent and its exponential (1 u, 1 u, 2 u); the scale by a, the result
    bound = (parts.PARTS + 4 + 2) * ref.U * float(y) / 3
    note(f"products of parts, gradients k={k}")
    F, H = torch.zeros((3, k), device="cuda"), torch.zeros((1, k), device="cuda")
    F[2] = rows[0]  # dH = f_0 - (f_0 + f_1 + f_2) / 3
    dH, _ = X.score_grad(H, F, X.score(H, F).lse, ids=ids, dlogp=one, want_F=False)
    assert np.all(np.abs(dH.double().cpu().numpy() + float(y) / 3) <= bound)
    F = torch.zeros((3, k), device="cuda")  # dF = (2 / 3, -1 / 3, -1 / 3) h
    _, dF = X.score_grad(rows, F, X.score(rows, F).lse, ids=ids, dlogp=one, want_H=False)
    want = np.array([2.0, -1.0, -1.0])[:, None] * float(y) / 3
    assert np.all(np.abs(dF.double().cpu().numpy() - want) <= bound + 2 * ref.U * float(y))  # the sum with the listed part
