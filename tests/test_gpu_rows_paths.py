"""The row operators' courses that sizes choose: listed items sorted beside the pass's parts, sums of rows of every
length."""
import numpy as np
import pytest

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


def _near(got, want, bound, v, what):
    off = np.abs(got.double().cpu().numpy() - want)
    bound = bound + v * (np.abs(want) + bound)
    assert np.all(off <= bound), (what, float((off - bound).max()))


# More than 2^24 comparisons of ids by the workgroups of the items' pass (128 items each), so that the listed
# items' part is sorted: 24 x 800,000, 782 x 25,000.
@pytest.mark.parametrize("prec", ["fp32", "bf16"])
@pytest.mark.parametrize("T,n,m,k", [(2000, 3000, 400, 16), (250, 100_003, 100, 32)])
def test_gradients_with_sorted_listed_items(X, prec, T, n, m, k):
    import torch
    g = np.random.default_rng(T + m)
    assert -(-n // 128) * T * m > 2 ** 24
    H, Hd = _table(g, T, k, prec)
    F, Fd = _table(g, n, k, prec)
    b = g.normal(0, 1, n).astype(np.float32)
    out = g.random(n) < 0.1
    out[[7, 8, 9, n - 1]] = False
    b[out] = -np.inf
    F[torch.from_numpy(out).cuda()] = float("nan")
    Fd[out] = 0.0
    ids = g.integers(-1, n, (T, m))
    ids[:, :3], ids[:, 3], ids[:100, 4] = 7, n - 1, 8  # 6,000 (750), 2,000 (250) and 100 entries of one item
    ids[:, 5] = np.flatnonzero(out)[3]
    ids[T // 2] = -1
    a, e = g.standard_normal((T, m)).astype(np.float32), g.standard_normal(T).astype(np.float32)
    scale = 0.25
    note(f"sorted listed items {prec} T={T} n={n} m={m}")
    i, bg = _gpu(ids, np.int32), _gpu(b)
    r = X.score(H, F, scale=scale, bias=bg, entropy=True)
    call = lambda: X.score_grad(H, F, r.lse, ids=i, dlogp=_gpu(a), entropy=r.entropy, dentropy=_gpu(e), scale=scale,  # noqa: E731
                                bias=bg)
    got = call()
    dz, size = ref.dz_score(Hd, Fd, ids, a, e, scale, b)
    lse, zb = ref.softmax_over(Hd, Fd, scale, b, 1.0)[1], ref.z_bound(Hd, Fd, out, scale, 1.0, b)
    # a row adds n terms and m listed ones; an item T terms and its entries by pieces of 64 of pieces of 64
    bounds = ref.grad_bounds(size, Hd, Fd, out, scale, zb, lse, n + m, T + 130 + T * m // 4096, prec == "bf16")
    v = ref.V if prec == "bf16" else 2 * ref.U
    for x, w, bound, what in zip(got, ref.grads(dz, Hd, Fd, out, scale), bounds, ("dH", "dF")):
        _near(x, w, bound, v, what)
    assert torch.count_nonzero(got[1][torch.from_numpy(out).cuda()]) == 0
    again = call()
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])
    # the same through a distillation's weights
    tau, t, d = 2.0, _gpu(2 * a), _gpu(e)
    loss, lse_d = X.distill(H, F, i, t, scale=scale, temperature=tau, bias=bg)
    got = X.distill_grad(H, F, i, t, lse_d, d, scale=scale, temperature=tau, bias=bg)
    want, wlse = ref.distill(Hd, Fd, ids, 2 * a, scale, b, tau)
    zb = ref.z_bound(Hd, Fd, out, scale, tau, b)
    assert np.all(np.abs(loss.double().cpu().numpy() - want) <= tau * tau * ref.lse_bound(zb, wlse, n) + 4 * ref.U * np.abs(want))
    dz, size = ref.dz_distill(Hd, Fd, ids, 2 * a, e, scale, b, tau)
    bounds = ref.grad_bounds(size, Hd, Fd, out, scale / tau, zb, wlse, n + m, T + 130 + T * m // 4096, prec == "bf16")
    for x, w, bound, what in zip(got, ref.grads(dz, Hd, Fd, out, scale / tau), bounds, ("dH", "dF")):
        _near(x, w, bound, v, what)
    X.rows_check()


# Whole numbers, whose sums are exact in fp32, so that only the result is rounded.
@pytest.mark.parametrize("prec", ["fp32", "bf16"])
@pytest.mark.parametrize("k", [8, 32, 128])
@pytest.mark.parametrize("n", [50_021, 100_000, 2_003])  # few rows named, and many
def test_lookup_gradient_of_rows_of_every_length(X, prec, k, n):
    import torch
    g = np.random.default_rng(n + k)
    lengths = [1, 2, 3, 4, 5, 63, 64, 65, 66, 127, 128, 129, 700, 4096, 4097, 1, 0, 2, 1, 65]
    rows = list(range(4, 4 + len(lengths) - 2)) + [n - 2, n - 1]  # beside one another, and the last two
    ids = np.concatenate([np.full(c, r) for r, c in zip(rows, lengths)] + [g.integers(100, n - 2, 600), np.full(37, -1)])
    ids = g.permutation(ids)
    assert 2048 < len(ids)
    G = g.integers(-8, 9, (len(ids), k)).astype(np.float32)
    want = np.zeros((n, k))
    np.add.at(want, ids[ids >= 0], G[ids >= 0])
    Gt = _gpu(G).bfloat16() if prec == "bf16" else _gpu(G)
    note(f"lookup gradient, rows of every length {prec} k={k} n={n}")
    for scale in (1.0, -0.5):
        got = X.lookup_grad(Gt, _gpu(ids, np.int32), n, scale=scale)
        assert torch.equal(got.cpu(), torch.from_numpy((scale * want).astype(np.float32)).to(Gt.dtype))
    X.rows_check()
