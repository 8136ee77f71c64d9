"""The row operators at the ends of what they take: scores far from zero, the paths that sizes choose, signed
zeros, what is refused."""
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


# --------------------------------------------------- scores far from zero

@pytest.mark.parametrize("prec", ["fp32", "bf16"])
@pytest.mark.parametrize("T", [3, 45])
def test_rows_far_below_zero_are_empty_in_results_and_gradients(X, prec, T):
    """Scores of about -1e8: no item of the even rows may be had; the odd rows are ordinary."""
    import torch
    g = np.random.default_rng(T)
    n, k, top = 70, 16, 4
    F, Fd = _table(g, n, k, prec)
    F[:, 0] = Fd[:, 0] = 1.0
    H, Hd = _table(g, T, k, prec)
    H[::2, 0] = -2.0 ** 27
    H[1::2, 0] = 0.0
    Hd = H.double().cpu().numpy()
    ids = g.integers(0, n, (T, 2))
    i, a = _gpu(ids, np.int32), _gpu(g.standard_normal((T, 2)))
    note(f"rows far below zero {prec} T={T}")
    r = X.score(H, F, ids=i, top=top, entropy=True)
    even = slice(0, None, 2)
    assert bool(torch.isneginf(r.lse[even]).all()) and bool(torch.isneginf(r.logp[even]).all())
    assert bool(torch.isneginf(r.top_logp[even]).all()) and bool((r.top_ids[even] == -1).all())
    assert torch.count_nonzero(r.entropy[even]) == 0
    w = ref.score(Hd[1::2], Fd, ids[1::2], 1.0, None, top)
    assert np.array_equal(r.top_ids[1::2].cpu().numpy(), w["top_ids"])
    zb = ref.z_bound(Hd[1::2], Fd, np.zeros(n, bool), 1.0, 1.0, None)
    assert np.all(np.abs(r.lse[1::2].double().cpu().numpy() - w["lse"]) <= ref.lse_bound(zb, w["lse"], n))
    dH, dF = X.score_grad(H, F, r.lse, ids=i, dlogp=a, entropy=r.entropy, dentropy=torch.ones_like(r.lse))
    assert torch.count_nonzero(dH[even]) == 0
    odd = [x[1::2].contiguous() for x in (H, r.lse, i, a, r.entropy)]
    _, want = X.score_grad(odd[0], F, odd[1], ids=odd[2], dlogp=odd[3], entropy=odd[4], dentropy=torch.ones_like(odd[1]))
    size = ref.dz_score(Hd[1::2], Fd, ids[1::2], odd[3].cpu().numpy(), np.ones(len(odd[1])), 1.0, None)[1].T @ np.abs(Hd[1::2])
    # the same terms, added in another order (T additions each) and rounded to the type
    tol = size * (2 * (T + 2) * ref.U + (2 * ref.V if prec == "bf16" else 2 * ref.U))
    assert np.all(np.abs((dF.double() - want.double()).cpu().numpy()) <= tol)
    loss, lse = X.distill(H, F, i, a)
    assert torch.count_nonzero(loss[even]) == 0 and bool(torch.isneginf(lse[even]).all())
    dH, dF = X.distill_grad(H, F, i, a, lse, torch.ones_like(loss))
    assert torch.count_nonzero(dH[even]) == 0 and bool(torch.isfinite(dF).all())


@pytest.mark.parametrize("prec", ["fp32", "bf16"])
def test_soft_masks_at_a_small_temperature(X, prec):
    """A bias of -1e6 at temperature 0.01 on every item leaves nothing; on some, these have p = 0 and a finite log
    probability, and the loss that lists them has the formula's gradient."""
    import torch
    g = np.random.default_rng(5)
    T, n, k, m, tau = 40, 90, 32, 4, 0.01
    F, Fd = _table(g, n, k, prec)
    H, Hd = _table(g, T, k, prec)
    ids = g.integers(0, n, (T, m))
    teacher = (tau * g.standard_normal((T, m))).astype(np.float32)
    dloss, scale = g.standard_normal(T).astype(np.float32), float(np.float32(0.002))
    b = np.full(n, -1e6, np.float32)
    i, t, d = _gpu(ids, np.int32), _gpu(teacher), _gpu(dloss)
    note(f"soft masks {prec}")
    opts = dict(scale=scale, temperature=tau, bias=_gpu(b))
    loss, lse = X.distill(H, F, i, t, **opts)
    assert bool(torch.isneginf(lse).all()) and torch.count_nonzero(loss) == 0
    for x in X.distill_grad(H, F, i, t, lse, d, **opts):
        assert torch.count_nonzero(x) == 0
    far = np.arange(n) % 3 != 0
    b[~far] = 0.0
    opts["bias"] = _gpu(b)
    loss, lse = X.distill(H, F, i, t, **opts)
    want, wlse = ref.distill(Hd, Fd, ids, teacher, scale, b.astype(np.float64), tau)
    zb = ref.z_bound(Hd, Fd, far, scale, tau, np.where(far, 0.0, b))  # of the items that have a probability
    lb = ref.lse_bound(zb, wlse, n)
    assert np.all(np.abs(lse.double().cpu().numpy() - wlse) <= lb)
    assert np.all(np.abs(loss.double().cpu().numpy() - want) <= tau * tau * lb + 4 * ref.U * np.abs(want))
    got = X.distill_grad(H, F, i, t, lse, d, **opts)
    dz, size = ref.dz_distill(Hd, Fd, ids, teacher, dloss, scale, b.astype(np.float64), tau)
    none, s = np.zeros(n, bool), scale / tau
    bounds = ref.grad_bounds(size, Hd, Fd, none, s, zb, wlse, n, T, False)
    # what two bf16 parts of a weight leave out
    parts = (s * size @ np.abs(Fd), s * size.T @ np.abs(Hd))
    v2, v = (ref.V ** 2, ref.V) if prec == "bf16" else (0.0, 2 * ref.U)
    for x, w, bound, part in zip(got, ref.grads(dz, Hd, Fd, none, s), bounds, parts):
        bound = bound + v2 * part
        bound = bound + v * (np.abs(w) + bound)
        assert np.all(np.abs(x.double().cpu().numpy() - w) <= bound)


@pytest.mark.parametrize("prec", ["fp32", "bf16"])
def test_scores_far_above_zero_leave_no_nan(X, prec):
    """A bias of 250 at temperature 1e-6 (a score of 2.5e8) beside rows of a tile that are none."""
    import torch
    g = np.random.default_rng(9)
    F, _ = _table(g, 40, 16, prec)
    H = torch.zeros((3, 16), device="cuda").to(F.dtype)
    b = np.zeros(40, np.float32)
    b[5] = 250.0
    ids = _gpu(np.full((3, 1), 5), np.int32)
    t = torch.zeros((3, 1), device="cuda")
    note(f"far above zero {prec}")
    loss, lse = X.distill(H, F, ids, t, temperature=1e-6, scale=1e-6, bias=_gpu(b))
    dH, dF = X.distill_grad(H, F, ids, t, lse, torch.ones_like(loss), temperature=1e-6, scale=1e-6, bias=_gpu(b))
    for x in (loss, lse, dH, dF):
        assert bool(torch.isfinite(x).all())


# ----------------------------------------------------------------- refusals

@pytest.mark.parametrize("scale", [float("nan"), float("inf"), -float("inf"), 1e39])
def test_lookups_refuse_a_scale_that_is_not_finite(X, scale):
    """Else the zeros of id -1 and of rows that no id names came out as NaN."""
    import torch
    import paper_2608_00977_amd as tsid
    F, out = torch.ones((5, 8), device="cuda"), torch.full((2, 8), 7.0, device="cuda")
    for call in (lambda: X.lookup(F, _gpu([1, -1], np.int32), scale=scale, out=out),
                 lambda: X.lookup_grad(F[:2], _gpu([1, -1], np.int32), 2, scale=scale, out=out)):
        with pytest.raises(tsid.TsidError) as e:
            call()
        assert e.value.status == 1
    torch.cuda.synchronize()
    assert bool((out == 7.0).all())


@pytest.mark.parametrize("prec", ["fp32", "bf16"])
@pytest.mark.parametrize("T", [3, 40])
@pytest.mark.parametrize("scale", [1.0, -1.0, 0.0])
def test_ties_of_zeros_of_both_signs_go_to_the_lowest_id(X, prec, T, scale):
    """A zero row and a bias of 0 and -0: all scores are equal."""
    import torch
    g = np.random.default_rng(2)
    F, _ = _table(g, 3000, 16, prec)
    H = torch.zeros((T, 16), device="cuda").to(F.dtype)
    bias = np.where(g.random(3000) < 0.5, -0.0, 0.0).astype(np.float32)
    note(f"zeros of both signs {prec} T={T} scale={scale}")
    r = X.score(H, F, scale=scale, bias=_gpu(bias), top=20)
    assert r.top_ids.tolist() == [list(range(20))] * T


# ------------------------------------------------- the C entry points' forms

def _c(X):
    """The library, and tables as its structures."""
    from paper_2608_00977_amd import binding as B
    return B, lambda x: B.tsid_rows(x.data_ptr(), x.shape[0], x.stride(0))


def _ws(nbytes):
    import torch
    ws = torch.empty(nbytes + 256, dtype=torch.uint8, device="cuda")
    return ws, (ws.data_ptr() + 255) & ~255


@pytest.mark.parametrize("prec", ["fp32", "bf16"])
@pytest.mark.parametrize("T", [9, 70])
def test_scores_at_a_temperature_and_any_output_alone(X, prec, T):
    """tsid_score divides by the head's temperature as a scale and a bias that are divided by it do (a power of two,
    so the same bits), and gives the same where only some outputs are wanted."""
    import torch
    B, rows = _c(X)
    g = np.random.default_rng(T)
    n, k, top = 333, 32, 6
    F, _ = _table(g, n, k, prec)
    H, _ = _table(g, T, k, prec)
    bias, ids = _gpu(g.standard_normal(n)), _gpu(g.integers(-1, n, (T, 3)), np.int32)
    want = X.score(H, F, ids=ids, scale=0.25, bias=bias / 4, top=top, entropy=True)
    head = B.tsid_head(rows(H), rows(F), bias.data_ptr(), k, B.BF16 if prec == "bf16" else B.FP32, 1.0, 4.0)
    outs = [torch.empty_like(x) for x in want]  # lse, logp, entropy, top_ids, top_logp
    note(f"temperature {prec} T={T}")
    for wanted in ((0, 1, 2, 3, 4), (0,), (1,), (2,), (3, 4), ()):
        for o in outs:
            o.fill_(77)
        t = top if 3 in wanted else 0
        need = B.tsid_score_workspace(T, n, k, head.prec, t)
        ws, at = _ws(need)
        p = [o.data_ptr() if q in wanted else None for q, o in enumerate(outs)]
        st = B.tsid_score(X.ctx, head, ids.data_ptr() if 1 in wanted else None, 3 if 1 in wanted else 0, t, p[0], p[1], p[2],
                          p[3], p[4], at, need, torch.cuda.current_stream().cuda_stream)
        assert st == 0
        torch.cuda.synchronize()
        for q, (o, w) in enumerate(zip(outs, want)):
            assert torch.equal(o, w) if q in wanted else bool((o == 77).all()), (wanted, q)
    # the gradient at a temperature
    a = _gpu(g.standard_normal((T, 3)))
    w = X.score_grad(H, F, want.lse, ids=ids, dlogp=a, scale=0.25, bias=bias / 4)
    need = B.tsid_head_grad_workspace(T, n, k, head.prec, 3)
    ws, at = _ws(need)
    full = [torch.full((x.shape[0] + 2, k + 16), 5.0, device="cuda").to(x.dtype) for x in (H, F)]
    views = [f[1:-1, 8:8 + k] for f in full]
    st = B.tsid_score_grad(X.ctx, head, ids.data_ptr(), 3, want.lse.data_ptr(), a.data_ptr(), None, None, rows(views[0]),
                           rows(views[1]), at, need, torch.cuda.current_stream().cuda_stream)
    assert st == 0
    torch.cuda.synchronize()
    for f, v, x in zip(full, views, w):
        assert torch.equal(v, x)
        v.fill_(5.0)
        assert bool((f == 5.0).all())  # what lies beside the strided rows is as it was


def test_an_error_is_reported_once_whichever_stream_met_it(X):
    import torch
    import paper_2608_00977_amd as tsid
    F = torch.ones((4, 8), device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        X.lookup(F, _gpu([9], np.int32))
    side.synchronize()
    with pytest.raises(tsid.TsidError) as e:
        X.rows_check()
    assert e.value.status == 2
    X.rows_check()
    with torch.cuda.stream(side):
        X.rows_check()


@pytest.mark.parametrize("prec", ["fp32", "bf16"])
@pytest.mark.parametrize("T", [3, 40])
@pytest.mark.parametrize("n", [3000, 70_000])  # blocks, and groups of blocks
def test_items_far_below_others_are_better_than_excluded_ones(X, prec, T, n):
    """Five ordinary items, the first half excluded, the rest biased to -1e9 and less at temperature 0.001."""
    import torch
    B, rows = _c(X)
    k, top = 16, 12
    H = torch.zeros((T, k), device="cuda").to(torch.float32 if prec == "fp32" else torch.bfloat16)
    F, _ = _table(np.random.default_rng(n), n, k, prec)
    b = -1e6 - 16.0 * (np.arange(n) % 1000)  # ties go to the lowest id
    b[:n // 2] = -np.inf
    b[n // 2 + 100:n // 2 + 600:100] = [-5.0, -4.0, -3.0, -2.0, -1.0]
    bias = _gpu(b)
    want = np.argsort(-b.astype(np.float32), kind="stable")[:top]
    head = B.tsid_head(rows(H), rows(F), bias.data_ptr(), k, B.BF16 if prec == "bf16" else B.FP32, 1.0, 1e-3)
    need = B.tsid_score_workspace(T, n, k, head.prec, top)
    ws, at = _ws(need)
    ids, logp = torch.empty((T, top), dtype=torch.int32, device="cuda"), torch.empty((T, top), device="cuda")
    note(f"far below others {prec} T={T} n={n}")
    assert B.tsid_score(X.ctx, head, None, 0, top, None, None, None, ids.data_ptr(), logp.data_ptr(), at, need,
                        torch.cuda.current_stream().cuda_stream) == 0
    assert ids.tolist() == [want.tolist()] * T
    z = b[want] * 1000.0
    assert np.allclose(logp.double().cpu().numpy(), z - z[0], rtol=4 * ref.U, atol=1e3 * 8 * ref.U)
