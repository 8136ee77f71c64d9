"""The row operators without a GPU: the 64-bit definitions that the GPU tests compare with, against automatic
differentiation and differences; workspace sizes; refusals that need no device."""
import numpy as np
import pytest
import torch

import rows_ref as ref


def _problem(bias):
    g = np.random.default_rng(4)
    T, n, k, m = 6, 40, 8, 5
    H, F = g.standard_normal((T, k)), g.standard_normal((n, k))
    b = None
    if bias:
        b = g.standard_normal(n)
        b[[3, 11, 12]] = -np.inf, np.finfo(np.float32).min, -1e21
    ids = g.integers(-1, n, (T, m))
    ids[:, 1] = ids[:, 0]
    ids[2] = -1
    if bias:
        ids[0, 0] = 11
    return g, H, F, b, ids


def _scores(H, F, b, scale, tau):
    z = scale * H @ F.T
    if b is not None:
        off = torch.from_numpy(b < ref.EXCLUDED)
        z = (z + torch.from_numpy(np.where(b < ref.EXCLUDED, 0.0, b))).masked_fill(off, -torch.inf)
    return torch.log_softmax(z / tau, 1)


@pytest.mark.parametrize("bias", [False, True])
def test_score_gradient_is_the_derivative(bias):
    g, H, F, b, ids = _problem(bias)
    scale, out = -0.7, np.zeros(F.shape[0], bool) if b is None else b < ref.EXCLUDED
    dlogp, dent = g.standard_normal(ids.shape), g.standard_normal(H.shape[0])
    h, f = (torch.from_numpy(x).requires_grad_() for x in (H, F))
    lp = _scores(h, f, b, scale, 1.0)
    have = torch.from_numpy(ref.listed(ids, out, F.shape[0]))
    got = torch.where(have, lp.gather(1, torch.from_numpy(np.maximum(ids, 0))), 0.0)
    fin = torch.isfinite(lp)
    ent = -torch.where(fin, lp.exp() * torch.where(fin, lp, 0.0), 0.0).sum(1)
    w = ref.score(H, F, ids, scale, b, 4)
    assert np.allclose(w["entropy"], ent.detach().numpy(), rtol=1e-12)
    assert np.allclose(np.where(have, w["logp"], 0.0), got.detach().numpy(), rtol=1e-12)
    (torch.where(have, got * torch.from_numpy(dlogp), 0.0).sum() + (ent * torch.from_numpy(dent)).sum()).backward()
    dz, size = ref.dz_score(H, F, ids, dlogp, dent, scale, b)
    dH, dF = ref.grads(dz, H, F, out, scale)
    assert np.allclose(dH, h.grad.numpy(), atol=1e-12) and np.allclose(dF, f.grad.numpy(), atol=1e-12)
    assert np.all(np.abs(dz) <= size + 1e-15)


@pytest.mark.parametrize("bias", [False, True])
def test_distillation_gradient_is_the_derivative(bias):
    g, H, F, b, ids = _problem(bias)
    scale, tau, out = 0.6, 2.0, np.zeros(F.shape[0], bool) if b is None else b < ref.EXCLUDED
    teacher, dloss = g.standard_normal(ids.shape), g.standard_normal(H.shape[0])
    h, f = (torch.from_numpy(x).requires_grad_() for x in (H, F))
    lp = _scores(h, f, b, scale, tau).gather(1, torch.from_numpy(np.maximum(ids, 0)))
    have = torch.from_numpy(ref.listed(ids, out, F.shape[0]))
    w = torch.softmax(torch.from_numpy(teacher / tau).masked_fill(~have, -torch.inf), 1).nan_to_num(0.0)
    loss = tau * tau * torch.where(have, w * (w.clamp(min=1e-300).log() - torch.where(have, lp, 0.0)), 0.0).sum(1)
    want, _ = ref.distill(H, F, ids, teacher, scale, b, tau)
    assert np.allclose(want, loss.detach().numpy(), rtol=1e-12) and want[2] == 0.0
    (loss * torch.from_numpy(dloss)).sum().backward()
    dz, size = ref.dz_distill(H, F, ids, teacher, dloss, scale, b, tau)
    dH, dF = ref.grads(dz, H, F, out, scale / tau)
    assert np.allclose(dH, h.grad.numpy(), atol=1e-12) and np.allclose(dF, f.grad.numpy(), atol=1e-12)
    assert np.all(np.abs(dz) <= size + 1e-15)
    e = 1e-6  # and against differences
    D = g.standard_normal(H.shape)
    q = sum(s * (dloss * ref.distill(H + s * e * D, F, ids, teacher, scale, b, tau)[0]).sum() for s in (1, -1)) / (2 * e)
    assert q == pytest.approx((dH * D).sum(), rel=1e-6)


def test_workspace_sizes_need_no_device():
    from paper_2608_00977_amd import binding as B
    for T, n in ((0, 0), (1, 1), (33, 100), (5000, 70_000)):
        for k in (8, 128):
            for prec in (0, 1):
                assert B.tsid_score_workspace(T, n, k, prec, 0) >= 256
                assert B.tsid_score_workspace(T, n, k, prec, 10) >= B.tsid_score_workspace(T, n, k, prec, 0)
                assert B.tsid_head_grad_workspace(T, n, k, prec, 3) >= 256
        assert B.tsid_lookup_grad_workspace(T, n, 64) > 0  # few entries are summed without a sort
    assert B.tsid_lookup_grad_workspace(5000, 70_000, 64) >= 24 * 5000
    # the blocks' maxima of many rows over a long table are taken a run of rows at a time
    assert B.tsid_score_workspace(100_000, 2_000_000, 64, 1, 10) < 3 << 30
    for bad in ((-1, 5, 8, 0, 0), (5, -1, 8, 0, 0), (5, 5, 9, 0, 0), (5, 5, 8, 2, 0), (5, 5, 8, 0, 65),
                (5, 5, 8, 0, -1), (2 ** 31, 5, 8, 0, 0)):
        assert B.tsid_score_workspace(*bad) == 0
    assert B.tsid_head_grad_workspace(2 ** 30, 5, 8, 0, 2) == 0
    assert B.tsid_lookup_grad_workspace(5, 5, 7) == 0


def test_null_context_and_tensors_elsewhere_are_refused():
    import ctypes as C
    import paper_2608_00977_amd as tsid
    from paper_2608_00977_amd import binding as B
    L = B.lib()
    assert L.tsid_rows_check(None, None) == 1
    assert L.tsid_lookup(None, 0, 8, None, None, C.c_float(1), None, None) == 1
    assert L.tsid_score(None, None, None, 0, 0, None, None, None, None, None, None, 0, None) == 1
    assert L.tsid_distill(None, None, None, 1, None, None, None, None, 0, None) == 1
    x = B.Tsid.__new__(B.Tsid)  # no context: what is refused before any call needs none
    x.device, x.ctx, x._keep = 0, None, []
    H, F = torch.zeros((3, 8)), torch.zeros((5, 8))
    for call in (lambda: x.lookup(F, torch.zeros(2, dtype=torch.int32)), lambda: x.score(H, F),
                 lambda: x.lookup_grad(H, torch.zeros(3, dtype=torch.int32), 5),
                 lambda: x.distill(H, F, torch.zeros((3, 1), dtype=torch.int32), torch.zeros((3, 1)))):
        with pytest.raises(tsid.TsidError) as e:
            call()
        assert e.value.status == 1
