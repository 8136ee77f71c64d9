"""The row operators where sizes change their course: tables whose blocks are found through groups of blocks (with
and without a bias), more rows than one run takes, and tables beyond 32-bit offsets."""
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


def _check_rows(H, F, bias, scale, r, rows, top):
    """Rows of a result against 64 bits on the GPU."""
    import torch
    h, f = H[rows].double(), F.double()
    z = scale * (h @ f.t())
    size = abs(scale) * (h.abs() @ f.abs().t())
    if bias is not None:
        out = bias < ref.EXCLUDED
        z = (z + torch.where(out, torch.zeros_like(bias), bias).double()).masked_fill(out, -torch.inf)
        size = (size + torch.where(out, torch.zeros_like(bias), bias).double().abs()).masked_fill(out, 0.0)
    lse = torch.logsumexp(z, 1)
    lb = (2 * H.shape[1] + 16) * ref.U * size.max(1).values + (F.shape[0] / 16 + 72) * ref.U + 2 * ref.U * lse.abs()
    order = torch.sort(z, dim=1, descending=True, stable=True)
    assert torch.equal(r.top_ids[rows].long(), order.indices[:, :top])
    assert bool(((r.lse[rows].double() - lse).abs() <= lb).all())
    want = order.values[:, :top] - lse[:, None]
    assert bool(((r.top_logp[rows].double() - want).abs() <= lb[:, None] + 2 * ref.U * want.abs()).all())


@pytest.mark.parametrize("prec", ["fp32", "bf16"])
@pytest.mark.parametrize("T", [3, 45])
@pytest.mark.parametrize("n", [65_536, 65_537, 131_105])
def test_groups_of_blocks_with_a_bias(X, prec, T, n):
    import torch
    dt = torch.float32 if prec == "fp32" else torch.bfloat16
    g = torch.Generator(device="cuda").manual_seed(n + T)
    F = torch.randn((n, 32), generator=g, device="cuda").to(dt)
    H = torch.randn((T, 32), generator=g, device="cuda").to(dt)
    bias = torch.randn(n, generator=g, device="cuda")
    bias[torch.rand(n, generator=g, device="cuda") < 0.3] = -np.inf
    bias[-1] = 30.0  # the best item is the last
    note(f"groups of blocks {prec} T={T} n={n}")
    r = X.score(H, F, scale=0.4, bias=bias, top=33, entropy=True)
    assert r.top_ids[:, 0].tolist() == [n - 1] * T
    _check_rows(H, F, bias, float(np.float32(0.4)), r, torch.arange(T, device="cuda"), 33)


def test_more_rows_than_one_run_takes(X):
    """9,000 rows over 1 M items: the blocks' maxima of 8,448 rows fill the workspace's share."""
    import torch
    n, T = 1_000_000, 9_000
    g = torch.Generator(device="cuda").manual_seed(3)
    F = torch.randn((n, 8), generator=g, device="cuda").to(torch.bfloat16)
    H = torch.randn((T, 8), generator=g, device="cuda").to(torch.bfloat16)
    ids = torch.randint(0, n, (T, 2), generator=g, device="cuda", dtype=torch.int32)
    note("more rows than one run takes")
    r = X.score(H, F, ids=ids, top=5, entropy=True)
    rows = torch.cat([torch.arange(a, b, device="cuda") for a, b in ((0, 9), (8440, 8456), (T - 9, T))])
    _check_rows(H, F, None, 1.0, r, rows, 5)
    z = (H.double()[:, None, :] * F[ids.long()].double()).sum(2) - r.lse.double()[:, None]
    assert bool(((r.logp.double() - z).abs() <= 1e-6 * (1 + z.abs())).all())  # both from the same log sum, rounded once


def test_tables_beyond_32_bit_offsets(X):
    """20 M rows of 128 bf16: 2.6e9 elements, 5.1 GB."""
    import torch
    n, k = 20_000_000, 128
    F = torch.zeros((n, k), dtype=torch.bfloat16, device="cuda")
    marks = torch.tensor([0, 16_777_216, 16_777_217, n - 1], device="cuda")
    F[marks] = torch.arange(1, 5, dtype=torch.bfloat16, device="cuda")[:, None]
    note("a table beyond 32-bit offsets")
    out = X.lookup(F, marks.to(torch.int32), scale=2.0)
    assert torch.equal(out, 2 * F[marks])
    H = torch.full((1, k), 1 / k, dtype=torch.bfloat16, device="cuda")
    r = X.score(H, F, ids=marks.to(torch.int32)[None], top=6, entropy=True)  # scores 1, 2, 3, 4 and zeros
    assert r.top_ids.tolist() == [[n - 1, 16_777_217, 16_777_216, 0, 1, 2]]
    lse = np.log(n - 4 + np.exp([1.0, 2.0, 3.0, 4.0]).sum())
    # 2 n / 512 additions a lane at most, of ones for the most part
    assert abs(r.lse.item() - lse) <= (n / 512 + 72) * ref.U + 2 * ref.U * lse
    assert np.allclose(r.logp.cpu().numpy(), [np.arange(1, 5) - lse], atol=(n / 512 + 72) * ref.U + 4 * ref.U * lse)
    del r
    dF = X.lookup_grad(F[marks], marks.to(torch.int32), n, out=F)
    assert torch.equal(dF[marks][:, 0].float().cpu(), torch.tensor([1.0, 2.0, 3.0, 4.0]))
    assert torch.count_nonzero(dF).item() == 4 * k
    X.rows_check()
