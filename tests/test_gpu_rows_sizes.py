"""The row operators on so many rows that a launch with a wave or a workgroup per row has more than 2^32 threads."""
import pytest

from gpu_util import note

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def X():
    import paper_2608_00977_amd as tsid
    t = tsid.Tsid(0)
    yield t
    t.close()


def _rows(T):
    """Rows of H whose first factor is 0, 1 or 2, by turns."""
    import torch
    H = torch.zeros((T, 8), dtype=torch.bfloat16, device="cuda")
    turn = torch.arange(T, device="cuda") % 3
    H[:, 0] = turn
    return H, turn


def _table():
    import torch
    F = torch.zeros((3, 8), device="cuda")
    F[0, 0], F[2, 0] = 1.0, -1.0
    return F.bfloat16()


def test_best_items_of_more_than_2_24_rows(X):
    import torch
    T = 2 ** 24 + 5
    H, turn = _rows(T)
    note("best items of 2^24 rows")
    r = X.score(H, _table(), top=2)
    z = torch.tensor([[0.0, 0, 0], [1, 0, -1], [2, 0, -2]], dtype=torch.float64, device="cuda")
    lse = torch.logsumexp(z, 1)
    assert bool((r.top_ids == torch.tensor([0, 1], dtype=torch.int32, device="cuda")).all())
    assert bool((r.lse.double() - lse[turn]).abs().max() < 1e-6)
    assert bool((r.top_logp.double() - (z[:, :2] - lse[:, None])[turn]).abs().max() < 1e-6)


def test_gradients_of_more_than_2_26_rows(X):
    import torch
    T = 2 ** 26 + 5
    H, turn = _rows(T)
    ids = torch.zeros((T, 1), dtype=torch.int32, device="cuda")
    note("gradients of 2^26 rows")
    r = X.score(H, _table(), ids=ids)
    z = torch.tensor([[0.0, 0, 0], [1, 0, -1], [2, 0, -2]], dtype=torch.float64, device="cuda")
    logp = torch.log_softmax(z, 1)
    assert bool((r.logp[:, 0].double() - logp[turn, 0]).abs().max() < 1e-6)
    a = torch.ones((T, 1), device="cuda")
    dH, _ = X.score_grad(H, _table(), r.lse, ids=ids, dlogp=a, want_F=False)
    want = 1.0 - (logp.exp()[:, 0] - logp.exp()[:, 2])  # f_0 - sum_i p_i f_i
    assert bool((dH[:, 0].double() - want[turn]).abs().max() < 2.0 ** -8)
    assert torch.count_nonzero(dH[:, 1:]) == 0


def test_lookup_gradient_into_more_than_2_26_rows(X):
    import torch
    n = 2 ** 26 + 5
    G = torch.arange(1, 4, device="cuda").bfloat16()[:, None].expand(3, 8).contiguous()
    note("lookup gradient into 2^26 rows")
    d = X.lookup_grad(G[:2], torch.tensor([n - 1, 7], dtype=torch.int32, device="cuda"), n, out=torch.ones((n, 8), dtype=G.dtype, device="cuda"))
    assert torch.equal(d[[7, n - 1]], G[[1, 0]]) and torch.count_nonzero(d) == 16


def test_lookup_gradient_of_a_table_of_2_32_pieces(X):
    """2^28 + 3 rows of 16 pieces of 16 bytes (69 GB), by the sort."""
    import torch
    n, k, count = 2 ** 28 + 3, 128, 3000
    if torch.cuda.mem_get_info()[0] < 90 << 30:
        pytest.skip("needs 90 GiB of free device memory")
    ids = torch.arange(count, dtype=torch.int64, device="cuda") * (n // count)
    ids[-3:] = torch.tensor([n - 1, n - 1, n - 2], device="cuda")
    G = torch.ones((count, k), dtype=torch.bfloat16, device="cuda")
    out = torch.full((n, k), 7.0, dtype=torch.bfloat16, device="cuda")
    note("lookup gradient of a table of 69 GB")
    X.lookup_grad(G, ids.to(torch.int32), n, out=out)
    assert bool((out[ids[:-3]] == 1).all()) and bool((out[n - 1] == 2).all()) and bool((out[n - 2] == 1).all())
    step = 2 ** 24
    assert sum(int(torch.count_nonzero(out[i:i + step])) for i in range(0, n, step)) == (count - 1) * k
    del out
    torch.cuda.empty_cache()
