"""What the row operators choose by sizes, as the workspaces that they ask for show it (no GPU)."""
from paper_2608_00977_amd import binding as B


def test_a_lookup_gradient_is_summed_without_a_sort_into_small_tables_only():
    for count, n in ((1, 1), (500, 8192), (2048, 65_536)):
        assert B.tsid_lookup_grad_workspace(count, n, 32) == 256
    for count, n in ((1, 1_000_000), (128, 100_000), (2049, 100)):  # keys and values twice, and a pointer per row
        assert B.tsid_lookup_grad_workspace(count, n, 32) >= 24 * count + 4 * n


def test_listed_items_are_sorted_where_few_workgroups_would_look_through_them():
    """A pass over 2,000 items has 16 workgroups a slice: they do not take 512 x 1,000 ids among them."""
    T, n, m = 512, 2000, 1000
    assert B.tsid_head_grad_workspace(T, n, 32, 0, m) >= (4 + 24) * T * m  # weights; keys and values twice
    T, n, m = 4096, 8192, 20
    assert B.tsid_head_grad_workspace(T, n, 64, 0, m) - B.tsid_head_grad_workspace(T, n, 64, 0, 0) < 24 * T * m
