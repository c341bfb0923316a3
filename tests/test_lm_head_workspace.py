"""Workspace of the vocabulary loss over the number of rows (host arithmetic, no GPU): a caller that allocates once, for
its largest batch, may use that workspace for every smaller batch of the same vocabulary and width."""
import pytest

from paper_2607_05147_b200 import binding as B


@pytest.mark.parametrize("V,d", [(129280, 1024), (129280, 2048), (129280, 64), (40000, 300), (10007, 500), (5000, 64), (1, 1), (300, 65536), (1 << 24, 8)])
def test_fewer_rows_never_need_more(V, d):
    f = B.dspark_lm_head_loss_workspace_bytes
    # every number of rows at which the layout changes, up to 9 000, then a stride
    rows = sorted({1, 2, 127, 128, 129} | {n + o for n in range(256, 9217, 256) for o in (0, 1)} | set(range(9300, 1 << 18, 9973)) | {1 << 20})
    sizes = [f(n, V, d) for n in rows]
    assert min(sizes) > 0
    for a, b, n in zip(sizes, sizes[1:], rows[1:]):
        assert a <= b, n


def test_the_largest_batch_s_workspace_is_accepted_for_smaller_ones():
    # a workspace of exactly that many bytes passes the check of size: the call is refused for its alignment, which comes after
    P = 0x10000
    for V, d, N, fewer in ((129280, 1024, 4096, 2817), (129280, 2048, 2048, 1281)):
        n = B.dspark_lm_head_loss_workspace_bytes(N, V, d)
        for rows in (N, fewer, 1):
            args = (P, d, P, d, P, rows, V, d, P, P, P, P + 128, n, None)
            assert B.lib().dspark_lm_head_loss(*args) == 3
            back = (P, d, P, d, P, P, P, rows, V, d, P, d, P, d, P, P + 128, n, None)
            assert B.lib().dspark_lm_head_loss_backward(*back) == 3
