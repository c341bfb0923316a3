"""The draw of the last token next to a border: whatever the rounding of the sums, the token has a share of what is left."""
import pytest
import torch

import tree_helpers as T
from test_gpu_verify_tree import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("R", [1, 40])                        # runs of the vocabulary: 128, 64
@pytest.mark.parametrize("small", [2.0 ** -54, 2.0 ** -53, 2.0 ** -55, 3 * 2.0 ** -55])
def test_the_token_drawn_at_a_border_has_a_share(R, small):
    # 1/2, two shares of half a rounding step of 1/2, nothing for long, 1/2: the running sums of the parts between, added up in
    # different orders, differ by a step, and the number 1/2 lies between them
    V = 128 * 128
    run_of = 128 if R == 1 else 256
    p = torch.zeros(R, V, device="cuda")
    p[:, 3] = 0.5
    p[:, 5 * run_of + 1] = small
    p[:, 9 * run_of + 2] = small
    p[:, 60 * run_of] = 0.5
    u = torch.zeros(R, device="cuda")
    for at in (0.5, 0.5 - 2.0 ** -25, 0.0, 1 - 2.0 ** -24):
        acc, out, path, st = run(p, None, T.i32([0] * R), [-1] * R, list(range(R + 1)), u, torch.full((R,), at, device="cuda"))
        assert st == 0 and acc == [0] * R and path == [-1] * R
        assert all(0 <= t < V for t in out) and bool((p[torch.arange(R), out] > 0).all())
        if at == 0.0 or at < 0.5:
            assert out == [3] * R
        if at > 0.5:
            assert out == [60 * run_of] * R
