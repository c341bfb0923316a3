"""Rows of requests whose own offsets are right, in a batch where another's are not: written and read all the same, whichever CTA
they begin in."""
import pytest
import torch

from paper_2607_05147_b200 import binding as B
import tree_helpers as T
from test_gpu_kv_cache import read, rows_of, write

pytestmark = pytest.mark.gpu


def owners(off, n):
    """For each row the requests with sound offsets that have it."""
    return [[r for r in range(len(off) - 1) if 0 <= off[r] <= i < off[r + 1] <= n] for i in range(n)]


@pytest.mark.parametrize("kind", ["bf16", "int8"])
@pytest.mark.parametrize("heads,d", [(8, 128), (1, 64), (2, 256), (5, 80)])        # 4, 64, 8 and 6.4 rows a CTA
@pytest.mark.parametrize("off,n", [([0, 5, 3, 4], 5), ([0, 5, 3, 4], 40), ([0, 9, 2, 2, 1, 3], 9), ([0, 4, 100, 6, 20], 20), ([0, 6, -3, 6, 12], 12),
                                   ([0, 30, 0, 0, 1, 0, 2], 30)])
@pytest.mark.parametrize("idle", [0, 300, 1100])              # requests without rows behind: the three ways of looking a request up
def test_sound_requests_beside_falling_offsets(kind, heads, d, off, n, idle):
    off = off + [off[-1]] * idle
    R = len(off) - 1
    first = [3 + 40 * (r % 7) for r in range(R)]
    cache, want = (T.Cache([f + (40 if r < 8 else 0) for r, f in enumerate(first)], 16, heads, d, kind, seed=1) for _ in range(2))
    k, v = rows_of(n, heads, d, 5)
    has = owners(off, n)
    alone = [i for i in range(n) if len(has[i]) == 1]
    assert write(cache, k, v, T.i32(first), T.i32(off)) & B.DEV_BAD_OFFSETS
    a, b, st = read(cache, T.i32(first), T.i32(off), n, torch.float32)
    assert st & B.DEV_BAD_OFFSETS
    for i in alone:
        r = has[i][0]
        at = first[r] + i - off[r]
        want.put(r, [at], k[i: i + 1], v[i: i + 1])
        x, y = want.values(r, [at])
        got_x, got_y = cache.values(r, [at])
        assert torch.equal(x, got_x) and torch.equal(y, got_y)
        assert torch.equal(a[i], x[0].float()) and torch.equal(b[i], y[0].float())
    for i in range(n):
        if not has[i]:
            assert (a[i] == 3).all() and (b[i] == 3).all()
