"""dspark_tree_attention when its waits run out (dspark_set_wait_poll_limit): the call ends, says so in dev_status, and leaves the
device as it was: the next call gives the ordinary call's bits."""
import pytest
import torch

from paper_2607_05147_b200 import binding as B
import tree_helpers as T

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("nodes,group", [(1, 8), (4, 8), (8, 8), (16, 8), (32, 8)])      # 8, 32, 64, 128 and 256 rows with a head
def test_waits_that_run_out(kind, nodes, group):
    R, heads, d, first = 20, 2, 128, 2000
    cache = T.Cache([first + nodes] * R, 64, heads, d, kind)
    g = T.gen(nodes)
    for r in range(R):
        cache.put(r, range(first + nodes), *torch.randn(2, first + nodes, heads, d, generator=g, device="cuda"))
    q = torch.randn(R * nodes, heads * group, d, generator=g, device="cuda").bfloat16()
    call = lambda: T.run_attention(cache, q, T.i32([first] * R), T.offsets([nodes] * R), None, d ** -0.5)
    want, lse, st = call()
    assert st == 0
    B.dspark_set_wait_poll_limit(1)                           # no poll at all: every wait runs out
    try:
        assert call()[2] == B.DEV_TIMEOUT
    finally:
        B.dspark_set_wait_poll_limit(0)
    again = call()
    assert again[2] == 0 and torch.equal(again[0], want) and torch.equal(again[1], lse)
