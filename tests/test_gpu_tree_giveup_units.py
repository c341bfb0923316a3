"""dspark_tree_attention when some of its waits run out, at any of several units of an SM: warps that look for the others' giving up
between two units leave whole.  A call either gives the ordinary call's bits or says that its waits ran out, and ends."""
import pytest
import torch

from paper_2607_05147_b200 import binding as B
import tree_helpers as T

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("nodes,group", [(1, 8), (4, 8), (8, 8), (24, 8)])      # 8, 32, 64 and 192 rows with a head
def test_waits_that_run_out_between_units(kind, nodes, group):
    R, heads, d, first = 500, 2, 64, 100                      # some seven units an SM
    cache = T.Cache([first + nodes] * R, 64, heads, d, kind)
    g = T.gen(nodes)
    for c in (cache.k, cache.v):
        if kind == "bf16":
            c.normal_(generator=g)
        else:
            c.copy_(torch.randint(-100, 100, c.shape, generator=g, device="cuda").to(c.dtype))
    for s in (cache.ks, cache.vs):
        if s is not None:
            s.fill_(0.01)
    q = torch.randn(R * nodes, heads * group, d, generator=g, device="cuda").bfloat16()
    first, off = T.i32([first] * R), T.offsets([nodes] * R)
    call = lambda: T.run_attention(cache, q, first, off, None, d ** -0.5)
    want, lse, st = call()
    assert st == 0
    try:
        for polls in (2, 3, 5, 9, 33, 257):                   # one poll less each: 1, 2, 4, ..
            B.dspark_set_wait_poll_limit(polls)
            got, got_lse, st = call()
            assert st == B.DEV_TIMEOUT or (st == 0 and torch.equal(got, want) and torch.equal(got_lse, lse))
    finally:
        B.dspark_set_wait_poll_limit(0)
    again = call()
    assert again[2] == 0 and torch.equal(again[0], want) and torch.equal(again[1], lse)
