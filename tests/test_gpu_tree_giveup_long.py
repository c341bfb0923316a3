"""dspark_tree_attention when waits run out in the middle of long sums, which are put by from time to time: the call ends, and the next one
gives the ordinary call's bits."""
import pytest
import torch

from paper_2607_05147_b200 import binding as B
import tree_helpers as T

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("group", [4, 20, 60, 100])           # rows with a head; a head an SM
def test_waits_that_run_out_in_long_sums(kind, group):
    page, heads, d, times = 1 << 16, 148, 16, 3
    cache = T.Cache([page], page, heads, d, kind, spare=0)
    g = T.gen(group)
    for c in (cache.k, cache.v):
        c.copy_(torch.randint(-100, 100, c.shape, generator=g, device="cuda").to(c.dtype))
    for s in (cache.ks, cache.vs):
        if s is not None:
            s.fill_(0.01)
    cache.handle = B.KvCache(cache.k, cache.v, torch.zeros(1, times, dtype=torch.int32, device="cuda"), cache.ks, cache.vs)
    q = torch.randn(1, heads * group, d, generator=g, device="cuda").bfloat16()
    first, off = T.i32([page * times - 1]), T.i32([0, 1])
    call = lambda: T.run_attention(cache, q, first, off, None, 0.002)
    want, lse, st = call()
    assert st == 0
    try:
        for polls in (1, 2, 3, 9, 65):
            B.dspark_set_wait_poll_limit(polls)
            got, got_lse, st = call()
            assert st == B.DEV_TIMEOUT or (st == 0 and torch.equal(got, want) and torch.equal(got_lse, lse))
    finally:
        B.dspark_set_wait_poll_limit(0)
    again = call()
    assert again[2] == 0 and torch.equal(again[0], want) and torch.equal(again[1], lse)
