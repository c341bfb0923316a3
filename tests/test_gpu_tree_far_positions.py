"""Requests that end at the last positions there are (2^31 - 2), over a cache whose pages most entries of the block table share."""
import math

import pytest
import torch

from paper_2607_05147_b200 import binding as B
import tree_helpers as T

pytestmark = pytest.mark.gpu

PAGE, PAGES, D = 1 << 20, 2048, 16
END = 2 ** 31 - 1


def far_cache(kind, heads=1):
    """Entries 0 .. 2046 of the table are page 1, the last one page 0; the prefix' keys point away from the queries."""
    cache = T.Cache([PAGE], PAGE, heads, D, kind, spare=1)
    last = int(cache.table[0, 0])
    cache.table = torch.full((1, PAGES), 1 - last, dtype=torch.int32, device="cuda")
    cache.table[0, PAGES - 1] = last
    cache.handle = B.KvCache(cache.k, cache.v, cache.table, cache.ks, cache.vs)
    cache.k[..., 0] = -128 if kind == "bf16" else torch.tensor(-127).to(cache.k.dtype)
    if kind == "bf16":
        cache.v.fill_(1.0)
    else:
        cache.v.fill_(1)
        cache.ks.fill_(1.0)
        cache.vs.fill_(1.0)
    return cache


@pytest.mark.parametrize("kind", ["bf16", "int8"])
@pytest.mark.parametrize("nodes,group,tree", [(1, 4, False), (7, 4, True), (100, 1, False), (70, 3, True)])
def test_attention_at_the_last_positions(kind, nodes, group, tree):
    # e^-250 and less for the positions far before; what counts is the last 300
    cache = far_cache(kind)
    first, near = END - nodes, 300
    g = T.gen(nodes)
    x = torch.randn(2, near + nodes, 1, D, generator=g, device="cuda")
    x[0, ..., 0] = 0
    cache.put(0, range(first - near, END), x[0], x[1])
    q = torch.randn(nodes, group, D, generator=g, device="cuda").bfloat16()
    q[..., 0] = 8.0
    parents = T.random_parents([nodes], 1) if tree else None
    scale = 0.25
    got, lse, st = T.run_attention(cache, q, T.i32([first]), T.i32([0, nodes]), None if parents is None else T.i32(parents), scale)
    assert st == 0

    class Near:                                               # the same cache without the positions that do not count
        kind, heads, vs = cache.kind, cache.heads, cache.vs

        @staticmethod
        def slots(r, pos):
            return cache.slots(0, torch.as_tensor(pos, device="cuda").long() + (first - near))

        @staticmethod
        def values(r, pos, layer=0):
            return cache.values(0, torch.as_tensor(pos, device="cuda").long() + (first - near), layer)
    want, bound, want_lse, lse_bound = T.attention(Near, q, [near], [0, nodes], parents, scale)
    assert bool(((got.double() - want).abs() <= bound).all()) and bool(((lse.double() - want_lse).abs() <= lse_bound).all())


@pytest.mark.parametrize("kind", ["bf16", "int8"])
def test_rows_at_the_last_positions(kind):
    cache = far_cache(kind, heads=2)
    n = 9
    k, v = (torch.randn(n, 2, D, generator=T.gen(s), device="cuda").bfloat16() for s in (1, 2))
    first, off, st = T.i32([END - n]), T.i32([0, n]), T.status()
    a, b = torch.zeros(2, n, 2, D, device="cuda")
    B.dspark_kv_write(cache.handle, k, v, first, off, dev_status=st)
    B.dspark_kv_read(cache.handle, first, off, out_k=a, out_v=b, dev_status=st)
    out = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.dspark_kv_commit(cache.handle, first, off, T.i32([2]), T.i32([3, n - 1] + [0] * (n - 2)), out_first=out, dev_status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0 and out.tolist() == [END - n + 3]
    x, y = cache.values(0, range(END - n, END))
    whole = 127 if kind == "int8" else None
    for got, src, now in ((a, k, x), (b, v, y)):
        if whole:
            z, scale = T.quantised(src, kind)
            src = (z.float() * scale[..., None]).float()
        assert torch.equal(got, src.float())
        assert torch.equal(now[1:3].float(), src[[3, n - 1]].float()) and torch.equal(now[3:].float(), src[3:].float())
    # one position further is past the end
    before = cache.snapshot()
    B.dspark_kv_write(cache.handle, k, v, first + 1, off, dev_status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == B.DEV_BAD_PAGE and T.same(cache.snapshot(), before)
