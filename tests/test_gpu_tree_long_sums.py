"""Attention over contexts so long that one SM adds up very many positions.  A block table that has one page over and over makes them:
the weights and so the result are those of the page alone."""
import math

import pytest
import torch

from paper_2607_05147_b200 import binding as B
import tree_helpers as T

pytestmark = pytest.mark.gpu

PAGE, HEADS, D = 1 << 16, 148, 16                             # a head an SM


@pytest.mark.parametrize("kind", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("group,times", [(4, 64), (4, 5), (20, 64), (48, 64), (96, 64), (96, 5)])       # rows with a head, pages
def test_long_contexts_of_many_heads(kind, group, times):
    cache = T.Cache([PAGE], PAGE, HEADS, D, kind, spare=0)
    g = T.gen(group)
    # values of one sign: what is cut of a sum does not average out
    if kind == "bf16":
        cache.k.normal_(generator=g)
        cache.v.copy_(1 + torch.rand(cache.v.shape, generator=g, device="cuda"))
    else:
        cache.k.copy_(torch.randint(-100, 100, cache.k.shape, generator=g, device="cuda").to(cache.k.dtype))
        cache.v.copy_(torch.randint(60, 127, cache.v.shape, generator=g, device="cuda").to(cache.v.dtype))
        cache.ks.fill_(0.02)
        cache.vs.fill_(1 / 64)
    q = (torch.randn(1, HEADS * group, D, generator=g, device="cuda") * 0.5).bfloat16()
    length = PAGE * times
    handle = B.KvCache(cache.k, cache.v, torch.zeros(1, times, dtype=torch.int32, device="cuda"), cache.ks, cache.vs)
    out, lse, st = torch.empty_like(q), torch.empty(1, HEADS * group, device="cuda"), T.status()
    ws = B.workspace(B.dspark_tree_attention_workspace_bytes(1, HEADS * group, HEADS, D))
    ws.fill_(255)
    B.dspark_tree_attention(q, handle, T.i32([length - 1]), T.i32([0, 1]), scale=0.25, out=out, out_lse=lse, dev_status=st, workspace=ws)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    some = slice(0, 3)                                        # of the rows with a head
    k, v = cache.values(0, range(PAGE))
    x = q[0].view(HEADS, group, D)[:, some].double()
    z = torch.einsum("hgd,lhd->hgl", x, k) * 0.25
    w = torch.softmax(z, -1)
    want = torch.einsum("hgl,lhd->hgd", w, v)                 # of positive values: also the sum of the magnitudes
    got = out[0].view(HEADS, group, D)[:, some].double()
    # the result's rounding to bf16 is half a step, 2^-9 of a value just above a power of two; weights rounded to 16 bits one by one, in
    # both directions, 2^-9 each at most; sums: 256 tiles of eight products cut by a step of 2^-23 of the sum at most, which grows
    # from nothing, 2^-13; 64 * 512 / 256 such parts added with rounding, 2^-24 each; scores and exponentials as in tree_helpers
    size = float((x.abs().amax() * k.abs().amax() * D * 0.25))
    bound = want * (2.0 ** -8 + 2.0 ** -13 + 2 * (D * 2.0 ** -23 * size + 2.0 ** -20) + 128 * 2.0 ** -24)
    assert bool(((got - want).abs() <= bound).all()), float(((got - want).abs() / want).max())
    # the roundings to 16 bits are as often up as down: over all results what is left is what has been cut
    assert abs(float(((got - want) / want).mean())) < 2.0 ** -11
    want_lse = torch.logsumexp(z, -1) + math.log(times)
    assert float((lse.view(HEADS, group)[:, some].double() - want_lse).abs().max()) < 2.0 ** -12
