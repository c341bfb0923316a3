"""Attention over caches whose scales another writer has chosen: of either sign, zero, far from one.  value = scale * stored."""
import pytest
import torch

import tree_helpers as T
from test_gpu_tree_attention import step

pytestmark = pytest.mark.gpu

STEPS = [
    # first, nodes, group: 4, 32 and 256 rows with a head
    ([700, 130, 0], [1, 1, 1], 4),
    ([300, 127, 250], [8, 3, 5], 4),
    ([260, 40], [40, 33], 7),
]


class Magnitudes:
    """The cache with the magnitudes of V's scales, as the bound of T.attention takes them."""

    def __init__(self, cache):
        self.kind, self.heads, self.slots, self.values = cache.kind, cache.heads, cache.slots, cache.values
        self.vs = None if cache.vs is None else cache.vs.abs()


def check(cache, q, first, nodes, parents, scale, lost=0.0):
    """lost: what is lost of each position beside the bound of T.attention, of the largest weight and stored value."""
    off = T.offsets(nodes)
    got, lse, st = T.run_attention(cache, q, T.i32(first), off, None if parents is None else T.i32(parents), scale)
    assert st == 0
    want, bound, want_lse, lse_bound = T.attention(Magnitudes(cache), q, first, off.tolist(), parents, scale)
    if lost:
        bound = bound + lost * max(f + n for f, n in zip(first, nodes)) * (127 if cache.kind == "int8" else 448)
    assert bool(((got.double() - want).abs() <= bound).all()), float(((got.double() - want).abs() / bound).max())
    assert bool(((lse.double() - want_lse).abs() <= lse_bound).all())
    return got


def signs(x, g, zeros=0.1):
    """Half of the entries negative, some zero."""
    u = torch.rand(x.shape, generator=g, device="cuda")
    x.mul_(torch.where(u < 0.5, -1.0, 1.0)).mul_(torch.where(u > 1 - zeros, 0.0, 1.0))


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("shape", range(len(STEPS)))
@pytest.mark.parametrize("tree", ["chain", "tree"])
@pytest.mark.parametrize("scale", [0.2, -0.2, 0.0])
def test_scales_of_k_of_either_sign(kind, shape, tree, scale):
    first, nodes, group = STEPS[shape]
    cache, q = step(first, nodes, 16, 2, group, 64, kind, seed=shape)
    signs(cache.ks, T.gen(3))
    check(cache, q, first, nodes, None if tree == "chain" else T.random_parents(nodes, 3), scale)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("shape", range(len(STEPS)))
def test_small_scales_of_k(kind, shape):
    # times large queries: scores of an ordinary size
    first, nodes, group = STEPS[shape]
    cache, q = step(first, nodes, 16, 2, group, 64, kind, seed=shape)
    cache.ks.mul_(1e-22)
    q = (q.float() * 1e22).bfloat16()
    check(cache, q, first, nodes, T.random_parents(nodes, 3), 0.2)


@pytest.mark.parametrize("kind", ["bf16", "int8"])
@pytest.mark.parametrize("scale", [1e-24, -1e-24])
def test_a_small_scale_of_the_scores(kind, scale):
    first, nodes, group = STEPS[1]
    cache, q = step(first, nodes, 16, 2, group, 64, kind, seed=4)
    if kind == "bf16":
        cache.k.mul_(2.0 ** 40)
        q = (q.float() * 2.0 ** 38).bfloat16()
    else:
        cache.ks.mul_(2.0 ** 40)
        q = (q.float() * 2.0 ** 38).bfloat16()
    check(cache, q, first, nodes, T.random_parents(nodes, 3), scale)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("shape", range(len(STEPS)))
def test_a_node_that_a_row_does_not_see_with_a_negative_scale(kind, shape):
    # nor does its sign matter to the others
    first, nodes, group = STEPS[shape]
    nodes = [max(n, 3) for n in nodes]
    parents = T.random_parents(nodes, 3, "star")
    cache, q = step(first, nodes, 16, 2, group, 64, kind, seed=shape)
    clean = check(cache, q, first, nodes, parents, 0.3)
    off = T.offsets(nodes).tolist()
    changed = []
    for r, f in enumerate(first):
        pg, at = cache.slots(r, [f + 2])
        cache.ks[0, pg, :, at] *= -50.0
        changed.append(off[r] + 2)
    got = check(cache, q, first, nodes, parents, 0.3)
    same = torch.ones(q.shape[0], dtype=torch.bool, device="cuda")
    same[changed] = False
    assert torch.equal(got[same], clean[same])


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("shape", range(len(STEPS)))
@pytest.mark.parametrize("tree", ["chain", "tree"])
def test_scales_of_v_of_either_sign(kind, shape, tree):
    first, nodes, group = STEPS[shape]
    cache, q = step(first, nodes, 16, 2, group, 64, kind, seed=shape)
    signs(cache.vs, T.gen(3))
    check(cache, q, first, nodes, None if tree == "chain" else T.random_parents(nodes, 3), 0.2)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("shape", range(len(STEPS)))
@pytest.mark.parametrize("size", [-1.0, -100.0, -1e9, -1e20])
def test_scales_of_v_all_negative(kind, shape, size):
    first, nodes, group = STEPS[shape]
    cache, q = step(first, nodes, 16, 2, group, 64, kind, seed=shape)
    cache.vs.mul_(size)
    check(cache, q, first, nodes, T.random_parents(nodes, 3), 0.2)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("shape", range(len(STEPS)))
@pytest.mark.parametrize("tree", ["chain", "tree"])
def test_small_scales_of_v(kind, shape, tree):
    # the largest at 2^-79: no digit is lost
    first, nodes, group = STEPS[shape]
    cache, q = step(first, nodes, 16, 2, group, 64, kind, seed=shape)
    assert not cache.vs.isfinite().all()                      # (places that no request has)
    seen = torch.where(cache.vs.isfinite(), cache.vs, 0.0)
    cache.vs.mul_(2.0 ** -79 / float(seen.max()))
    check(cache, q, first, nodes, None if tree == "chain" else T.random_parents(nodes, 3), 0.2)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("shape", range(len(STEPS)))
def test_values_around_1e_minus_26(kind, shape):
    # scales of 2^-92 and less, as dspark_kv_write stores them: 2^-112 of the largest weight is lost of a position, half a step of
    # 2^-24 where the reference's weight is 2^7 at a scale of 2^-80; twice that, for the reference may be above the largest weight's
    first, nodes, group = STEPS[shape]
    cache, q = step(first, nodes, 16, 2, group, 64, kind, seed=shape)
    g = T.gen(shape)
    for r, n in enumerate(f + m for f, m in zip(first, nodes)):
        x = torch.randn(2, n, 2, 64, generator=g, device="cuda")
        cache.put(r, range(n), x[0], (x[1] + 0.5) * 1e-26)
    check(cache, q, first, nodes, T.random_parents(nodes, 3), 0.2, lost=2 * 2.0 ** -112)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("shape", range(len(STEPS)))
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("size", [2.0 ** 100, 2.0 ** -70])
def test_scales_of_k_far_from_one(kind, shape, sign, size):
    # scores of an ordinary size: queries as far from one on the other side
    first, nodes, group = STEPS[shape]
    cache, q = step(first, nodes, 16, 2, group, 64, kind, seed=shape)
    cache.ks.mul_(sign * size)
    q = (q.float() / size).bfloat16()
    check(cache, q, first, nodes, T.random_parents(nodes, 3), 0.2)
