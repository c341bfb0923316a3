"""Attention of drafted nodes over the paged cache against its definition in 64 bits; the bounds are derived in
tree_helpers.attention."""
import math

import pytest
import torch

from paper_2607_05147_b200 import binding as B
import tree_helpers as T

pytestmark = pytest.mark.gpu


def step(first, nodes, page, heads, group, d, kind, seed=0, layout="nhd", spread=1.0, layers=1, layer=0, fill=255):
    """A cache full of garbage with the step's positions written, and queries."""
    need = [f + n for f, n in zip(first, nodes)]
    cache = T.Cache(need, page, heads, d, kind, layout=layout, seed=seed, fill=fill, layers=layers)
    g = T.gen(seed + 7)
    for r, n in enumerate(need):
        if n:
            x = torch.randn(2, n, heads, d, generator=g, device="cuda") * spread
            x[1] += 0.5
            cache.put(r, range(n), x[0], x[1], layer=layer)
    q = (torch.randn(sum(nodes), heads * group, d, generator=g, device="cuda") * spread).bfloat16()
    return cache, q


def check(cache, q, first, nodes, parents, scale, layer=0):
    off = T.offsets(nodes)
    got, lse, st = T.run_attention(cache, q, T.i32(first), off, None if parents is None else T.i32(parents), scale, layer=layer)
    assert st == 0
    want, bound, want_lse, lse_bound = T.attention(cache, q, first, off.tolist(), parents, scale, layer)
    err = (got.double() - want).abs()
    assert torch.isfinite(got).all()
    assert bool((err <= bound).all()), (float((err / bound).max()), float(err.max()))
    assert bool(((lse.double() - want_lse).abs() <= lse_bound).all()), float((lse.double() - want_lse).abs().max())
    # the whole result: roundings of the weights average out, the result's own is 2^-8 / sqrt(3) of each value at most
    assert float(err.norm() / want.norm()) < 2.0 ** -8
    return got


SHAPES = [
    # first, nodes, page, heads, group, d
    ([0], [1], 64, 1, 1, 128),                                # a single position
    ([700], [1], 64, 2, 4, 128),
    ([127, 128, 129, 0], [1, 1, 1, 1], 16, 2, 8, 64),         # ends of a tile
    ([5, 300, 0, 77], [3, 16, 0, 1], 8, 3, 5, 80),
    ([255, 1], [130, 7], 32, 1, 16, 128),                     # several row tiles, nodes across tiles
    ([40], [200], 64, 2, 1, 96),                              # a chunk of a prompt: more than one tile of nodes
    ([600, 333], [9, 4], 200, 2, 3, 48),                      # pages that are no multiple of a tile
    ([1000], [6], 1024, 1, 128, 16),                          # one group of 128 heads: a node a row tile
    ([90, 20], [5, 70], 128, 1, 71, 64),                      # a group that leaves rows of a tile unused
]


@pytest.mark.parametrize("kind", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
@pytest.mark.parametrize("tree", ["chain", "tree"])
def test_shapes(kind, shape, tree):
    first, nodes, page, heads, group, d = SHAPES[shape]
    cache, q = step(first, nodes, page, heads, group, d, kind, seed=shape)
    check(cache, q, first, nodes, None if tree == "chain" else T.random_parents(nodes, shape), 1 / math.sqrt(d))


@pytest.mark.parametrize("kind,layout", [("bf16", "hnd"), ("bf16", "pair"), ("int8", "hnd"), ("e4m3", "pair")])
def test_layouts_and_layers(kind, layout):
    first, nodes = [200, 31], [12, 20]
    cache, q = step(first, nodes, 16, 2, 4, 128, kind, seed=3, layout=layout, layers=3, layer=2)
    check(cache, q, first, nodes, T.random_parents(nodes, 1), 0.1, layer=2)


@pytest.mark.parametrize("shape", ["star", "comb", "chain"])
def test_trees(shape):
    first, nodes = [100, 0, 250], [33, 64, 150]
    cache, q = step(first, nodes, 32, 2, 2, 64, "bf16", seed=4)
    check(cache, q, first, nodes, T.random_parents(nodes, 0, shape), 0.125)


@pytest.mark.parametrize("kind", ["bf16", "int8"])
def test_long_contexts(kind):
    # few rows and many positions: the sum over the positions is split
    first, nodes = [20000, 3], [2, 5]
    cache, q = step(first, nodes, 64, 2, 4, 128, kind, seed=5)
    check(cache, q, first, nodes, None, 1 / math.sqrt(128))


@pytest.mark.parametrize("kind", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("spread,scale", [(3.0, 0.5), (1.0, 0.0), (1.0, -0.3), (0.01, 1.0), (8.0, 1.0)])
def test_scores_of_any_size(kind, spread, scale):
    # one position takes all weight, all have the same, growing and falling maxima
    first, nodes = [500, 130], [6, 9]
    cache, q = step(first, nodes, 32, 2, 4, 64, kind, seed=6, spread=spread)
    check(cache, q, first, nodes, T.random_parents(nodes, 2), scale)


@pytest.mark.parametrize("kind", ["bf16", "int8", "e4m3"])
def test_a_first_position_that_takes_most_of_the_weight(kind):
    # 2^-12 and less for each of the others, which together hold a third of the weight: none may be lost
    first, nodes, d = [6000], [2], 64
    cache, q = step(first, nodes, 64, 1, 4, d, kind, seed=8, spread=0.02)
    k = torch.zeros(1, 1, d, device="cuda")
    k[0, 0, 0] = 8.0
    v = torch.full((1, 1, d), -1.0, device="cuda")
    cache.put(0, [0], k, v)
    q[..., 0] = 8.0
    check(cache, q, first, nodes, None, 0.15)                 # e^9.6 = 15 000 against 6 000 positions of 1


@pytest.mark.parametrize("kind", ["bf16", "int8", "e4m3"])
def test_values_of_very_different_sizes(kind):
    # the heavy position has a small value, a light one a large value
    first, nodes, d = [300], [3], 64
    cache, q = step(first, nodes, 32, 1, 4, d, kind, seed=9, spread=0.5)
    x = torch.randn(2, 300, 1, d, generator=T.gen(5), device="cuda")
    size = torch.exp2(torch.arange(300, device="cuda") % 13 - 6.0)[:, None, None]
    cache.put(0, range(300), x[0] * 0.5, x[1] * size)
    check(cache, q, first, nodes, None, 0.3)


@pytest.mark.parametrize("kind", ["bf16", "int8"])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
def test_what_other_nodes_hold_does_not_reach_a_row(kind, what):
    first, nodes = [60, 127], [20, 10]
    parents = T.random_parents(nodes, 3, "star")
    cache, q = step(first, nodes, 16, 2, 4, 64, kind, seed=10)
    clean = check(cache, q, first, nodes, parents, 0.2)
    for at_k, at_v in ((1, 0), (0, 1), (1, 1)):
        k, v = (x.float() for x in cache.values(0, range(67, 69)))
        save = cache.snapshot()
        if kind == "bf16":
            pg, at = cache.slots(0, [67, 68])
            if at_k:
                cache.k[0, pg, at] = what
            if at_v:
                cache.v[0, pg, at, :, 3] = what
        else:
            if at_k:
                k[:] = what
            if at_v:
                v[:] = what
            cache.put(0, range(67, 69), k, v)
        got, _, st = T.run_attention(cache, q, T.i32(first), T.offsets(nodes), T.i32(parents), 0.2)
        assert st == 0
        own = torch.tensor([7, 8], device="cuda")             # rows of the two nodes themselves
        others = torch.ones(30, dtype=torch.bool, device="cuda")
        others[own] = False
        assert torch.equal(got[others], clean[others])
        if at_k and what != -math.inf or (at_k and kind == "int8"):
            assert torch.isnan(got[own]).any()
        elif at_v and kind == "bf16" and not at_k:
            assert not torch.isfinite(got[own][..., 3]).any() and torch.equal(got[own][..., 4:], clean[own][..., 4:])
        raw = [cache.k, cache.v] if kind == "bf16" else [cache.k.view(torch.uint8), cache.v.view(torch.uint8)]
        for x, s in zip(raw, save):
            x.copy_(s.view(x.dtype).view(x.shape) if kind != "bf16" else s.view(torch.bfloat16).view(x.shape))
        for x, s in zip([t for t in (cache.ks, cache.vs) if t is not None], save[2:]):
            x.copy_(s.view(torch.float32))


def test_a_prefix_position_with_nan_reaches_every_row():
    first, nodes = [60], [4]
    cache, q = step(first, nodes, 16, 1, 4, 64, "bf16", seed=11)
    pg, at = cache.slots(0, [20])
    cache.v[0, pg, at, 0, 9] = math.nan
    got, _, _ = T.run_attention(cache, q, T.i32(first), T.offsets(nodes), None, 0.2)
    assert torch.isnan(got[..., 9]).all() and torch.isfinite(got[..., :9]).all()


def test_nan_codes_of_other_nodes():
    # 0x7f and 0xff are e4m3's NaN: dspark_kv_write stores none, another writer may
    first, nodes = [60, 127], [20, 10]
    parents = T.random_parents(nodes, 3, "star")
    cache, q = step(first, nodes, 16, 2, 4, 64, "e4m3", seed=10)
    clean = check(cache, q, first, nodes, parents, 0.2)
    pg, at = cache.slots(0, [67, 68])
    cache.v.view(torch.uint8)[0, pg, at, :, 3] = 0x7f
    cache.k.view(torch.uint8)[0, pg[:1], at[:1], :, 5] = 0xff
    got, _, st = T.run_attention(cache, q, T.i32(first), T.offsets(nodes), T.i32(parents), 0.2)
    others = torch.ones(30, dtype=torch.bool, device="cuda")
    others[7:9] = False
    assert st == 0 and torch.equal(got[others], clean[others])
    assert torch.isnan(got[7]).all() and torch.isnan(got[8, :, 3]).all() and torch.equal(got[8, :, 4:], clean[8, :, 4:])


def test_large_scales_of_other_nodes():
    # what a node that a row does not see has stored is not in that row's arithmetic, whatever its size
    first, nodes = [60], [20]
    parents = T.random_parents(nodes, 3, "star")
    cache, q = step(first, nodes, 16, 2, 4, 64, "int8", seed=10)
    clean = check(cache, q, first, nodes, parents, 0.2)
    pg, at = cache.slots(0, [67, 68])
    cache.vs[0, pg, :, at] = 1e30
    got, _, _ = T.run_attention(cache, q, T.i32(first), T.offsets(nodes), T.i32(parents), 0.2)
    others = torch.ones(20, dtype=torch.bool, device="cuda")
    others[7:9] = False
    assert torch.equal(got[others], clean[others]) and torch.isfinite(got).all()


def test_rows_strides_outputs_in_place_and_rows_behind_the_last_request():
    first, nodes, d = [50, 10], [6, 3], 64
    cache, q0 = step(first, nodes, 16, 2, 4, d, "bf16", seed=12)
    want, bound, _, _ = T.attention(cache, q0, first, [0, 6, 9], None, 0.2)
    wide = torch.full((14, 12, d), 5.0, dtype=torch.bfloat16, device="cuda")       # q as the first heads of a projection
    q = wide[:, :8]
    q[:9] = q0
    out = torch.full((14, 10, 2 * d), 2.0, dtype=torch.bfloat16, device="cuda")
    view = out[:, 1:9, :d]
    got, lse, st = T.run_attention(cache, q, T.i32(first), T.offsets(nodes), None, 0.2, out=view)
    assert st == 0 and bool(((got[:9].double() - want).abs() <= bound[:9]).all())
    assert (out[9:] == 2).all() and (out[:, 0] == 2).all() and (out[:, 9] == 2).all() and (out[:, :, d:] == 2).all() and (lse[9:] == 7).all()
    T.run_attention(cache, q, T.i32(first), T.offsets(nodes), None, 0.2, out=q)
    assert torch.equal(q[:9], view[:9]) and (wide[:, 8:] == 5).all() and (q[9:] == 5).all()


def test_the_same_bits_again_and_with_other_requests():
    first, nodes = [3000, 50, 900], [5, 2, 8]
    cache, q = step(first, nodes, 64, 2, 4, 128, "int8", seed=13)
    a = T.run_attention(cache, q, T.i32(first), T.offsets(nodes), None, 0.1)[0]
    for _ in range(3):
        assert torch.equal(a, T.run_attention(cache, q, T.i32(first), T.offsets(nodes), None, 0.1)[0])


def test_what_the_device_refuses():
    first, nodes = [50, 20, 30, 40], [3, 3, 3, 3]
    cache, q = step(first, nodes, 16, 2, 4, 64, "bf16", seed=14)
    off = T.offsets(nodes)
    want = T.run_attention(cache, q, T.i32(first), off, None, 0.2)[0]
    # a negative length, one past the table: their rows stay, the others are computed
    got, lse, st = T.run_attention(cache, q, T.i32([50, -1, 30, 1000]), off, None, 0.2)
    assert st == B.DEV_BAD_PAGE
    assert torch.equal(got[:3], want[:3]) and torch.equal(got[6:9], want[6:9]) and (got[3:6] == 7).all() and (got[9:] == 7).all()
    got, _, st = T.run_attention(cache, q, T.i32(first), T.i32([0, 3, 6, 9, 13]), None, 0.2)
    assert st == B.DEV_BAD_OFFSETS and torch.equal(got[:9], want[:9]) and (got[9:] == 7).all()
    assert T.run_attention(cache, q, T.i32(first), T.i32([0, 6, 3, 9, 12]), None, 0.2)[2] & B.DEV_BAD_OFFSETS
    # a parent that is no earlier node ends the ancestors there
    par = T.random_parents(nodes, 0, "chain")
    par[5] = 2                                                # node 2 of request 1: itself
    assert T.run_attention(cache, q, T.i32(first), off, T.i32(par), 0.2)[2] == B.DEV_BAD_TREE
    # pages that are not there read as zeros
    cache.table[0, 1] = cache.pages
    cache.table[2, 0] = -1
    got, _, st = T.run_attention(cache, q, T.i32(first), off, None, 0.2)
    assert st == B.DEV_BAD_PAGE and torch.equal(got[3:6], want[3:6]) and torch.equal(got[9:], want[9:]) and torch.isfinite(got).all()


def test_captured_graphs_share_a_workspace():
    shapes = [([400, 20], [5, 9]), ([30, 1500], [2, 7])]
    steps = []
    for first, nodes in shapes:
        cache, q = step(first, nodes, 32, 2, 4, 128, "int8", seed=15)
        steps.append((cache, q, T.i32(first), T.offsets(nodes), torch.zeros_like(q), T.status(), first, nodes))
    ws = B.workspace(max(B.dspark_tree_attention_workspace_bytes(s[1].shape[0], 8, 2, 128) for s in steps))
    graphs = []
    for cache, q, first, off, out, st, _, _ in steps:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side), torch.cuda.graph(g, stream=side):
            B.dspark_tree_attention(q, cache.handle, first, off, scale=0.1, out=out, dev_status=st, workspace=ws)
        graphs.append(g)
    for _ in range(3):
        for g, (cache, q, first, off, out, st, f, n) in zip(graphs, steps):
            ws.fill_(255)
            q.copy_(torch.randn(q.shape, generator=T.gen(1), device="cuda"))
            g.replay()
    torch.cuda.synchronize()
    for cache, q, first, off, out, st, f, n in steps:
        want, bound, _, _ = T.attention(cache, q, f, off.tolist(), None, 0.1)
        assert int(st.item()) == 0 and bool(((out.double() - want).abs() <= bound).all())


def test_many_requests():
    # more requests than threads that look for them, many of them empty
    R = 1300
    first, nodes = [(i * 13) % 40 for i in range(R)], [(i % 5) % 3 for i in range(R)]
    cache, q = step(first, nodes, 8, 1, 2, 16, "bf16", seed=16)
    check(cache, q, first, nodes, None, 0.25)


@pytest.mark.parametrize("kind", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("group,tree", [(4, "chain"), (4, "tree"), (8, "tree"), (16, "chain")])
def test_units_of_all_lengths_in_a_run(kind, group, tree):
    # more tiles than SMs, units of one to nine of them that begin anywhere in an SM's run and end in the next one's
    first = [(r * 97) % 1100 for r in range(60)]
    nodes = [1 + (r * 5) % 4 for r in range(60)]
    parents = None if tree == "chain" else T.random_parents(nodes, 3)
    cache, q = step(first, nodes, 32, 2, group, 64, kind, seed=11)
    check(cache, q, first, nodes, parents, 0.125)


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
@pytest.mark.parametrize("group", [4, 40])
def test_what_other_requests_and_branches_hold(kind, group):
    # eight and eighty rows with a head: NaN scales at positions that a node does not see leave its row alone, also where the tile is the
    # only one of its unit, and scales far above those that it sees do not cost it its digits
    first, nodes = [0, 100, 128, 250], [2, 2, 2, 2]
    parents = [-1, 0] * 4
    cache, q = step(first, nodes, 16, 2, group, 128, kind, seed=5)
    for r in range(4):
        pg, at = cache.slots(r, [first[r] + 1])
        cache.vs[0, pg, :, at] = 2.0 ** 30 if r % 2 else math.nan
    off = T.offsets(nodes)
    got, _, st = T.run_attention(cache, q, T.i32(first), off, T.i32(parents), 0.1)
    want, bound, _, _ = T.attention(cache, q, first, off.tolist(), parents, 0.1)
    assert st == 0
    for r in range(4):
        root = off[r].item()
        assert bool(((got[root].double() - want[root]).abs() <= bound[root]).all())
        if r % 2 == 0:
            assert bool(got[root + 1].isnan().all())
