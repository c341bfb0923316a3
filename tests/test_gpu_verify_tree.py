"""Verification of drafted trees from given random numbers against the walk in 64 bits on the host: the same integers."""
import math

import pytest
import torch

from paper_2607_05147_b200 import binding as B
import tree_helpers as T

pytestmark = pytest.mark.gpu


def batch(nodes, V, seed, shape="tree", near=0.7, pitch=0):
    g = T.gen(seed)
    n = sum(nodes)
    z = torch.randn(n, V, generator=g, device="cuda") * 2
    z[:, :: max(1, V // 16)] += 6
    wide = [torch.full((n, V + pitch), math.nan, device="cuda") for _ in range(2)]
    p, q = (w[:, :V] for w in wide)
    p.copy_(torch.softmax(z, 1))
    q.copy_(torch.softmax(z + near * torch.randn(n, V, generator=g, device="cuda"), 1))
    parents = T.random_parents(nodes, seed, shape)
    off = T.offsets(nodes).tolist()
    tokens = torch.zeros(n, dtype=torch.int64, device="cuda")
    for r in range(len(nodes)):
        for i in range(1, nodes[r]):
            tokens[off[r] + i] = torch.multinomial(q[off[r] + parents[off[r] + i]], 1, generator=g)[0]
    u, u_last = torch.rand(n, generator=g, device="cuda"), torch.rand(len(nodes), generator=g, device="cuda")
    return p, q, tokens.to(torch.int32), parents, off, u, u_last


def run(p, q, tokens, parents, off, u, u_last, path=True):
    R, n = len(off) - 1, p.shape[0]
    acc, out, pth = (torch.full((m,), -7, dtype=torch.int32, device="cuda") for m in (R, n, n))
    st = T.status()
    B.dspark_verify_tree(p, q, tokens, T.i32(parents), T.i32(off), u, u_last, accepted_len=acc, out_tokens=out,
                         out_path=pth if path else None, dev_status=st)
    torch.cuda.synchronize()
    return acc.tolist(), out.tolist(), pth.tolist(), int(st.item())


def check(p, q, tokens, parents, off, u, u_last):
    acc, out, path, st = run(p, q, tokens, parents, off, u, u_last)
    want = T.verify(p, q, tokens.tolist(), parents, off, u.tolist(), u_last.tolist())
    assert st == 0 and (acc, out, path) == want
    return acc


@pytest.mark.parametrize("nodes,V,pitch", [([1], 1, 0), ([1, 1], 5, 3), ([2, 1, 7], 10, 0), ([16, 9, 30], 1000, 0), ([16, 9, 30], 1001, 0),
                                           ([12] * 20, 4097, 2), ([32, 5], 129280, 0), ([8, 64], 16384 * 8 + 1, 7)])
@pytest.mark.parametrize("draft", [True, False])
def test_sizes(nodes, V, pitch, draft):
    b = list(batch(nodes, V, 3, pitch=pitch))
    if not draft:
        b[1] = None
    check(*b)


@pytest.mark.parametrize("shape", ["chain", "star", "comb", "tree"])
@pytest.mark.parametrize("near", [0.0, 0.3, 3.0])
def test_trees(shape, near):
    # near 0: every first child is accepted; 3: most are rejected, and several at a node
    acc = check(*batch([20] * 24, 700, 5, shape, near))
    if near == 0.0:
        assert (min(acc) == 19) if shape == "chain" else True
    if shape == "star":
        assert max(acc) <= 1


def test_the_distribution_is_the_targets():
    # a small vocabulary, two drafted tokens: what is emitted first is distributed as the target says (lossless)
    V, R = 6, 20000
    g = T.gen(9)
    p1, q1 = torch.softmax(torch.randn(V, generator=g, device="cuda"), 0), torch.softmax(torch.randn(V, generator=g, device="cuda"), 0)
    p, q = p1.repeat(3 * R, 1), q1.repeat(3 * R, 1)
    tokens = torch.multinomial(q1, 3 * R, replacement=True, generator=g).to(torch.int32)
    parents, off = [-1, 0, 0] * R, list(range(0, 3 * R + 1, 3))
    u, u_last = torch.rand(3 * R, generator=g, device="cuda"), torch.rand(R, generator=g, device="cuda")
    _, out, _, st = run(p, q, tokens, parents, off, u, u_last)
    assert st == 0
    seen = torch.bincount(torch.tensor(out[::3]), minlength=V).double() / R
    # five standard deviations of a count
    assert bool(((seen - p1.double().cpu()).abs() < 5 * (p1.double().cpu() / R).sqrt()).all())


def test_the_same_token_drafted_twice():
    V = 50
    for draft in (True, False):
        p, q, tokens, parents, off, u, u_last = batch([6] * 30, V, 7, "star", 2.0)
        tokens[:] = tokens.view(30, 6)[:, 1:2].expand(30, 6).reshape(-1)
        u[:] = torch.where(torch.arange(180, device="cuda") % 6 < 3, 0.999, 0.5)
        check(p, q if draft else None, tokens, parents, off, u, u_last)


def test_a_residual_without_mass():
    # p = q, and a number so near to one that rounding rejects nothing; then q larger than p at the token alone, all of p there
    V = 8
    p = torch.zeros(2, V, device="cuda")
    p[:, 3] = 1.0
    acc, out, path, st = run(p, None, T.i32([0, 5]), [-1, 0], [0, 2], torch.tensor([0.5, 0.0], device="cuda"), torch.tensor([0.99], device="cuda"))
    assert (acc, out, path, st) == ([0], [3, -1], [-1, -1], 0)
    q = torch.full((2, V), 1.0, device="cuda")                # no distribution: it takes all of p away
    acc, out, path, st = run(p, q, T.i32([0, 5]), [-1, 0], [0, 2], torch.tensor([0.5, 0.5], device="cuda"), torch.tensor([0.0], device="cuda"))
    assert (acc, out, st) == ([0], [3, -1], 0)


def test_numbers_at_the_ends():
    V = 300
    p, q, tokens, parents, off, u, u_last = batch([5, 5], V, 8)
    top = 1 - 2.0 ** -24
    for a in (0.0, top):
        for b in (0.0, top):
            check(p, q, tokens, parents, off, torch.full_like(u, a), torch.full_like(u_last, b))


def test_what_voids_a_request():
    nodes, V = [4, 4, 4, 4, 4, 4], 40
    p, q, tokens, parents, off, u, u_last = batch(nodes, V, 2, "chain", 0.0)
    good = run(p, q, tokens, parents, off, u, u_last)
    parents = list(parents)
    parents[4 * 1 + 2] = 2                                    # itself
    tokens[4 * 2 + 3] = V
    p[4 * 3] = math.nan
    p[4 * 4] = 0.0
    q[4 * 4] = 0.0                                            # nothing at the root
    acc, out, path, st = run(p, q, tokens, parents, off, u, u_last)
    assert st == B.DEV_BAD_TREE | B.DEV_BAD_TOKEN | B.DEV_BAD_ROW
    for r in (0, 5):
        assert acc[r] == good[0][r] and out[4 * r: 4 * r + 4] == good[1][4 * r: 4 * r + 4]
    for r in (1, 2, 3, 4):
        assert acc[r] == 0 and out[4 * r: 4 * r + 4] == [-1] * 4 and path[4 * r: 4 * r + 4] == [-1] * 4
    acc, out, _, st = run(p, q, tokens, parents, [0, 4, 4, 2, 30, 24, 24], u, u_last)
    assert st & B.DEV_BAD_OFFSETS and acc[1] == 0 and acc[3] == 0


def test_more_nodes_than_it_takes():
    n = B.TREE_MAX_NODES + 1
    p, q, tokens, parents, off, u, u_last = batch([n - 1], 20, 4, "chain", 0.05)
    check(p, q, tokens, parents, off, u, u_last)
    p, q, tokens, parents, off, u, u_last = batch([n, 3], 20, 4, "chain", 0.05)
    acc, out, path, st = run(p, q, tokens, parents, off, u, u_last)
    assert st == B.DEV_BAD_OFFSETS and acc[0] == 0 and out[:n] == [-1] * n and path[:n] == [-1] * n and out[n + acc[1]] >= 0


def test_captured_without_path():
    p, q, tokens, parents, off, u, u_last = batch([9, 3], 2000, 6)
    par, o = T.i32(parents), T.i32(off)
    acc, out, st = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(12, dtype=torch.int32, device="cuda"), T.status()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        B.dspark_verify_tree(p, q, tokens, par, o, u, u_last, accepted_len=acc, out_tokens=out, dev_status=st)
    for seed in (1, 2, 3):
        u.copy_(torch.rand(12, generator=T.gen(seed), device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        want = T.verify(p, q, tokens.tolist(), parents, off, u.tolist(), u_last.tolist())
        assert int(st.item()) == 0 and acc.tolist() == want[0] and out.tolist() == want[1]
