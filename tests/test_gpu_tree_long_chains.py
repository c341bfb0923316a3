"""Requests of many nodes given with parents: prompts' chunks in a batch with trees, trees behind a chain, deep trees."""
import math

import pytest
import torch

from paper_2607_05147_b200 import binding as B
import tree_helpers as T

pytestmark = pytest.mark.gpu

D = 32


def ancestors_of(parents):
    """[n, n] of one request: whether node j is i or an ancestor of it."""
    n = len(parents)
    seen = torch.eye(n, dtype=torch.bool, device="cuda")
    for i in range(1, n):
        seen[i] |= seen[parents[i]]
    return seen


def dense(cache, r, q, first, seen, scale):
    """(out, bound) of request r's rows q [n, heads * group, d] in 64 bits; the bound as tree_helpers.attention derives it."""
    n, hq, d = q.shape
    h = cache.heads
    k, v = cache.values(r, range(first + n))
    hidden = torch.cat([torch.zeros(n, first, dtype=torch.bool, device="cuda"), ~seen], 1)
    out, bound = (torch.zeros(n, hq, d, dtype=torch.float64, device="cuda") for _ in range(2))
    for a in range(hq):
        b = a * h // hq
        x = q[:, a].double()
        w = torch.softmax((x @ k[:, b].T * scale).masked_fill(hidden, -math.inf), -1)
        size = (x.abs() @ k[:, b].abs().T * abs(scale)).masked_fill(hidden, 0).amax(-1, keepdim=True)
        o, m = w @ v[:, b], w @ v[:, b].abs()
        tiny = 0.0
        if cache.kind != "bf16":
            tiny = (first + n) * 2.0 ** -32 * 2 * (127 if cache.kind == "int8" else 448) * float(cache.vs.abs().nan_to_num(0).max()) * w.amax(-1, keepdim=True)
        out[:, a], bound[:, a] = o, tiny + 2.0 ** -8 * (m + o.abs()) * 1.01 + 2 * (d * 2.0 ** -23 * size + 2.0 ** -20) * m + 1e-37
    return out, bound


def batch(requests, kind, heads, group, seed=0):
    """requests: (first, parents) each."""
    first, nodes = [f for f, _ in requests], [len(p) for _, p in requests]
    cache = T.Cache([f + n for f, n in zip(first, nodes)], 32, heads, D, kind, seed=seed, fill=255)
    g = T.gen(seed)
    for r, (f, n) in enumerate(zip(first, nodes)):
        x = torch.randn(2, f + n, heads, D, generator=g, device="cuda")
        x[1] += 0.5
        cache.put(r, range(f + n), x[0], x[1])
    q = torch.randn(sum(nodes), heads * group, D, generator=g, device="cuda").bfloat16()
    return cache, q, first, nodes


def check(requests, kind, heads, group, scale=0.2):
    cache, q, first, nodes = batch(requests, kind, heads, group)
    off = T.offsets(nodes)
    got, _, st = T.run_attention(cache, q, T.i32(first), off, T.i32([p for _, ps in requests for p in ps]), scale)
    assert st == 0
    o = off.tolist()
    for r, (f, ps) in enumerate(requests):
        rows = slice(o[r], o[r + 1])
        want, bound = dense(cache, r, q[rows], f, ancestors_of(ps), scale)
        assert bool(((got[rows].double() - want).abs() <= bound).all()), r


def chain(n):
    return [-1] + list(range(n - 1))


def behind(n, m, seed, shape="tree"):
    """A chain of n nodes, then m nodes of a tree that grows from any of the last eight of the chain."""
    g = torch.Generator().manual_seed(seed)
    out = chain(n)
    for i in range(n, n + m):
        low = max(0, n - 8)
        out.append(int(torch.randint(low, i, (1,), generator=g)) if shape == "tree" else n - 1)
    return out


@pytest.mark.parametrize("kind", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("group", [1, 4])
def test_a_chunk_with_parents_gives_the_bits_of_one_without(kind, group):
    requests = [(70, chain(1500)), (0, chain(129)), (33, chain(128)), (5, chain(1)), (500, chain(3))]
    for some in (requests, requests[:1], requests + [(i, chain(1)) for i in range(100)]):
        cache, q, first, nodes = batch(some, kind, 1, group)
        off, par = T.offsets(nodes), T.i32([p for _, ps in some for p in ps])
        a = T.run_attention(cache, q, T.i32(first), off, None, 0.2)
        b = T.run_attention(cache, q, T.i32(first), off, par, 0.2)
        assert a[2] == b[2] == 0 and torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("kind", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("others", [0, 60])                   # 60 single tokens beside: the kernel for few rows
@pytest.mark.parametrize("n,m", [(127, 30), (128, 1), (129, 70), (511, 20), (512, 20), (513, 20), (700, 300), (2, 400), (1, 300)])
def test_a_tree_behind_a_chain(kind, others, n, m):
    requests = [(70, behind(n, m, n)), (3, behind(n // 2 + 1, m, 1, "star"))] + [(i % 50, chain(1)) for i in range(others)] + [(20, chain(200))]
    check(requests, kind, 1, 3 if others else 1)


@pytest.mark.parametrize("others", [0, 600])
def test_a_deep_tree(others):
    # node 1 is a leaf, the others a chain past it
    n = 4097 if others == 0 else 900
    parents = [-1, 0, 0] + list(range(2, n - 1))
    check([(10, parents)] + [(7, chain(1))] * others, "bf16", 1, 1)


def test_two_long_branches():
    # 3000 nodes each from a prompt of 200
    n = 6200
    parents = [-1] + [199 if i == 3200 else i - 1 for i in range(1, n)]
    check([(10, parents), (30, chain(5))], "bf16", 1, 1)


def test_more_ancestors_than_are_looked_at():
    # 65536 outside the chain that a request begins with; here that chain is node 0 and 1, and node 1 is a leaf
    n, last = 65536 + 300, 65536
    parents = [-1, 0, 0] + list(range(2, n - 1))
    cache = T.Cache([n], 64, 1, 16, "bf16")
    g = T.gen(1)
    cache.k.normal_(generator=g)
    cache.v.normal_(generator=g)
    q = torch.randn(n, 1, 16, generator=g, device="cuda").bfloat16()
    got, _, st = T.run_attention(cache, q, T.i32([0]), T.i32([0, n]), T.i32(parents), 0.2)
    assert st == B.DEV_BAD_TREE and bool(got.isfinite().all())
    # as a chain without node 1: the rows up to the last whose walk is whole
    k, v = (x[:, 0] for x in cache.values(0, range(n)))
    for row in (2, 3, 5000, 40000, last - 100, last, last + 1):
        seen = torch.tensor([0] + list(range(2, row + 1)), device="cuda")
        x = q[row, 0].double()
        w = torch.softmax(k[seen] @ x * 0.2, 0)
        want, m = w @ v[seen], w @ v[seen].abs()
        size = float((k[seen].abs() @ x.abs()).max()) * 0.2
        bound = 2.0 ** -8 * (m + want.abs()) * 1.01 + 2 * (16 * 2.0 ** -23 * size + 2.0 ** -20) * m + 2.0 ** -11 * m
        assert bool(((got[row, 0].double() - want).abs() <= bound).all()), row


@pytest.mark.parametrize("others", [0, 60])
def test_a_bad_parent_behind_a_chain(others):
    parents = chain(300) + [299, 400, 299]                    # node 301's is no earlier node
    requests = [(10, parents)] + [(7, chain(1))] * others
    cache, q, first, nodes = batch(requests, "bf16", 1, 1)
    got, _, st = T.run_attention(cache, q, T.i32(first), T.offsets(nodes), T.i32([p for _, ps in requests for p in ps]), 0.2)
    assert st == B.DEV_BAD_TREE
    seen = ancestors_of(chain(300) + [299, 299, 299])
    seen[301] = False
    seen[301, 301] = True                                     # itself and what was before the step
    want, bound = dense(cache, 0, q[:303], 10, seen, 0.2)
    assert bool(((got[:303].double() - want).abs() <= bound).all())
