"""Rows written to the paged cache and read back, accepted paths moved together, against their definitions in 64 bits."""
import math

import pytest
import torch

from paper_2607_05147_b200 import binding as B
import tree_helpers as T

pytestmark = pytest.mark.gpu


def rows_of(n, heads, d, seed, wide=False):
    """bf16 K and V rows; as views of one projection's output when `wide`."""
    g = T.gen(seed)
    x = torch.randn(n, 3 if wide else 2, heads, d, generator=g, device="cuda") * (0.1 + 5 * torch.rand(n, 3 if wide else 2, heads, 1, generator=g, device="cuda"))
    x = x.bfloat16()
    return (x[:, 1], x[:, 2]) if wide else (x[:, 0].contiguous(), x[:, 1].contiguous())


def write(cache, k, v, first, off, layer=0):
    st = T.status()
    B.dspark_kv_write(cache.handle, k, v, first, off, layer=layer, dev_status=st)
    torch.cuda.synchronize()
    return int(st.item())


def read(cache, first, off, n, dtype, layer=0, fill=3.0):
    st = T.status()
    k, v = (torch.full((n, cache.heads, cache.d), fill, dtype=dtype, device="cuda") for _ in range(2))
    B.dspark_kv_read(cache.handle, first, off, out_k=k, out_v=v, layer=layer, dev_status=st)
    torch.cuda.synchronize()
    return k, v, int(st.item())


CASES = [
    # kind, first, nodes, page, heads, d, layout
    ("bf16", [0], [1], 64, 1, 128, "nhd"),
    ("int8", [0], [1], 64, 1, 128, "nhd"),
    ("e4m3", [700], [8], 64, 8, 128, "nhd"),
    ("int8", [3, 0, 17, 100], [5, 0, 1, 30], 8, 3, 80, "hnd"),
    ("e4m3", [3, 0, 17, 100], [5, 0, 1, 30], 16, 5, 16, "pair"),
    ("bf16", [3, 0, 17, 100], [5, 0, 1, 30], 16, 5, 48, "pair"),
    ("int8", [1000, 5], [3, 200], 200, 2, 256, "nhd"),
    ("e4m3", [129, 127, 128], [1, 1, 129], 128, 2, 64, "hnd"),
    ("int8", [i % 37 for i in range(300)], [(i * 7) % 4 for i in range(300)], 16, 2, 96, "nhd"),
    ("int8", [i % 5 for i in range(1500)], [i % 3 for i in range(1500)], 8, 1, 32, "nhd"),      # beyond the counted look-up
]


@pytest.mark.parametrize("kind,first,nodes,page,heads,d,layout", CASES)
@pytest.mark.parametrize("wide", [False, True])
def test_write_stores_the_definition_and_nothing_else(kind, first, nodes, page, heads, d, layout, wide):
    need = [f + n for f, n in zip(first, nodes)]
    cache, want = (T.Cache(need, page, heads, d, kind, layers=2, layout=layout, seed=5) for _ in range(2))
    rows = sum(nodes)
    k, v = rows_of(rows + 3, heads, d, 11, wide)              # three rows behind the last request: not looked at
    off = T.offsets(nodes)
    assert write(cache, k, v, T.i32(first), off, layer=1) == 0
    o = off.tolist()
    for r in range(len(nodes)):
        if nodes[r]:
            want.put(r, range(first[r], first[r] + nodes[r]), k[o[r]: o[r + 1]], v[o[r]: o[r + 1]], layer=1)
    assert T.same(cache.snapshot(), want.snapshot())
    for dtype in (torch.bfloat16, torch.float32):
        a, b, st = read(cache, T.i32(first), off, rows + 3, dtype, layer=1)
        assert st == 0
        for r in range(len(nodes)):
            if nodes[r]:
                x, y = cache.values(r, range(first[r], first[r] + nodes[r]), layer=1)
                # one product in fp32, one rounding to the output's type
                assert torch.equal(a[o[r]: o[r + 1]], x.float().to(dtype)) and torch.equal(b[o[r]: o[r + 1]], y.float().to(dtype))
        assert (a[rows:] == 3).all() and (b[rows:] == 3).all()


@pytest.mark.parametrize("kind", ["int8", "e4m3"])
def test_rows_at_the_ends_of_the_range(kind):
    d = 64
    cache, want = (T.Cache([40], 16, 1, d, kind) for _ in range(2))
    x = torch.randn(10, 1, d, generator=T.gen(3), device="cuda").bfloat16()
    x[0] = 0
    x[1, 0, 5] = math.nan
    x[2, 0, 63] = math.inf
    x[3, 0, 0] = -math.inf
    x[4] = x[4] * 3e38
    x[4].clamp_(-3.3e38, 3.3e38)
    x[5] = x[5] * 1e-38
    x[6] = torch.tensor(2.0 ** -133).bfloat16()               # the smallest bf16
    x[7] = 0
    x[7, 0, 9] = -1
    # ties: 127 x / max is a half for max = 2: x = k / 127 has none, so powers of two: max 127, x = n + 1/2
    x[8] = 0.5 + torch.arange(d, device="cuda")[None].bfloat16()
    x[8, 0, 63] = 127
    x[9] = (1 + torch.arange(d, device="cuda") / 16.0)[None].bfloat16()
    x[9, 0, 63] = 448
    assert write(cache, x, x, T.i32([7]), T.i32([0, 10])) == 0
    want.put(0, range(7, 17), x, x)
    a, b = cache.snapshot(), want.snapshot()
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    s, t = cache.ks, want.ks
    assert torch.equal(torch.isnan(s), torch.isnan(t)) and torch.isnan(s).sum() == 3
    assert torch.equal(s.nan_to_num(0), t.nan_to_num(0))
    k, _, st = read(cache, T.i32([7]), T.i32([0, 10]), 10, torch.float32)
    assert st == 0 and torch.isnan(k[1:4]).all() and (k[0] == 0).all() and torch.isfinite(k[4:]).all()


def test_a_cache_whose_offsets_pass_32_bits():
    # 40 000 pages of 16 x 8 x 128 bf16 elements: 655 million elements, K alone 1.3 GB; with int8 in two layers past 2^31 bytes
    page, heads, d, pages = 64, 8, 128, 33000
    k, v = (torch.zeros(2, pages, page, heads, d, dtype=torch.int8, device="cuda") for _ in range(2))
    ks, vs = (torch.zeros(2, pages, heads, page, device="cuda") for _ in range(2))
    assert k.numel() > 2 ** 32
    table = T.i32([[pages - 1, 0, pages - 2]])
    cache = B.KvCache(k, v, table, ks, vs)
    x, y = rows_of(130, heads, d, 4)
    st = T.status()
    B.dspark_kv_write(cache, x, y, T.i32([3]), T.i32([0, 130]), layer=1, dev_status=st)
    a, b = torch.empty_like(x), torch.empty_like(y)
    B.dspark_kv_read(cache, T.i32([3]), T.i32([0, 130]), out_k=a, out_v=b, layer=1, dev_status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    for got, src, c, s in ((a, x, k, ks), (b, y, v, vs)):
        q, scale = T.quantised(src, "int8")
        assert torch.equal(got, (q.float() * scale[..., None].float()).bfloat16())
        assert torch.equal(c[1, pages - 1, 3:], q[:61].to(torch.int8)) and torch.equal(c[1, pages - 2, :5], q[125:].to(torch.int8))
        assert int(c[0].count_nonzero()) == 0


@pytest.mark.parametrize("kind", ["bf16", "int8"])
def test_what_the_device_refuses(kind):
    need = [20, 20, 20, 20]
    cache = T.Cache(need, 8, 2, 32, kind)
    cache.table[1, 2] = cache.pages                           # a page that is not there
    cache.table[2, 2] = -5
    k, v = rows_of(16, 2, 32, 1)
    before = cache.snapshot()
    # request 3's rows pass the end of its row of the table; request 0 has a negative number of tokens
    assert write(cache, k, v, T.i32([-1, 18, 18, 22]), T.offsets([4, 4, 4, 4])) == B.DEV_BAD_PAGE
    assert T.same(cache.snapshot(), before)
    a, b, st = read(cache, T.i32([-1, 18, 18, 22]), T.offsets([4, 4, 4, 4]), 16, torch.float32)
    assert st == B.DEV_BAD_PAGE
    assert (a[:4] == 3).all() and (a[12:] == 3).all() and (a[4:12] == 0).all() and (b[4:12] == 0).all()
    # offsets that fall or pass the arrays
    assert write(cache, k, v, T.i32([0, 0, 0, 0]), T.i32([0, 4, 2, 2, 30])) & B.DEV_BAD_OFFSETS
    assert write(cache, k, v, T.i32([0, 0, 0, 0]), T.i32([-4, -2, -1, -1, -1])) & B.DEV_BAD_OFFSETS


@pytest.mark.parametrize("kind,page,heads,d,layers,layout", [
    ("bf16", 16, 8, 128, 3, "nhd"), ("int8", 8, 3, 80, 2, "pair"), ("e4m3", 256, 1, 64, 1, "hnd"), ("int8", 32, 40, 48, 2, "nhd")])
def test_commit_moves_the_path(kind, page, heads, d, layers, layout):
    nodes = [1, 2, 9, 40, 0, 12, 12]
    first = [5, 0, 30, 121, 9, 15, 7]
    paths = [[], [1], [2, 4, 7, 8], [1, 2, 3, 9, 10, 11, 12, 13, 20, 21, 22, 30, 31, 32, 38, 39], [], list(range(1, 12)), [3, 11]]
    need = [f + n for f, n in zip(first, nodes)]
    cache, want = (T.Cache(need, page, heads, d, kind, layers=layers, layout=layout, seed=2) for _ in range(2))
    for layer in range(layers):
        for r in range(len(nodes)):
            if need[r]:
                x = torch.randn(2, need[r], heads, d, generator=T.gen(100 * layer + r), device="cuda")
                for c in (cache, want):
                    c.put(r, range(need[r]), x[0], x[1], layer=layer)
    off = T.offsets(nodes)
    o = off.tolist()
    path = torch.full((o[-1],), -1, dtype=torch.int32, device="cuda")
    for r, p in enumerate(paths):
        path[o[r]: o[r] + len(p)] = T.i32(p)
        for i, node in enumerate(p):
            (a, b), (y, z) = want.slots(r, [first[r] + node]), want.slots(r, [first[r] + 1 + i])
            for c in (want.k, want.v) if kind == "bf16" else (want.k.view(torch.uint8), want.v.view(torch.uint8)):
                c[:, y, z] = c[:, a, b].clone()
            for s in (want.ks, want.vs):
                if s is not None:
                    s[:, y, :, z] = s[:, a, :, b].clone()
    out, st = torch.full((7,), -9, dtype=torch.int32, device="cuda"), T.status()
    B.dspark_kv_commit(cache.handle, T.i32(first), off, T.i32([len(p) for p in paths]), path, out_first=out, dev_status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    assert out.tolist() == [f + (1 + len(p) if n else 0) for f, n, p in zip(first, nodes, paths)]
    assert T.same(cache.snapshot(), want.snapshot())


def test_commit_refuses_what_is_no_path():
    nodes, first = [4] * 6, [3] * 6
    cache = T.Cache([7] * 6, 8, 2, 32, "bf16")
    cache.k.normal_(generator=T.gen(1))
    cache.v.normal_(generator=T.gen(2))
    before = cache.snapshot()
    path = T.i32([0, 1, 0, 0, 2, 2, 0, 0, 3, 1, 0, 0, 1, 4, 0, 0, 1, 2, 3, 0, -1, 2, 0, 0])
    out, st = torch.zeros(6, dtype=torch.int32, device="cuda"), T.status()
    # the root, a node twice, falling, past the nodes, more than there are, negative
    B.dspark_kv_commit(cache.handle, T.i32(first), T.offsets(nodes), T.i32([2, 2, 2, 2, 4, 2]), path, out_first=out, dev_status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == B.DEV_BAD_TREE and out.tolist() == first and T.same(cache.snapshot(), before)
    B.dspark_kv_commit(cache.handle, T.i32(first), T.offsets(nodes), T.i32([-1] * 6), path, out_first=out, dev_status=st)
    torch.cuda.synchronize()
    assert out.tolist() == first and T.same(cache.snapshot(), before)
    cache.table[0, 0] = cache.pages + 7
    st.zero_()
    B.dspark_kv_commit(cache.handle, T.i32(first), T.offsets(nodes), T.i32([1] * 6), T.i32([2, 0, 0, 0] * 6), out_first=out, dev_status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == B.DEV_BAD_PAGE and out.tolist() == [5] * 6


def test_captured_and_on_another_stream():
    cache = T.Cache([80], 16, 2, 64, "int8")
    k, v = rows_of(9, 2, 64, 6)
    first, off, st = T.i32([5]), T.i32([0, 9]), T.status()
    a, b = torch.empty_like(k), torch.empty_like(v)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            B.dspark_kv_write(cache.handle, k, v, first, off, dev_status=st)
            B.dspark_kv_read(cache.handle, first, off, out_k=a, out_v=b, dev_status=st)
    for f in (5, 40, 0):
        first.fill_(f)
        k.copy_(rows_of(9, 2, 64, 60 + f)[0])
        graph.replay()
        torch.cuda.synchronize()
        x, y = cache.values(0, range(f, f + 9))
        assert int(st.item()) == 0 and torch.equal(a, x.float().bfloat16()) and torch.equal(b, y.float().bfloat16())
        q, scale = T.quantised(k, "int8")
        assert torch.equal(x, q * scale[..., None].double())
