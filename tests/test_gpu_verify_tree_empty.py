"""Verification of a batch with requests that have no rows: nothing to do, no error, as in the step's other calls."""
import pytest
import torch

from paper_2607_05147_b200 import binding as B
import tree_helpers as T
from test_gpu_verify_tree import batch, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("draft", [True, False])
def test_requests_without_rows(draft):
    nodes = [0, 5, 0, 0, 9, 0]
    p, q, tokens, parents, off, u, u_last = batch(nodes, 200, 4)
    acc, out, path, st = run(p, q if draft else None, tokens, parents, off, u, u_last)
    live = [r for r, n in enumerate(nodes) if n]
    want = T.verify(p, q if draft else None, tokens.tolist(), parents, [0, 5, 14], u.tolist(), u_last[live].tolist())
    assert st == 0
    assert [acc[r] for r in live] == want[0] and out == want[1] and path == want[2]
    assert all(acc[r] == 0 for r, n in enumerate(nodes) if n == 0)


def test_a_whole_step_with_an_idle_slot():
    nodes, first, heads, d, V = [4, 0, 2], [20, 33, 0], 2, 64, 40
    g = T.gen(1)
    cache = T.Cache([f + 4 for f in first], 16, heads, d, "int8")
    for r, f in enumerate(first):
        if f:
            cache.put(r, range(f), *torch.randn(2, f, heads, d, generator=g, device="cuda"))
    off, fst, st = T.offsets(nodes), T.i32(first), T.status()
    parents = T.random_parents(nodes, 1)
    k, v = torch.randn(2, 6, heads, d, generator=g, device="cuda").bfloat16()
    q = torch.randn(6, heads, d, generator=g, device="cuda").bfloat16()
    out = torch.zeros_like(q)
    ws = B.workspace(B.dspark_tree_attention_workspace_bytes(6, heads, heads, d))
    p, dr = (torch.softmax(torch.randn(6, V, generator=g, device="cuda"), 1) for _ in range(2))
    tokens = torch.randint(0, V, (6,), generator=g, device="cuda", dtype=torch.int32)
    u, u_last = torch.rand(6, generator=g, device="cuda"), torch.rand(3, generator=g, device="cuda")
    acc, tok, path, nxt = (torch.zeros(m, dtype=torch.int32, device="cuda") for m in (3, 6, 6, 3))
    B.dspark_kv_write(cache.handle, k, v, fst, off, dev_status=st)
    B.dspark_tree_attention(q, cache.handle, fst, off, parents=T.i32(parents), scale=0.1, out=out, dev_status=st, workspace=ws)
    B.dspark_verify_tree(p, dr, tokens, T.i32(parents), off, u, u_last, accepted_len=acc, out_tokens=tok, out_path=path, dev_status=st)
    B.dspark_kv_commit(cache.handle, fst, off, acc, path, out_first=nxt, dev_status=st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    a = acc.tolist()
    assert a[1] == 0 and nxt.tolist() == [first[0] + 1 + a[0], first[1], first[2] + 1 + a[2]]
