"""A step of speculative decoding with trees of drafted tokens over a paged cache: what is measured.

Four operators and their plain forms: K and V rows of a step written to a paged cache in 8 or 16 bits and read back
(`cache`), attention of the drafted nodes over that cache (`attend`), verification of a drafted tree against the target's
probabilities from given random numbers (`verify`), and the accepted path's rows moved together in the cache of all layers
(`commit`).

Rows are ragged: request r owns the rows [row_offsets[r], row_offsets[r + 1]), one per node of its tree; node 0 is the
root (the last token that is certain), a node's parent has a smaller index.  first[r] tokens are in the cache before them;
row i's K and V are at position first[r] + i.
"""
import math

import torch

own = False

V_FULL = 129280          # vocabulary of the full-size workloads


def listed():
    return [
        # one request decoding one token, the latency of a call
        {"name": "attend 1 request 1 token", "op": "attend", "R": 1, "prefix": 700, "nodes": 1, "tree": False, "heads": 8, "group": 4,
         "d": 128, "page": 64, "cache": "bf16"},
        # 64 requests verifying trees of 16 nodes
        {"name": "attend 64 trees of 16", "op": "attend", "R": 64, "prefix": 4096, "nodes": 16, "tree": True, "heads": 8, "group": 4,
         "d": 128, "page": 64, "cache": "bf16"},
        # 128 requests decoding one token over an int8 cache
        {"name": "attend 128x1 int8", "op": "attend", "R": 128, "prefix": 8192, "nodes": 1, "tree": False, "heads": 8, "group": 8,
         "d": 128, "page": 128, "cache": "int8"},
        # one long context, a large tree: more rows than a tile, the cache in e4m3
        {"name": "attend 131072 e4m3, 64 nodes", "op": "attend", "R": 1, "prefix": 131072, "nodes": 64, "tree": True, "heads": 8,
         "group": 4, "d": 128, "page": 64, "cache": "e4m3"},
        # drafted chains of uneven lengths, an odd group and width, small pages
        {"name": "attend 37 chains, odd", "op": "attend", "R": 37, "prefix": 1500, "nodes": 11, "tree": False, "heads": 3, "group": 5,
         "d": 80, "page": 16, "cache": "bf16"},
        # the rows of one request's drafted block
        {"name": "cache 1 block int8", "op": "cache", "R": 1, "prefix": 700, "nodes": 8, "heads": 8, "d": 128, "page": 64, "cache": "int8",
         "out": "bf16"},
        # the drafted blocks of 64 requests, odd width and pages, read back in fp32
        {"name": "cache 64 blocks e4m3 odd", "op": "cache", "R": 64, "prefix": 1000, "nodes": 9, "heads": 5, "d": 80, "page": 16,
         "cache": "e4m3", "out": "fp32"},
        # prompts being written
        {"name": "cache 16 prompts int8", "op": "cache", "R": 16, "prefix": 0, "nodes": 1024, "heads": 8, "d": 128, "page": 64,
         "cache": "int8", "out": "bf16"},
        # one request's accepted path, a small model
        {"name": "commit 1 request", "op": "commit", "R": 1, "prefix": 700, "nodes": 16, "layers": 4, "heads": 8, "d": 128, "page": 64},
        # 64 requests, the layers of a whole model
        {"name": "commit 64 requests 32 layers", "op": "commit", "R": 64, "prefix": 500, "nodes": 32, "layers": 32, "heads": 8, "d": 128,
         "page": 64},
        # one request's tree against the whole vocabulary
        {"name": "verify 1 tree of 16", "op": "verify", "R": 1, "nodes": 16, "V": V_FULL, "draft": True},
        # a batch of trees
        {"name": "verify 128 trees of 32", "op": "verify", "R": 128, "nodes": 32, "V": V_FULL, "draft": True},
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["attend", "attend", "cache", "commit", "verify"])
    if op == "attend":
        R, heads, group = _log(rng, 1, 128), rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 2, 4, 5, 7, 8, 16])
        d = rng.choice([64, 80, 96, 128, 128])
        tree = rng.random() < 0.6
        nodes = _log(rng, 1, 64) if tree else _log(rng, 1, 128)
        # the cache's tokens of all requests, and the scores, within those of the listed cases
        most = min(131072, 1 << 20, 8 * (1 << 20) // (R * heads), (1 << 28) // (R * heads * group * nodes))
        return {"op": op, "R": R, "prefix": _log(rng, 1, max(2, most)), "nodes": nodes, "tree": tree, "heads": heads, "group": group,
                "d": d, "page": rng.choice([8, 16, 32, 64, 128, 256]), "cache": rng.choice(["bf16", "int8", "e4m3"])}
    if op == "cache":
        R = _log(rng, 1, 128)
        return {"op": op, "R": R, "prefix": rng.choice([0, _log(rng, 1, 4096)]), "nodes": _log(rng, 1, max(2, 16384 // R)),
                "heads": rng.choice([1, 2, 3, 5, 8]), "d": rng.choice([64, 80, 96, 128]), "page": rng.choice([8, 16, 32, 64, 128]),
                "cache": rng.choice(["bf16", "int8", "e4m3"]), "out": rng.choice(["bf16", "fp32"])}
    if op == "commit":
        return {"op": op, "R": _log(rng, 1, 64), "prefix": _log(rng, 1, 1000), "nodes": _log(rng, 2, 64), "layers": _log(rng, 1, 32),
                "heads": rng.choice([1, 2, 4, 8]), "d": rng.choice([64, 80, 128]), "page": rng.choice([16, 32, 64])}
    return {"op": op, "R": _log(rng, 1, 128), "nodes": _log(rng, 1, 32), "V": _log(rng, 1000, V_FULL), "draft": rng.random() < 0.7}


_BYTES = {"bf16": 2, "int8": 1, "e4m3": 1, "fp32": 4}


def _lengths(case):
    """(first, nodes) of every request: around the case's numbers, the same for every seed."""
    R = case["R"]
    p = case.get("prefix", 0)
    first = [p if R == 1 else p // 2 + (p + 1) * r // R for r in range(R)]
    if case["op"] == "verify" or case.get("tree") or case["op"] == "commit":
        nodes = [case["nodes"]] * R
    else:
        nodes = [max(1, case["nodes"] - (r * 7) % (case["nodes"] // 2 + 1)) for r in range(R)]
    return first, nodes


def work(case):
    first, nodes = _lengths(case)
    rows = sum(nodes)
    if case["op"] == "attend":
        d, h, g = case["d"], case["heads"], case["group"]
        per = 2 * d * _BYTES[case["cache"]] + (0 if case["cache"] == "bf16" else 8)
        tokens = sum(f + n for f, n in zip(first, nodes))
        return {"bytes": tokens * h * per + 2 * rows * h * g * d * 2,
                "flops": 4 * d * h * g * sum((f + (n + 1) / 2 if not case["tree"] else f + min(n, 6)) * n for f, n in zip(first, nodes))}
    if case["op"] == "cache":
        n = rows * case["heads"]
        scales = 0 if case["cache"] == "bf16" else 16
        return {"bytes": n * (2 * case["d"] * (2 + 2 * _BYTES[case["cache"]] + _BYTES[case["out"]]) + 2 * scales), "flops": 4 * n * case["d"]}
    if case["op"] == "commit":
        moved = sum(_accepted(case, r) for r in range(case["R"]))
        return {"bytes": max(1, moved) * case["layers"] * case["heads"] * case["d"] * 2 * 2 * 2, "flops": 0}
    return {"bytes": case["R"] * case["V"] * 4 * (2 if case["draft"] else 1), "flops": case["R"] * case["V"] * 3}


def _accepted(case, r):
    """Length of request r's accepted path."""
    return min((case["nodes"] - 1) // 3, 1 + (r * 5) % 7)


def _ragged(case):
    first, nodes = _lengths(case)
    off = torch.zeros(len(nodes) + 1, dtype=torch.int64)
    off[1:] = torch.tensor(nodes).cumsum(0)
    return torch.tensor(first, dtype=torch.int32, device="cuda"), off.to(torch.int32).cuda(), int(off[-1])


def _parents(case, g):
    """Trees as drafters grow them: a node's parent is one of the nodes before it, near ones of a level more often."""
    n = case["nodes"]
    i = torch.arange(n, device="cuda")
    u = torch.rand(case["R"], n, generator=g, device="cuda")
    p = ((i - 1).clamp(min=0) * (0.25 + 0.75 * u)).long().clamp(max=n)
    p = torch.minimum(p, (i - 1).clamp(min=0))
    p[:, 0] = -1
    return p.to(torch.int32).reshape(-1)


def _pages(case, first, nodes, g, extra=0):
    """A block table over pages in any order."""
    ps = case["page"]
    need = [-(-(f + n) // ps) for f, n in zip(first, nodes)]
    width = max(need) + extra
    total = sum(need) + 3
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    table = torch.zeros(len(need), width, dtype=torch.int32, device="cuda")
    at = torch.arange(width, device="cuda")[None] + torch.tensor([sum(need[:r]) for r in range(len(need))], device="cuda")[:, None]
    table.copy_(order[at.clamp(max=total - 1)])
    return table, total


def _to_e4m3(x):
    """The nearest e4m3 value in the type of x, ties to even; |x| <= 448."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(e - 3)
    return torch.round(x / step) * step


def _quantised(x, kind):
    """(8-bit values, scales) of rows in the last dimension, fp32."""
    top = x.float().abs().amax(-1, keepdim=True)
    if kind == "int8":
        return torch.round(x.float() * 127 / top).to(torch.int8), top[..., 0] / 127
    return (x.float() * 448 / top).to(torch.float8_e4m3fn), top[..., 0] / 448


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op = case["op"]
    s = {"case": case, "status": torch.zeros(1, dtype=torch.int32, device="cuda")}
    if op == "verify":
        R, n, V = case["R"], case["nodes"], case["V"]
        s["parents"] = _parents(case, g)
        s["off"] = torch.arange(R + 1, dtype=torch.int32, device="cuda") * n
        # target rows: noise with a few likely tokens; the drafter's rows are near them
        z = torch.randn(R * n, V, generator=g, device="cuda") * 2
        like = torch.randint(0, V, (R * n, 16), generator=g, device="cuda")
        z.scatter_add_(1, like, (11 - 1.5 * torch.arange(16, device="cuda").float()).expand(R * n, 16).contiguous())
        s["p"] = torch.softmax(z, 1)
        z.add_(torch.randn(R * n, V, generator=g, device="cuda") * 0.7)
        q = torch.softmax(z, 1)
        del z
        at = s["parents"].view(R, n).clamp(min=0).long() + torch.arange(R, device="cuda")[:, None] * n
        tokens = torch.empty(R * n, dtype=torch.int64, device="cuda")
        for k in range(0, R * n, 1024):                      # a child is drawn from its parent's row
            row = q[at.view(-1)[k: k + 1024]]
            tokens[k: k + 1024] = (row / torch.empty_like(row).exponential_(generator=g)).argmax(1)
        s["tokens"] = tokens.to(torch.int32)
        s["q"] = q if case["draft"] else None
        s["u"] = torch.rand(R * n, generator=g, device="cuda")
        s["u_last"] = torch.rand(R, generator=g, device="cuda")
        s["accepted"] = torch.empty(R, dtype=torch.int32, device="cuda")
        s["out_tokens"], s["path"] = torch.empty(R * n, dtype=torch.int32, device="cuda"), torch.empty(R * n, dtype=torch.int32, device="cuda")
        return s
    first, nodes = _lengths(case)
    s["first"], s["off"], rows = _ragged(case)
    h, d, ps = case["heads"], case["d"], case["page"]
    s["table"], pages = _pages(case, first, nodes, g)
    if op == "commit":
        s["k"] = torch.empty(case["layers"], pages, ps, h, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
        s["v"] = torch.empty(case["layers"], pages, ps, h, d, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
        # paths of trees in the order of their levels: accepted nodes stand behind the places they go to, so that a second
        # call moves the same rows
        n, R = case["nodes"], case["R"]
        acc = torch.tensor([_accepted(case, r) for r in range(R)], device="cuda")
        far = torch.rand(R, n, generator=g, device="cuda")
        far[torch.arange(n, device="cuda")[None] <= acc[:, None]] = 2.0        # node 0 and the places 1 .. accepted
        pick = far.argsort(1)
        order = torch.where(torch.arange(n, device="cuda")[None] < acc[:, None], pick, n).sort(1).values
        s["path"] = torch.where(order < n, order, -1).to(torch.int32).reshape(-1)
        s["accepted"] = acc.to(torch.int32)
        s["out_first"] = torch.empty(R, dtype=torch.int32, device="cuda")
        return s
    if op == "cache":
        x = torch.randn(rows, 2, h, d, generator=g, device="cuda") * (0.2 + 3 * torch.rand(rows, 2, h, 1, generator=g, device="cuda"))
        s["kv"] = x.bfloat16()                                # K and V as one projection leaves them
        kind = {"bf16": torch.bfloat16, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}[case["cache"]]
        s["k"], s["v"] = (torch.zeros(pages, ps, h, d, dtype=kind, device="cuda") for _ in range(2))
        if case["cache"] != "bf16":
            s["ks"], s["vs"] = (torch.zeros(pages, h, ps, device="cuda") for _ in range(2))
        out = torch.bfloat16 if case["out"] == "bf16" else torch.float32
        s["out_k"], s["out_v"] = (torch.empty(rows, h, d, dtype=out, device="cuda") for _ in range(2))
        return s
    # attention: a first token that takes much of the weight, values with a mean
    way = torch.randn(h, 1, d, generator=g, device="cuda")
    s["q"] = (1.5 * torch.randn(rows, h, case["group"], d, generator=g, device="cuda") + 0.7 * way).bfloat16().view(rows, -1, d)
    k = torch.randn(pages, ps, h, d, generator=g, device="cuda").bfloat16()
    v = (torch.randn(pages, ps, h, d, generator=g, device="cuda") + 0.3 * way[:, 0]).bfloat16()
    k[s["table"][:, 0].long(), 0] += way[:, 0].bfloat16()
    if case["cache"] == "bf16":
        s["k"], s["v"] = k, v
    else:
        s["k"], ks = _quantised(k, case["cache"])
        s["v"], vs = _quantised(v, case["cache"])
        s["ks"], s["vs"] = ks.transpose(1, 2).contiguous(), vs.transpose(1, 2).contiguous()
    s["parents"] = _parents(case, g) if case["tree"] else None
    s["scale"] = 1 / math.sqrt(d)
    s["out"] = torch.empty_like(s["q"])
    return s


def _handle(B, s):
    """The cache's handle and the workspace, made once as a program does."""
    if "handle" not in s:
        s["handle"] = B.KvCache(s["k"], s["v"], s["table"], s.get("ks"), s.get("vs"))
        if s["case"]["op"] == "attend":
            n, hq, d = s["q"].shape
            s["workspace"] = B.workspace(B.dspark_tree_attention_workspace_bytes(n, hq, s["case"]["heads"], d))
    return s["handle"]


def _own(s):
    from paper_2607_05147_b200 import binding as B
    op = s["case"]["op"]
    if op == "verify":
        B.dspark_verify_tree(s["p"], s["q"], s["tokens"], s["parents"], s["off"], s["u"], s["u_last"], accepted_len=s["accepted"],
                             out_tokens=s["out_tokens"], out_path=s["path"], dev_status=s["status"])
        return {"accepted": s["accepted"], "tokens": s["out_tokens"], "path": s["path"]}
    cache = _handle(B, s)
    if op == "attend":
        B.dspark_tree_attention(s["q"], cache, s["first"], s["off"], parents=s["parents"], scale=s["scale"], out=s["out"],
                                dev_status=s["status"], workspace=s["workspace"])
        return s["out"]
    if op == "cache":
        B.dspark_kv_write(cache, s["kv"][:, 0], s["kv"][:, 1], s["first"], s["off"], dev_status=s["status"])
        B.dspark_kv_read(cache, s["first"], s["off"], out_k=s["out_k"], out_v=s["out_v"], dev_status=s["status"])
        return {"k": s["out_k"], "v": s["out_v"]}
    B.dspark_kv_commit(cache, s["first"], s["off"], s["accepted"], s["path"], out_first=s["out_first"], dev_status=s["status"])
    return {"k": s["k"], "v": s["v"], "first": s["out_first"]}


def _padded(s):
    """(request, node) of every row."""
    off = s["off"].long()
    rows = s["q"].shape[0]
    row = torch.arange(rows, device="cuda")
    req = torch.searchsorted(off, row, right=True) - 1
    return req, row - off[req]


def _attend_plain(s):
    c = s["case"]
    R, h, g, d, ps = c["R"], c["heads"], c["group"], c["d"], c["page"]
    first, nodes = _lengths(c)
    N, L = max(nodes), max(f + n for f, n in zip(first, nodes))
    req, node = _padded(s)
    q = torch.zeros(R, N, h, g, d, device="cuda")
    q[req, node] = s["q"].float().view(-1, h, g, d)
    t = torch.arange(L, device="cuda")
    page, at = s["table"].long()[:, t // ps], t % ps
    k, v = s["k"][page, at].float(), s["v"][page, at].float()
    if "ks" in s:
        k *= s["ks"][page, :, at][..., None]
        v *= s["vs"][page, :, at][..., None]
    z = torch.einsum("rnhgd,rlhd->rhgnl", q, k)
    del k
    if s["parents"] is None:
        seen = torch.ones(N, N, device="cuda").tril().bool().expand(R, N, N)
    else:
        step = torch.eye(N, device="cuda", dtype=torch.float64).repeat(R, 1, 1)
        i = torch.arange(1, N, device="cuda")
        step[:, i] += torch.nn.functional.one_hot(s["parents"].view(R, N)[:, 1:].long(), N)
        seen = torch.linalg.matrix_power(step, N) > 0
    f = s["first"].long()
    j = t[None] - f[:, None]
    allowed = torch.gather(seen, 2, j.clamp(0, N - 1)[:, None].expand(R, N, L)) & (j < N)[:, None]
    allowed |= (j < 0)[:, None]
    z.mul_(s["scale"]).masked_fill_(~allowed[:, None, None], -math.inf)
    z.sub_(z.amax(-1, keepdim=True)).exp_()
    z.div_(z.sum(-1, keepdim=True))
    # positions that no row sees have no value
    v.masked_fill_((j >= N)[:, :, None, None], 0)
    o = torch.einsum("rhgnl,rlhd->rnhgd", z, v)
    return o[req, node].reshape(-1, h * g, d).to(torch.bfloat16)


def _verify_plain(s, real=torch.float64):
    """In 64 bits: sums next to a border decide.  A node is looked at when the walk stands at its parent; nodes ascend."""
    c = s["case"]
    R, n, V = c["R"], c["nodes"], c["V"]
    base = torch.arange(R, device="cuda") * n
    parents, tokens, u = s["parents"].view(R, n), s["tokens"].view(R, n).long(), s["u"].view(R, n).to(real)
    at = torch.zeros(R, dtype=torch.int64, device="cuda")
    length = torch.zeros(R, dtype=torch.int64, device="cuda")
    path = torch.full((R, n), -1, dtype=torch.int64, device="cuda")
    out = torch.full((R, n), -1, dtype=torch.int64, device="cuda")
    share = torch.zeros(R, dtype=real, device="cuda")         # A: how much of q has been taken off
    total = torch.ones(R, dtype=real, device="cuda")          # Z: what is left, 1 at a node's first child
    gone = torch.zeros(R, V, dtype=torch.bool, device="cuda") if s["q"] is None else None
    every = torch.arange(R, device="cuda")
    for i in range(1, n):
        x, here = tokens[:, i], parents[:, i] == at
        row = base + at
        p = s["p"][row, x].to(real)
        if s["q"] is None:
            p = p * ~gone[every, x]
            yes = here & (u[:, i] * total < p)
            no = here & ~yes
            total = torch.where(no, total - p, total)
            gone[every, x] |= no
        else:
            q = s["q"][row, x].to(real)
            yes = here & (u[:, i] * q * total < (p - share * q).clamp(min=0))
            no = here & ~yes
            share = torch.where(no, share + total, share)
            left = (s["p"][row].to(real) - share[:, None] * s["q"][row]).clamp_(min=0).sum(1)
            total = torch.where(no, left, total)
        path[every, length] = torch.where(yes, i, path[every, length])
        out[every, length] = torch.where(yes, x, out[every, length])
        length += yes
        at = torch.where(yes, i, at)
        share, total = torch.where(yes, 0, share), torch.where(yes, 1, total)
        if gone is not None:
            gone &= ~yes[:, None]
    row = base + at
    r = s["p"][row].to(real)
    if s["q"] is not None:
        r = (r - share[:, None] * s["q"][row]).clamp_(min=0)
    else:
        r = r * ~gone
    run = r.cumsum(1)
    last = (run > s["u_last"].to(real)[:, None] * run[:, -1:]).to(torch.uint8).argmax(1)
    out[every, length] = last
    return {"accepted": length.to(torch.int32), "tokens": out.to(torch.int32).view(-1), "path": path.to(torch.int32).view(-1)}


def _slots(s, position, req):
    ps = s["case"]["page"]
    return s["table"][req, position // ps].long(), position % ps


def _cache_plain(s):
    c = s["case"]
    out = torch.bfloat16 if c["out"] == "bf16" else torch.float32
    off = s["off"].long()
    row = torch.arange(s["kv"].shape[0], device="cuda")
    req = torch.searchsorted(off, row, right=True) - 1
    page, at = _slots(s, s["first"].long()[req] + row - off[req], req)

    def through(x, cache, scales):
        if c["cache"] == "bf16":
            cache[page, at] = x
            return cache[page, at].to(out)
        q, scale = _quantised(x, c["cache"])
        cache.view(torch.uint8)[page, at] = q.view(torch.uint8)
        scales[page, :, at] = scale
        return (cache.view(torch.uint8)[page, at].view(cache.dtype).float() * scales[page, :, at][..., None]).to(out)
    return {"k": through(s["kv"][:, 0], s["k"], s.get("ks")), "v": through(s["kv"][:, 1], s["v"], s.get("vs"))}


def _commit_plain(s):
    c = s["case"]
    R, n = c["R"], c["nodes"]
    path = s["path"].view(R, n).long()
    i = torch.arange(n - 1, device="cuda").expand(R, n - 1)
    req = torch.arange(R, device="cuda")[:, None].expand(R, n - 1)
    live = i < s["accepted"][:, None]
    f = s["first"].long()[:, None]
    to = f + 1 + i
    source = torch.where(live, f + path[:, : n - 1], to)      # the others stay where they are
    (a, b), (y, z) = _slots(s, source, req), _slots(s, to, req)
    s["k"][:, y, z] = s["k"][:, a, b]
    s["v"][:, y, z] = s["v"][:, a, b]
    return {"k": s["k"], "v": s["v"], "first": s["first"] + 1 + s["accepted"]}


def run(state):
    if own:
        return _own(state)
    return {"attend": _attend_plain, "verify": _verify_plain, "cache": _cache_plain, "commit": _commit_plain}[state["case"]["op"]](state)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    off = s["off"].tolist()
    if op == "attend":
        first, par = s["first"].tolist(), None if s["parents"] is None else s["parents"].tolist()
        h, g, d, ps = case["heads"], case["group"], case["d"], case["page"]
        out = torch.zeros(off[-1], h * g, d, dtype=torch.float64, device="cuda")
        for r in range(case["R"]):
            f, n = first[r], off[r + 1] - off[r]
            t = torch.arange(f + n, device="cuda")
            page = s["table"][r, t // ps].long()
            k, v = s["k"][page, t % ps].double(), s["v"][page, t % ps].double()
            if "ks" in s:
                k, v = k * s["ks"][page, :, t % ps][..., None].double(), v * s["vs"][page, :, t % ps][..., None].double()
            hidden = torch.zeros(n, f + n, dtype=torch.bool)
            hidden[:, f:] = True
            for i in range(n):
                j = i
                while j >= 0:
                    hidden[i, f + j] = False
                    j = j - 1 if par is None else par[off[r] + j]
            hidden = hidden.cuda()
            for a in range(h):
                q = s["q"][off[r]: off[r + 1], a * g: (a + 1) * g].double()
                z = (torch.tensordot(q, k[:, a], dims=([2], [1])) * s["scale"]).masked_fill(hidden[:, None], -math.inf)
                w = torch.softmax(z, -1)
                out[off[r]: off[r + 1], a * g: (a + 1) * g] = torch.tensordot(w, v[:, a], dims=([2], [0]))
        return out
    if op == "cache":
        def back(x):
            if case["cache"] == "bf16":
                return x.double()
            top, whole = x.double().abs().amax(-1, keepdim=True), 127 if case["cache"] == "int8" else 448
            y = x.double() * whole / top
            return (y.round() if case["cache"] == "int8" else _to_e4m3(y)) * top / whole
        return {"k": back(s["kv"][:, 0]), "v": back(s["kv"][:, 1])}
    if op == "commit":
        first, acc, path, table, ps = s["first"].tolist(), s["accepted"].tolist(), s["path"].tolist(), s["table"].tolist(), case["page"]
        for x in (s["k"], s["v"]):
            for r in range(case["R"]):
                for i in range(acc[r]):
                    a, b = first[r] + path[off[r] + i], first[r] + 1 + i
                    x[:, table[r][b // ps], b % ps] = x[:, table[r][a // ps], a % ps]
        return {"k": s["k"], "v": s["v"], "first": torch.tensor([f + 1 + a for f, a in zip(first, acc)], dtype=torch.int32)}
    par, tok, u, last = s["parents"].tolist(), s["tokens"].tolist(), s["u"].tolist(), s["u_last"].tolist()
    R, n = case["R"], case["nodes"]
    length, out, path = [0] * R, [-1] * (R * n), [-1] * (R * n)
    for r in range(R):
        b, at = r * n, 0
        while True:
            p = s["p"][b + at].double()
            q = s["q"][b + at].double() if s["q"] is not None else None
            left, z, nxt = p, 1.0, None
            for c in (i for i in range(1, n) if par[b + i] == at):
                x = tok[b + c]
                if u[b + c] * z * (1.0 if q is None else float(q[x])) < float(left[x]):
                    nxt = c
                    break
                if q is None:
                    z -= float(left[x])
                    left = left.clone()
                    left[x] = 0
                else:
                    left = (left - z * q).clamp(min=0)
                    z = float(left.sum())
            if nxt is None:
                break
            path[b + length[r]], out[b + length[r]] = nxt, tok[b + nxt]
            length[r] += 1
            at = nxt
        sums = left.cumsum(0)
        out[b + length[r]] = int(torch.nonzero(sums > last[r] * sums[-1])[0])
    return {"accepted": torch.tensor(length, dtype=torch.int32), "tokens": torch.tensor(out, dtype=torch.int32),
            "path": torch.tensor(path, dtype=torch.int32)}
