"""Steps of trees over a paged cache for the tests, and their definitions in 64 bits (torch, on the tensors' device)."""
from __future__ import annotations

import math

import torch

from paper_2607_05147_b200 import binding as B

KINDS = {"bf16": torch.bfloat16, "int8": torch.int8, "e4m3": torch.float8_e4m3fn}


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def offsets(nodes):
    off = [0]
    for n in nodes:
        off.append(off[-1] + n)
    return i32(off)


def status():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


def to_e4m3(x):
    """The nearest e4m3 value of |x| <= 448 in 64 bits, ties to even."""
    e = torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(e - 3)
    return torch.round(x / step) * step


def quantised(x, kind):
    """(stored values in 64 bits, scales in fp32) of the head rows in the last dimension."""
    t = x.double()
    top = t.abs().amax(-1, keepdim=True)
    whole = 127 if kind == "int8" else 448
    safe = torch.where(top > 0, top, 1.0)
    y = t * whole / safe
    bad = ~torch.isfinite(top) | torch.isnan(t).any(-1, keepdim=True)
    y = torch.where(bad, 0.0, y)
    q = y.round() if kind == "int8" else to_e4m3(y)
    scale = (top / whole).float()[..., 0]                    # fp32 division by a number may be a product with its inverse
    return q, torch.where(bad[..., 0], torch.nan, scale)


class Cache:
    """A cache of its own with pages in any order; layout: 'nhd' [pages, page, heads, d], 'hnd' [pages, heads, page, d] in
    memory, 'pair' K and V of a page side by side."""

    def __init__(self, need, page, heads, d, kind="bf16", layers=1, layout="nhd", seed=0, spare=2, fill=None):
        g = gen(seed + 1)
        self.page, self.heads, self.d, self.kind, self.layers = page, heads, d, kind, layers
        pages = [-(-t // page) for t in need]
        self.pages = sum(pages) + spare
        order = torch.randperm(self.pages, generator=g, device="cuda").to(torch.int32)
        self.table = torch.full((len(need), max(max(pages), 1)), -1, dtype=torch.int32, device="cuda")
        at = 0
        for r, n in enumerate(pages):
            self.table[r, :n] = order[at: at + n]
            at += n
        t = KINDS[kind]
        if layout == "nhd":
            k, v = (torch.zeros(layers, self.pages, page, heads, d, device="cuda", dtype=t) for _ in range(2))
        elif layout == "hnd":
            k, v = (torch.zeros(layers, self.pages, heads, page, d, device="cuda", dtype=t).transpose(2, 3) for _ in range(2))
        else:
            kv = torch.zeros(layers, self.pages, 2, page, heads, d, device="cuda", dtype=t)
            k, v = kv[:, :, 0], kv[:, :, 1]
        self.k, self.v, self.ks, self.vs = k, v, None, None
        if kind != "bf16":
            self.ks, self.vs = (torch.zeros(layers, self.pages, heads, page, device="cuda") for _ in range(2))
        if fill is not None:
            self.k.view(torch.uint8).fill_(fill) if kind != "bf16" else self.k.fill_(math.nan)
            self.v.view(torch.uint8).fill_(fill) if kind != "bf16" else self.v.fill_(math.nan)
            if kind != "bf16":
                self.ks.fill_(math.nan)
                self.vs.fill_(math.nan)
        self.handle = B.KvCache(self.k, self.v, self.table, self.ks, self.vs)

    def slots(self, r, positions):
        p = torch.as_tensor(positions, device="cuda").long()
        return self.table[r, p // self.page].long(), p % self.page

    def put(self, r, positions, k, v, layer=0):
        """Head rows [n, heads, d] stored as dspark_kv_write would."""
        pg, at = self.slots(r, positions)
        if self.kind == "bf16":
            self.k[layer, pg, at], self.v[layer, pg, at] = k.bfloat16(), v.bfloat16()
            return
        for x, c, s in ((k, self.k, self.ks), (v, self.v, self.vs)):
            q, scale = quantised(x.bfloat16(), self.kind)
            if self.kind == "int8":
                c[layer, pg, at] = q.to(torch.int8)
            else:
                c.view(torch.uint8)[layer, pg, at] = q.to(torch.float32).to(torch.float8_e4m3fn).view(torch.uint8)
            s[layer, pg, :, at] = scale.to(torch.float32)

    def values(self, r, positions, layer=0):
        """(K, V) of the positions in 64 bits, [n, heads, d]."""
        pg, at = self.slots(r, positions)
        out = []
        for c, s in ((self.k, self.ks), (self.v, self.vs)):
            x = c[layer, pg, at].double() if self.kind != "e4m3" else c.view(torch.uint8)[layer, pg, at].view(torch.float8_e4m3fn).double()
            out.append(x if s is None else x * s[layer, pg, :, at].double()[..., None])
        return out

    def snapshot(self):
        raw = [self.k, self.v] if self.kind == "bf16" else [self.k.view(torch.uint8), self.v.view(torch.uint8)]
        return [x.clone().contiguous().view(torch.uint8) for x in raw] + [x.clone().view(torch.int32) for x in (self.ks, self.vs) if x is not None]


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def random_parents(nodes, seed, shape="tree"):
    """Parents of all requests' nodes; shape: 'tree', 'chain', 'star' (all children of the root), 'comb'."""
    g = torch.Generator().manual_seed(seed)
    out = []
    for n in nodes:
        for i in range(n):
            if i == 0:
                out.append(-1)
            elif shape == "chain":
                out.append(i - 1)
            elif shape == "star":
                out.append(0)
            elif shape == "comb":
                out.append((i - 1) // 2 * 2 if i % 2 else i - 2)
            else:
                out.append(int(torch.randint(0, i, (1,), generator=g)))
    return out


def ancestors(parents, row0, i):
    """Node i and its ancestors; parents None: a chain."""
    seen = []
    while i >= 0:
        seen.append(i)
        if i == 0:
            break
        i = i - 1 if parents is None else parents[row0 + i]
    return seen


def attention(cache, q, first, off, parents, scale, layer=0):
    """(out, bound, lse, lse_bound) in 64 bits.

    bound: how far bf16 arithmetic may be off, element by element.  With a = sum w |v|: every weight is rounded to 16 bits
    (2^-8 a), the result to bf16 (2^-8 |out|); scores are fp32 sums of d products, off by at most d 2^-23 of the sum of their
    magnitudes (the tensor cores cut instead of rounding), which moves every weight by twice that; exponentials, the sum of
    the weights and its division: 2^-20 for lengths below 2^17 in runs of 128 added up in fp32.

    8-bit caches: the weights times V's scales are fp16 numbers whose smallest step is 2^-24, half of it lost at most.  They
    are stored with the largest weight of a cache tile times a power of two above its largest scale at 2^7 or more: a position
    is off by at most 2^-25 / 2^7 of that product, which is at most twice the largest weight times the largest scale of the
    positions seen, times the largest stored value (127 or 448)."""
    rows, hq, d = q.shape
    h = cache.heads
    g = hq // h
    out = torch.zeros(rows, hq, d, dtype=torch.float64, device="cuda")
    bound = torch.zeros_like(out)
    lse = torch.zeros(rows, hq, dtype=torch.float64, device="cuda")
    lse_bound = torch.zeros_like(lse)
    for r in range(len(off) - 1):
        for i in range(off[r + 1] - off[r]):
            row = off[r] + i
            pos = list(range(first[r])) + sorted(first[r] + j for j in ancestors(parents, off[r], i))
            k, v = cache.values(r, pos, layer)
            x = q[row].double().view(h, g, d)
            z = torch.einsum("hgd,lhd->hgl", x, k) * scale
            size = torch.einsum("hgd,lhd->hgl", x.abs(), k.abs()).amax(-1) * abs(scale)
            w = torch.softmax(z, -1)
            o = torch.einsum("hgl,lhd->hgd", w, v)
            a = torch.einsum("hgl,lhd->hgd", w, v.abs())
            off_by = (d * 2.0 ** -23 * size + 2.0 ** -20)
            out[row], lse[row] = o.reshape(hq, d), torch.logsumexp(z, -1).reshape(hq)
            tiny = torch.zeros(h, 1, 1, dtype=torch.float64, device="cuda")
            if cache.kind != "bf16":
                pg, at = cache.slots(r, pos)
                scale_top = cache.vs[layer, pg, :, at].double().amax(0)
                tiny = (len(pos) * 2.0 ** -32 * 2 * (127 if cache.kind == "int8" else 448) * scale_top)[:, None, None] * w.amax(-1, keepdim=True)
            bound[row] = (tiny + 2.0 ** -8 * (a + o.abs()) * 1.01 + 2 * off_by[..., None] * a + 1e-37).reshape(hq, d)
            lse_bound[row] = off_by.reshape(hq) + 2.0 ** -22 * (1 + lse[row].abs())
    return out, bound, lse, lse_bound


def run_attention(cache, q, first, off, parents, scale, lse=True, layer=0, out=None, workspace=None):
    out = torch.full_like(q, 7.0) if out is None else out
    l = torch.full(q.shape[:2], 7.0, device="cuda") if lse else None
    st = status()
    n, hq, d = q.shape
    if workspace is None:
        workspace = B.workspace(B.dspark_tree_attention_workspace_bytes(n, hq, cache.heads, d))
        workspace.fill_(255)                                 # any content: NaN
    B.dspark_tree_attention(q, cache.handle, first, off, parents=parents, scale=scale, out=out, out_lse=l, layer=layer, dev_status=st,
                            workspace=workspace)
    torch.cuda.synchronize()
    return out, l, int(st.item())


def verify(p, q, tokens, parents, off, u, u_last):
    """The walk and the draw in 64 bits on the host: (accepted, tokens, path) as lists."""
    R = len(off) - 1
    acc, out, path = [0] * R, [-1] * off[-1], [-1] * off[-1]
    for r in range(R):
        b, n, at = off[r], off[r + 1] - off[r], 0
        while True:
            pr = p[b + at].double()
            qr = q[b + at].double() if q is not None else None
            left, z, nxt = pr.clone(), 1.0, None
            for c in range(1, n):
                if parents[b + c] != at:
                    continue
                x = tokens[b + c]
                qx = 1.0 if qr is None else float(qr[x])
                if u[b + c] * qx * z < float(left[x]):
                    nxt = c
                    break
                if qr is None:
                    z -= float(left[x])
                    left[x] = 0
                else:
                    left = (left - z * qr).clamp(min=0)
                    z = float(left.sum())
            if nxt is None:
                break
            path[b + acc[r]], out[b + acc[r]] = nxt, tokens[b + nxt]
            acc[r] += 1
            at = nxt
        if float(left.sum()) == 0:
            left = pr
        run = left.cumsum(0)
        out[b + acc[r]] = int(torch.nonzero(run > u_last[r] * run[-1])[0])
    return acc, out, path
