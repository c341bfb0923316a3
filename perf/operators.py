"""The vocabulary projection, served in 8 bits and trained without keeping its logits: what is measured.

Three operators and their plain forms: the last norm of a model with the residual's addition and an int8 output
(`norm`), the int8 product with the vocabulary matrix that makes the logit rows the verifier reads (`head`), and the
cross entropy of a hidden state against the vocabulary with its gradients (`loss`: the loss alone, as an evaluation
calls it; `step`: loss and gradients, as a training step does).
"""
import math

import torch

own = False

V_FULL = 129280          # vocabulary of the full-size workloads


def listed():
    return [
        # one decoding request, the latency of a call
        {"name": "norm 1x4096", "op": "norm", "rows": 1, "d": 4096, "dtype": "bf16", "residual": True},
        # an odd width in fp32, the first norm of a stack (nothing to add)
        {"name": "norm 37x1001 fp32", "op": "norm", "rows": 37, "d": 1001, "dtype": "fp32", "residual": False},
        # the verified rows of 512 requests
        {"name": "norm 1482x4096", "op": "norm", "rows": 1482, "d": 4096, "dtype": "bf16", "residual": True},
        # a long prefill
        {"name": "norm 16384x4096", "op": "norm", "rows": 16384, "d": 4096, "dtype": "bf16", "residual": True},
        # one decoding request against the whole vocabulary: the weights' bytes
        {"name": "head 1 row", "op": "head", "rows": 1, "live": 1, "V": V_FULL, "K": 4096, "out": "bf16"},
        # 64 requests with up to 9 rows each, the buffers sized for all of them
        {"name": "head 352 of 576 rows", "op": "head", "rows": 576, "live": 352, "V": V_FULL, "K": 1024, "out": "bf16"},
        # 512 requests, long drafts
        {"name": "head 1482 rows", "op": "head", "rows": 1482, "live": 1482, "V": V_FULL, "K": 4096, "out": "bf16"},
        # an odd vocabulary and width, fp32 rows
        {"name": "head odd fp32", "op": "head", "rows": 77, "live": 77, "V": 10007, "K": 1001, "out": "fp32"},
        # the loss of one block of draft positions (held-out check)
        {"name": "loss 64 rows", "op": "loss", "rows": 64, "V": V_FULL, "d": 1024, "ignored": 0.0},
        # a held-out batch
        {"name": "loss 2048 rows", "op": "loss", "rows": 2048, "V": V_FULL, "d": 2048, "ignored": 0.25},
        # a small training step, odd sizes
        {"name": "step 200 rows odd", "op": "step", "rows": 200, "V": 10007, "d": 500, "ignored": 0.1},
        # a training step with the prompts' positions ignored
        {"name": "step 4096 rows", "op": "step", "rows": 4096, "V": V_FULL, "d": 2048, "ignored": 0.3},
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["norm", "head", "loss", "step"])
    if op == "norm":
        return {"op": op, "rows": _log(rng, 1, 16384), "d": _log(rng, 64, 4096), "dtype": rng.choice(["bf16", "bf16", "fp32"]),
                "residual": rng.random() < 0.75}
    if op == "head":
        rows = _log(rng, 1, 1482)
        live = rows if rng.random() < 0.5 else max(1, int(rows * rng.uniform(0.4, 1.0)))
        return {"op": op, "rows": rows, "live": live, "V": _log(rng, 1000, V_FULL), "K": _log(rng, 64, 4096),
                "out": rng.choice(["bf16", "bf16", "fp32"])}
    return {"op": op, "rows": _log(rng, 1, 2867), "V": _log(rng, 1000, V_FULL), "d": _log(rng, 64, 2048),
            "ignored": rng.choice([0.0, 0.1, 0.3])}


def _ignored(case):
    return min(case["rows"] - 1, int(round(case["ignored"] * case["rows"])))


def work(case):
    if case["op"] == "norm":
        e = 2 if case["dtype"] == "bf16" else 4
        n = case["rows"] * case["d"]
        per = e + 1 + (2 * e if case["residual"] else 0)
        return {"bytes": n * per + case["d"] * e + case["rows"] * 4, "flops": 6 * n}
    if case["op"] == "head":
        n, v, k = case["live"], case["V"], case["K"]
        return {"bytes": v * k + n * k + n * v * (2 if case["out"] == "bf16" else 4) + 4 * (n + v), "flops": 2 * n * v * k}
    n, v, d = case["rows"] - _ignored(case), case["V"], case["d"]
    if case["op"] == "loss":
        return {"bytes": 2 * (v + n) * d + 8 * n, "flops": 2 * n * v * d}
    # logits, their gradient's two products: the logits once, as the loss needs them, and two products of their size
    return {"bytes": 2 * 2 * (v + n) * d + 12 * n, "flops": 6 * n * v * d}


def _pitched(rows, cols, unit, dtype, gen):
    """[rows, cols] normal values with a row pitch of a multiple of `unit` elements, as tensor-map operands have."""
    pitch = -(-cols // unit) * unit
    t = torch.empty(rows, pitch, dtype=dtype, device="cuda")
    if dtype == torch.int8:
        # quantised rows: the largest value of a row at 127, the others spread around zero
        t.copy_((torch.randn(rows, pitch, generator=gen, device="cuda", dtype=torch.float32) * 32).round_().clamp_(-127, 127))
        t[:, 0] = 127
    else:
        t.normal_(generator=gen)
    return t[:, :cols]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op = case["op"]
    s = {"case": case, "status": torch.zeros(1, dtype=torch.int32, device="cuda")}
    if op == "norm":
        dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        n, d = case["rows"], case["d"]
        s["x"] = torch.randn(n, d, generator=g, device="cuda").to(dtype)
        s["residual"] = (torch.randn(n, d, generator=g, device="cuda") * 3).to(dtype) if case["residual"] else None
        s["w"] = (1 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(dtype)
        return s
    if op == "head":
        n, v, k = case["rows"], case["V"], case["K"]
        s["xq"] = _pitched(n, k, 16, torch.int8, g)
        s["wq"] = _pitched(v, k, 16, torch.int8, g)
        s["xs"] = torch.rand(n, generator=g, device="cuda") * 0.02 + 0.01
        s["ws"] = (torch.rand(v, generator=g, device="cuda") + 0.5) * (0.08 / math.sqrt(k))
        s["live"] = torch.tensor([case["live"]], dtype=torch.int32, device="cuda")
        return s
    n, v, d = case["rows"], case["V"], case["d"]
    w = _pitched(v, d, 8, torch.bfloat16, g)
    w.mul_(2.5 / math.sqrt(d))                               # logits of a standard deviation of 2.5
    labels = torch.randint(0, v, (n,), generator=g, device="cuda")
    h = _pitched(n, d, 8, torch.bfloat16, g)
    # a head that has learnt something: the label's logit is 0 to 12 above the others
    lift = torch.rand(n, 1, generator=g, device="cuda") * (12 / 2.5 ** 2)
    h.copy_(h.float() + lift * w[labels].float())
    drop = torch.randperm(n, generator=g, device="cuda")[: _ignored(case)]
    labels[drop] = -1
    s["h"], s["w"], s["labels"] = h, w, labels.to(torch.int32)
    # weights that fall with the position in a block of 16, over the number of rows that count
    at = torch.arange(n, device="cuda") % 16
    s["g"] = torch.exp(-at.float() / 16) / (n - _ignored(case))
    return s


def _norm_own(B, s):
    x = s["x"]
    n, d = x.shape
    q = torch.empty(n, d, dtype=torch.int8, device="cuda")
    scale = torch.empty(n, dtype=torch.float32, device="cuda")
    h = torch.empty_like(x) if s["residual"] is not None else None
    B.dspark_rms_norm_quant(x, s["w"], 1e-6, residual=s["residual"], out_residual=h, out_q=q, out_scale=scale)
    return {"residual": h, "y": q * scale[:, None], "scale": scale}


def _norm_plain(s):
    h = s["x"]
    if s["residual"] is not None:
        h = (h.float() + s["residual"].float()).to(h.dtype)
    t = h.double() * s["w"].double()                         # next to a half, 32 bits choose the other integer
    top = t.abs().amax(1, keepdim=True)
    q = torch.round(t * 127 / top)
    r = torch.rsqrt(h.float().square().mean(1) + 1e-6)
    scale = top[:, 0].float() * r / 127
    return {"residual": h if s["residual"] is not None else None, "y": q.float() * scale[:, None], "scale": scale}


def _head_own(B, s):
    c = s["case"]
    out = torch.empty(c["rows"], c["V"], dtype=torch.bfloat16 if c["out"] == "bf16" else torch.float32, device="cuda")
    B.dspark_lm_head_int8(s["xq"], s["xs"], s["wq"], s["ws"], out_logits=out, n_live=s["live"], dev_status=s["status"])
    return out[: c["live"]]


def _head_plain(s):
    c = s["case"]
    z = (s["xq"][: c["live"]].float() @ s["wq"].float().T) * s["xs"][: c["live"], None] * s["ws"]
    return z.to(torch.bfloat16 if c["out"] == "bf16" else torch.float32)


def _loss_own(B, s, step):
    h, w, labels = s["h"], s["w"], s["labels"]
    n, d = h.shape
    v = w.shape[0]
    loss = torch.empty(n, dtype=torch.float32, device="cuda")
    lse = torch.empty(n, dtype=torch.float32, device="cuda")
    ws = B.workspace(B.dspark_lm_head_loss_workspace_bytes(n, v, d))
    B.dspark_lm_head_loss(h, w, labels, out_loss=loss, out_lse=lse, dev_status=s["status"], workspace=ws)
    if not step:
        return {"loss": loss, "lse": lse}
    dh = torch.empty(n, d, dtype=torch.bfloat16, device="cuda")
    dw = torch.empty(v, d, dtype=torch.bfloat16, device="cuda")
    B.dspark_lm_head_loss_backward(h, w, labels, lse, s["g"], out_grad_hidden=dh, out_grad_weight=dw,
                                   dev_status=s["status"], workspace=ws)
    return {"loss": loss, "dh": dh, "dw": dw}


def _loss_form(s, step, real, out):
    """The loss in the type `real`; gradients in the type `out`."""
    h, w = s["h"].to(real), s["w"].to(real)
    live = s["labels"] >= 0
    at = s["labels"].clamp(min=0).long()[:, None]
    z = h @ w.T
    top = z.amax(1, keepdim=True)
    lse = (z - top).exp().sum(1).log() + top[:, 0]
    loss = torch.where(live, lse - z.gather(1, at)[:, 0], 0)
    if not step:
        return {"loss": loss, "lse": torch.where(live, lse, 0)}
    g = (z - lse[:, None]).exp()
    g.scatter_add_(1, at, torch.full_like(at, -1, dtype=real))
    g *= torch.where(live, s["g"].to(real), 0)[:, None]
    return {"loss": loss, "dh": (g @ w).to(out), "dw": (g.T @ h).to(out)}


def run(state):
    op = state["case"]["op"]
    if own:
        from paper_2607_05147_b200 import binding as B
        if op == "norm":
            return _norm_own(B, state)
        if op == "head":
            return _head_own(B, state)
        return _loss_own(B, state, op == "step")
    if op == "norm":
        return _norm_plain(state)
    if op == "head":
        return _head_plain(state)
    return _loss_form(state, op == "step", torch.float32, torch.bfloat16)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        h = s["x"].double()
        if s["residual"] is not None:
            h = (h + s["residual"].double()).to(s["x"].dtype).double()      # the stored sum is what is normalised
        y = h * s["w"].double() * (h.pow(2).sum(1, keepdim=True) / case["d"] + 1e-6).pow(-0.5)
        scale = y.abs().max(1, keepdim=True).values / 127
        # the integer from the quotient without the norm's factor, which cancels: its rounding must not decide a half
        t = h * s["w"].double()
        q = (t * 127 / t.abs().max(1, keepdim=True).values).round()
        return {"residual": h if s["residual"] is not None else None, "y": q * scale, "scale": scale[:, 0]}
    if case["op"] == "head":
        n = case["live"]
        z = torch.einsum("nk,vk->nv", s["xq"][:n].double(), s["wq"].double())
        return z.mul_(s["xs"][:n, None].double()).mul_(s["ws"].double())
    w, h, n = s["w"].double(), s["h"].double(), case["rows"]
    live = s["labels"] >= 0
    rows = torch.nonzero(live)[:, 0]
    z = torch.einsum("nd,vd->nv", h[rows], w)
    lse = torch.logsumexp(z, 1)
    of_label = z[torch.arange(len(rows), device="cuda"), s["labels"][rows].long()]
    loss, full = torch.zeros(n, dtype=torch.float64, device="cuda"), torch.zeros(n, dtype=torch.float64, device="cuda")
    loss[rows], full[rows] = lse - of_label, lse
    if case["op"] == "loss":
        return {"loss": loss, "lse": full}
    p = z.sub_(lse[:, None]).exp_()
    p[torch.arange(len(rows), device="cuda"), s["labels"][rows].long()] -= 1
    p *= s["g"][rows, None].double()
    dh = torch.zeros_like(h)
    dh[rows] = torch.einsum("nv,vd->nd", p, w)
    return {"loss": loss, "dh": dh, "dw": torch.einsum("nv,nd->vd", p, h[rows])}
