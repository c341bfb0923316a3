"""The vocabulary projection as it is used: norm -> int8 projection -> verifier on the rows that the scheduler asked for,
eagerly, captured in a CUDA graph and on other streams; a few training steps on the loss and its gradients."""
import numpy as np
import pytest
import torch

import oracle
from paper_2607_05147_b200 import binding as B
from paper_2607_05147_b200 import workloads as W

pytestmark = pytest.mark.gpu


class Serving:
    """A target model's last layers over a batch of R requests with at most gamma drafted tokens each."""

    def __init__(self, R=24, gamma=6, d=320, V=5000, seed=3):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.R, self.gamma, self.d, self.V, self.cap = R, gamma, d, V, R * (gamma + 1)
        self.weight = (torch.randn(V, d, generator=g, device="cuda") / d ** 0.5).bfloat16()
        self.norm_w = (1 + 0.1 * torch.randn(d, generator=g, device="cuda")).bfloat16()
        self.wq = torch.empty(V, d, dtype=torch.int8, device="cuda")
        self.ws = torch.empty(V, device="cuda")
        B.dspark_lm_head_quantize(self.weight, self.wq, self.ws)
        self.x = torch.empty(self.cap, d, dtype=torch.bfloat16, device="cuda")
        self.res = torch.empty_like(self.x)
        self.lengths = torch.empty(R, dtype=torch.int32, device="cuda")
        self.off = torch.empty(R + 1, dtype=torch.int32, device="cuda")
        self.h = torch.empty_like(self.x)
        self.q = torch.empty(self.cap, d, dtype=torch.int8, device="cuda")
        self.scale = torch.empty(self.cap, device="cuda")
        self.logits = torch.empty(self.cap, V, dtype=torch.bfloat16, device="cuda")
        self.tokens = torch.empty(self.cap, dtype=torch.int32, device="cuda")
        self.acc = torch.empty(R, dtype=torch.int32, device="cuda")
        self.out = torch.empty(self.cap, dtype=torch.int32, device="cuda")
        self.st = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.work = B.workspace(B.dspark_verify_workspace_bytes(R, self.cap, V))

    def fill(self, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.x.copy_(torch.randn(self.cap, self.d, generator=g, device="cuda"))
        self.res.copy_(torch.randn(self.cap, self.d, generator=g, device="cuda"))
        self.lengths.copy_(torch.randint(0, self.gamma + 1, (self.R,), generator=g, device="cuda"))
        self.tokens.copy_(torch.randint(0, self.V, (self.cap,), generator=g, device="cuda"))

    def step(self):
        B.dspark_build_offsets(self.lengths, self.off)
        n = self.off[self.R:]
        B.dspark_rms_norm_quant(self.x, self.norm_w, 1e-6, residual=self.res, out_residual=self.h, out_q=self.q, out_scale=self.scale, n_live=n)
        B.dspark_lm_head_int8(self.q, self.scale, self.wq, self.ws, out_logits=self.logits, n_live=n, dev_status=self.st)
        B.dspark_verify_greedy(self.logits, self.off, self.tokens, accepted_len=self.acc, out_tokens=self.out, dev_status=self.st,
                               workspace=self.work)

    def reference_logits(self, n):
        h = (self.x[:n].double() + self.res[:n].double()).bfloat16()
        t = h.double() * self.norm_w.double()
        top = t.abs().amax(1, keepdim=True)
        q = torch.round(t * 127 / top)
        scale = top[:, 0] / torch.sqrt(h.double().square().mean(1) + 1e-6) / 127
        wtop = self.weight.double().abs().amax(1, keepdim=True)
        wq = torch.round(self.weight.double() * 127 / wtop)
        return (q @ wq.T) * scale[:, None] * (wtop[:, 0] / 127)

    def check(self):
        torch.cuda.synchronize()
        assert int(self.st) == 0
        n = int(self.off[self.R])
        want = self.reference_logits(n)
        # the integers are exact; the scales are 48 x 2^-24 and 2^-23 off at most, three fp32 roundings, one to bf16
        tol = (2.0 ** -8 + 56 * 2.0 ** -24) * 1.01
        assert ((self.logits[:n].double() - want).abs() <= tol * want.abs() + 1e-30).all()
        o = oracle.verify_greedy(W.bf16_bits(self.logits[:n]), self.off.cpu().numpy(), self.tokens[:n].cpu().numpy())
        np.testing.assert_array_equal(self.acc.cpu().numpy(), o.accepted_len)
        np.testing.assert_array_equal(self.out[:n].cpu().numpy(), o.out_tokens[:n])


def test_norm_projection_and_verifier():
    s = Serving()
    for seed in (1, 2):
        s.fill(seed)
        s.logits.fill_(77)
        s.step()
        s.check()
        assert (s.logits[int(s.off[s.R]):] == 77).all()          # rows behind the batch's last one


def test_captured_once_replayed_on_other_batches():
    s = Serving()
    s.fill(1)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        s.step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            s.step()
    for seed in (5, 6, 7):
        s.fill(seed)
        torch.cuda.synchronize()
        graph.replay()
        s.check()


def test_the_sampling_verifier_reads_the_projections_rows():
    s = Serving(R=8, gamma=4, V=4096)
    s.fill(9)
    s.step()
    torch.cuda.synchronize()
    n, R = int(s.off[s.R]), s.R
    draft = (s.logits[:n].float() + 0.5 * torch.randn(n, s.V, device="cuda")).bfloat16()
    drafts = torch.cat([draft[int(s.off[r]): int(s.off[r + 1]) - 1] for r in range(R)])
    toks = drafts.float().argmax(1).to(torch.int32)
    flat = torch.zeros(n, dtype=torch.int32, device="cuda")
    at = 0
    for r in range(R):
        k = int(s.off[r + 1] - s.off[r]) - 1
        flat[int(s.off[r]): int(s.off[r]) + k] = toks[at: at + k]
        at += k
    B.dspark_verify(s.logits, drafts, s.off, flat, 0.8, 11, accepted_len=s.acc, out_tokens=s.out, dev_status=s.st, workspace=s.work, n_rows=n)
    torch.cuda.synchronize()
    o = oracle.verify(W.bf16_bits(s.logits[:n]), W.bf16_bits(drafts), s.off.cpu().numpy(), flat.cpu().numpy(), 0.8, 11)
    differ = np.nonzero(s.acc.cpu().numpy() != o.accepted_len)[0]
    assert int(s.st) == 0 and len(differ) == 0


class Training:
    def __init__(self, N, V, d, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.N, self.V, self.d = N, V, d
        self.w = (torch.randn(V, d, generator=g, device="cuda") / d ** 0.5).bfloat16()
        self.h = torch.randn(N, d, generator=g, device="cuda").bfloat16()
        self.labels = torch.randint(0, V, (N,), generator=g, device="cuda", dtype=torch.int32)
        self.labels[torch.rand(N, generator=g, device="cuda") < 0.2] = -1
        self.gl = torch.rand(N, generator=g, device="cuda") / N
        self.loss, self.lse = torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
        self.dh, self.dw = torch.empty_like(self.h), torch.empty_like(self.w)
        self.st = torch.zeros(1, dtype=torch.int32, device="cuda")

    def step(self, ws):
        B.dspark_lm_head_loss(self.h, self.w, self.labels, out_loss=self.loss, out_lse=self.lse, dev_status=self.st, workspace=ws)
        B.dspark_lm_head_loss_backward(self.h, self.w, self.labels, self.lse, self.gl, out_grad_hidden=self.dh, out_grad_weight=self.dw,
                                       dev_status=self.st, workspace=ws)

    def check(self):
        """Against autograd in 64 bits; G's and the result's roundings to bf16 (2^-8 at most each, spread evenly, as a norm
        2^-8 / sqrt(3) each) stay below 2^-8 of the gradient as a whole."""
        h, w = self.h.double().requires_grad_(), self.w.double().requires_grad_()
        live = self.labels >= 0
        z = (h @ w.T)[live]
        loss = torch.nn.functional.cross_entropy(z, self.labels[live].long(), reduction="none")
        (loss * self.gl[live].double()).sum().backward()
        assert int(self.st) == 0
        assert ((self.loss[live].double() - loss).abs() <= 1e-5 * (1 + loss.abs())).all() and (self.loss[~live] == 0).all()
        for got, want in ((self.dh, h.grad), (self.dw, w.grad)):
            assert float((got.double() - want).norm()) <= 2.0 ** -8 * float(want.norm())


def test_training_steps():
    t = Training(150, 2000, 96, 1)
    ws = B.workspace(B.dspark_lm_head_loss_workspace_bytes(t.N, t.V, t.d))
    for _ in range(3):
        t.step(ws)
        torch.cuda.synchronize()
        t.check()
        t.w = (t.w.float() - 20.0 * t.dw.float()).bfloat16()
        t.h = (t.h.float() - 20.0 * t.dh.float()).bfloat16()


def test_two_captured_steps_share_a_workspace():
    a, b = Training(300, 3000, 128, 2), Training(90, 1111, 72, 3)
    nbytes = max(B.dspark_lm_head_loss_workspace_bytes(t.N, t.V, t.d) for t in (a, b))
    ws = B.workspace(nbytes)
    stream = torch.cuda.Stream()
    graphs = []
    with torch.cuda.stream(stream):
        for t in (a, b):
            t.step(ws)
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                t.step(ws)
            graphs.append(g)
    for k in range(3):
        for t in (a, b):
            t.h.copy_(torch.randn(t.N, t.d, device="cuda"))
            t.labels.copy_(torch.randint(-1, t.V, (t.N,), device="cuda"))
            t.dw.fill_(float("nan"))
            t.dh.fill_(float("nan"))
        torch.cuda.synchronize()
        graphs[0].replay()
        graphs[1].replay()
        graphs[0].replay()
        torch.cuda.synchronize()
        a.check()
        b.check()


def test_two_streams_at_once():
    a, b = Training(260, 9000, 192, 4), Training(100, 12000, 256, 5)
    sides = [(t, torch.cuda.Stream(), B.workspace(B.dspark_lm_head_loss_workspace_bytes(t.N, t.V, t.d))) for t in (a, b)]
    torch.cuda.synchronize()
    for _ in range(5):
        for t, stream, ws in sides:
            with torch.cuda.stream(stream):
                t.step(ws)
    torch.cuda.synchronize()
    a.check()
    b.check()


def test_the_calls_run_on_the_callers_stream():
    # work queued before on the same stream is seen: the hidden states are written right before the call, after a delay
    t = Training(64, 3000, 64, 6)
    ws = B.workspace(B.dspark_lm_head_loss_workspace_bytes(t.N, t.V, t.d))
    stream = torch.cuda.Stream()
    src = torch.randn(t.N, t.d, device="cuda").bfloat16()
    big = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        for _ in range(8):
            big = big @ big * 1e-4
        t.h.copy_(src)
        t.step(ws)
    torch.cuda.synchronize()
    t.check()
