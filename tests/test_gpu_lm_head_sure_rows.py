"""Gradients of rows that are sure of their label: losses of 1e-4 to 1e-7 at logits of 17 to 24, where lse in fp32 no longer
holds what softmax - 1 at the label is.  The backward call that is given the loss keeps its digits.

Tolerances, relative to 1 - softmax at the label.  A logit is off by at most dz = (d / 16 + 8) 2^-23 sum |h w|, the loss of a
sure row therefore by 2 dz + 2^-19 of its size (the exponents, the exponentials).  The label's entry of G, expm1(-loss),
adds 2^-22 (the function, the product with grad_loss) and is rounded to bf16 in two parts, H^2.  Every other entry is a
probability: off by its exponent, 2 dz + 11 x 2^-24 lse + 2^-20, and half a step of bf16, H.  Results are rounded to bf16,
after fp32 sums (2^-20 of the sum of magnitudes)."""
import pytest
import torch

from paper_2607_05147_b200 import binding as B

pytestmark = pytest.mark.gpu

H = 2.0 ** -8


def make(N, pad):
    V, d = 2000, 1024
    g = torch.Generator(device="cuda").manual_seed(31 + N)
    w = (torch.randn(V, d, generator=g, device="cuda") * (0.2 / d ** 0.5)).bfloat16()
    labels = torch.randperm(V, generator=g, device="cuda")[:N].int()
    h = (torch.rand(N, d, generator=g, device="cuda") + 0.5) * w[labels.long()].float().sign()
    z = (h.double() * w[labels.long()].double()).sum(1, keepdim=True)
    h = h * (torch.linspace(17.3, 23.2, N, device="cuda")[:, None] / z).float()
    h = torch.cat([h, h[:, :pad]], 1).bfloat16()[:, :d]
    return h, w, labels, V, d


@pytest.mark.parametrize("N,pad", [(3, 0), (3, 1), (100, 0), (200, 0), (200, 3)])
@pytest.mark.parametrize("want_h,want_w", [(True, True), (True, False), (False, True)])
def test_the_label_s_entry_keeps_its_digits(N, pad, want_h, want_w):
    h, w, labels, V, d = make(N, pad)
    gl = torch.linspace(1.0, 2.0, N, device="cuda")
    hd, wd, at = h.double(), w.double(), labels.long()[:, None]
    z = hd @ wd.T
    lse = torch.logsumexp(z, 1, keepdim=True)
    want = (z.scatter(1, at, float("-inf")) - lse).exp().sum(1, keepdim=True)       # 1 - softmax at the label
    true_loss = -torch.log1p(-want)
    assert float(true_loss.max()) < 2e-4 and float(true_loss.min()) < 2e-6 and float(true_loss.min()) > 1e-8
    p = (z - lse).exp().scatter(1, at, 0.0)
    one = torch.zeros_like(p).scatter_(1, at, 1.0)
    G = p.scatter(1, at, -want)

    loss, out_lse = torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = B.workspace(B.dspark_lm_head_loss_workspace_bytes(N, V, d)).fill_(0xFF)
    B.dspark_lm_head_loss(h, w, labels, out_loss=loss, out_lse=out_lse, dev_status=st, workspace=ws)
    dz = (d / 16 + 8) * 2.0 ** -23 * float((hd.abs() @ wd.abs().T).max())
    of_loss = 2 * dz + 2.0 ** -19
    assert ((loss.double() - true_loss[:, 0]).abs() <= of_loss * true_loss[:, 0]).all()
    dh = torch.empty(N, d, dtype=torch.bfloat16, device="cuda") if want_h else None
    dw = torch.empty(V, d, dtype=torch.bfloat16, device="cuda") if want_w else None
    B.dspark_lm_head_loss_backward(h, w, labels, out_lse, gl, loss=loss, out_grad_hidden=dh, out_grad_weight=dw, dev_status=st, workspace=ws)
    torch.cuda.synchronize()
    assert int(st) == 0
    g = gl.double()[:, None]
    off = g * ((H + 2 * dz + 11 * 2.0 ** -24 * lse + 2.0 ** -20) * p + (of_loss + 2.0 ** -22 + H * H) * want * one)
    G = g * G
    if want_h:
        assert ((dh.double() - G @ wd).abs() <= off @ wd.abs() + H * (G @ wd).abs() + 2.0 ** -20 * (G.abs() @ wd.abs())).all()
    if want_w:
        assert ((dw.double() - G.T @ hd).abs() <= off.T @ hd.abs() + H * (G.T @ hd).abs() + 2.0 ** -20 * (G.abs().T @ hd.abs())).all()


def test_ordinary_rows_are_the_same_either_way():
    # losses of a few units: both forms are expm1 of the same number but for its last digits
    N, V, d = 300, 1500, 136
    g = torch.Generator(device="cuda").manual_seed(4)
    w = (torch.randn(V, d, generator=g, device="cuda") / d ** 0.5).bfloat16()
    h = torch.randn(N, d, generator=g, device="cuda").bfloat16()
    labels = torch.randint(0, V, (N,), generator=g, device="cuda", dtype=torch.int32)
    labels[::7] = -1
    labels[5] = V                                       # outside: ignored and reported
    gl = torch.rand(N, generator=g, device="cuda")
    loss, lse = torch.empty(N, device="cuda"), torch.empty(N, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = B.workspace(B.dspark_lm_head_loss_workspace_bytes(N, V, d)).fill_(0xFF)
    B.dspark_lm_head_loss(h, w, labels, out_loss=loss, out_lse=lse, dev_status=st, workspace=ws)
    dead = (labels < 0) | (labels >= V)
    loss[dead] = float("nan")                           # entries of ignored rows are not used
    out = []
    for given in (None, loss):
        dh, dw = torch.empty(N, d, dtype=torch.bfloat16, device="cuda"), torch.empty(V, d, dtype=torch.bfloat16, device="cuda")
        B.dspark_lm_head_loss_backward(h, w, labels, lse, gl, loss=given, out_grad_hidden=dh, out_grad_weight=dw, dev_status=st, workspace=ws)
        assert (dh[dead] == 0).all()
        out.append((dh.double(), dw.double()))
    torch.cuda.synchronize()
    assert int(st) == B.DEV_BAD_TOKEN
    # the label's entry differs by what lse and the logit are rounded by (2^-22 of it), a result next to a half by a step
    for a, b in zip(*out):
        assert (a - b).abs().max() <= 2 * H * b.abs().max()
        assert ((a - b) == 0).double().mean() > 0.99
