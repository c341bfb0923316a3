"""What the vocabulary projection's entry points refuse, on the host before anything is launched (no GPU needed: the
addresses are never used)."""
import pytest
import torch

from paper_2607_05147_b200 import binding as B

P = 0x10000          # an aligned address; every call below is refused before it would be used
OK, INVALID, SHAPE, ALIGN, WORKSPACE = 0, 1, 2, 3, 4


def norm(**kw):
    a = dict(x=P, xs=64, res=None, rs=0, w=P, dtype=1, rows=4, d=64, eps=1e-6, live=None, h=None, hs=0, q=P, qs=64, s=P, y=None, ys=0)
    a.update(kw)
    return B.lib().dspark_rms_norm_quant(a["x"], a["xs"], a["res"], a["rs"], a["w"], a["dtype"], a["rows"], a["d"], a["eps"], a["live"],
                                         a["h"], a["hs"], a["q"], a["qs"], a["s"], a["y"], a["ys"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), INVALID), (dict(w=None), INVALID), (dict(q=None), INVALID), (dict(s=None), INVALID), (dict(rows=0), INVALID),
    (dict(d=0), INVALID), (dict(dtype=2), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID),
    (dict(xs=63), INVALID), (dict(qs=63), INVALID), (dict(res=P, rs=63), INVALID), (dict(h=P, hs=1), INVALID), (dict(y=P, ys=1), INVALID),
    (dict(d=16385, xs=16385, qs=16385), SHAPE), (dict(x=P + 1), ALIGN), (dict(s=P + 2), ALIGN), (dict(live=P + 2), ALIGN),
    (dict(dtype=0, x=P + 2), ALIGN)])
def test_norm(kw, code):
    assert norm(**kw) == code


def head(**kw):
    a = dict(x=P, xs=64, sx=P, w=P, ws=64, sw=P, rows=4, V=100, K=64, live=None, out=P, dtype=1, os=100, st=P)
    a.update(kw)
    return B.lib().dspark_lm_head_int8(a["x"], a["xs"], a["sx"], a["w"], a["ws"], a["sw"], a["rows"], a["V"], a["K"], a["live"], a["out"],
                                       a["dtype"], a["os"], a["st"], None)


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), INVALID), (dict(sx=None), INVALID), (dict(w=None), INVALID), (dict(sw=None), INVALID), (dict(out=None), INVALID),
    (dict(st=None), INVALID), (dict(rows=0), INVALID), (dict(V=0), INVALID), (dict(K=0), INVALID), (dict(dtype=2), INVALID),
    (dict(xs=63), INVALID), (dict(ws=48), INVALID), (dict(os=99), INVALID), (dict(rows=(1 << 20) + 1), SHAPE),
    (dict(V=(1 << 24) + 1, os=1 << 25), SHAPE), (dict(K=65537, xs=65552, ws=65552), SHAPE),
    (dict(x=P + 8), ALIGN), (dict(w=P + 1), ALIGN), (dict(xs=72), ALIGN), (dict(ws=65), ALIGN), (dict(sx=P + 1), ALIGN), (dict(sw=P + 2), ALIGN),
    (dict(out=P + 1), ALIGN), (dict(out=P + 2, dtype=0), ALIGN), (dict(live=P + 1), ALIGN)])
def test_int8_head(kw, code):
    assert head(**kw) == code


def test_quantise():
    f = B.lib().dspark_lm_head_quantize
    assert f(None, 64, 4, 64, P, 64, P, None) == INVALID
    assert f(P, 64, 0, 64, P, 64, P, None) == INVALID
    assert f(P, 63, 4, 64, P, 64, P, None) == INVALID
    assert f(P, 64, 4, 64, P, 63, P, None) == INVALID
    assert f(P + 1, 64, 4, 64, P, 64, P, None) == ALIGN
    assert f(P, 64, 4, 64, P, 64, P + 2, None) == ALIGN


def loss(backward=False, **kw):
    a = dict(h=P, hs=64, w=P, ws=64, y=P, N=8, V=100, d=64, loss=P, lse=P, g=P, dh=P, dhs=64, dw=P, dws=64, st=P, wsp=P, n=None)
    a.update(kw)
    n = B.dspark_lm_head_loss_workspace_bytes(8, 100, 64) if a["n"] is None else a["n"]
    if backward:
        return B.lib().dspark_lm_head_loss_backward(a["h"], a["hs"], a["w"], a["ws"], a["y"], a["lse"], a["g"], a["N"], a["V"], a["d"], a["dh"],
                                                    a["dhs"], a["dw"], a["dws"], a["st"], a["wsp"], n, None)
    return B.lib().dspark_lm_head_loss(a["h"], a["hs"], a["w"], a["ws"], a["y"], a["N"], a["V"], a["d"], a["loss"], a["lse"], a["st"],
                                       a["wsp"], n, None)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("kw,code", [
    (dict(h=None), INVALID), (dict(w=None), INVALID), (dict(y=None), INVALID), (dict(st=None), INVALID), (dict(lse=None), INVALID),
    (dict(N=0), INVALID), (dict(V=0), INVALID), (dict(d=0), INVALID), (dict(hs=63), INVALID), (dict(ws=56), INVALID),
    (dict(N=(1 << 20) + 1), SHAPE), (dict(V=(1 << 24) + 1), SHAPE), (dict(d=65537, hs=65544, ws=65544, dhs=65544, dws=65544), SHAPE),
    (dict(h=P + 1), ALIGN), (dict(w=P + 8), ALIGN), (dict(ws=68), ALIGN), (dict(y=P + 2), ALIGN), (dict(lse=P + 2), ALIGN),
    (dict(wsp=None), WORKSPACE), (dict(n=100), WORKSPACE), (dict(wsp=P + 128), ALIGN)])
def test_loss(backward, kw, code):
    assert loss(backward, **kw) == code


def test_loss_forward_and_backward_alone():
    assert loss(False, loss=None) == INVALID
    assert loss(True, g=None) == INVALID
    assert loss(True, dh=None, dw=None) == INVALID
    assert loss(True, dhs=63) == INVALID
    assert loss(True, dws=63) == INVALID
    assert loss(True, dw=P + 1) == ALIGN
    assert loss(True, g=P + 1) == ALIGN


def test_workspace_sizes():
    f = B.dspark_lm_head_loss_workspace_bytes
    for bad in ((0, 10, 10), (10, 0, 10), (10, 10, 0), ((1 << 20) + 1, 10, 10), (10, (1 << 24) + 1, 10), (10, 10, 65537)):
        assert f(*bad) == 0
    # the compact rows, a piece of G and one set of partial sums at the least, far below the logits
    n = f(4096, 129280, 2048)
    assert 4096 * 2048 * 2 + 4096 * 8192 * 2 + 4096 * 2048 * 4 <= n < 4096 * 129280 * 2
    assert f(1 << 20, 1 << 24, 4096) > 0


def test_cpu_tensors_are_refused():
    t = torch.zeros(4, 64, dtype=torch.bfloat16)
    with pytest.raises(B.DsparkError):
        B.dspark_rms_norm_quant(t, t[0], 1e-6, out_q=torch.zeros(4, 64, dtype=torch.int8), out_scale=torch.zeros(4))
    with pytest.raises(B.DsparkError):
        B.dspark_lm_head_loss(t, t, torch.zeros(4, dtype=torch.int32), out_loss=torch.zeros(4), out_lse=torch.zeros(4),
                              dev_status=torch.zeros(1, dtype=torch.int32), workspace=torch.zeros(16))
