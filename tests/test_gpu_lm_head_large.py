"""The vocabulary projection at the far ends of its sizes: offsets past 2^31 elements, many rows, wide rows, a very large
vocabulary; and what the Python layer refuses."""
import pytest
import torch

from paper_2607_05147_b200 import binding as B
from test_gpu_lm_head_int8 import check as check_int8, operands
from test_gpu_lm_head_loss import check as check_loss, make
from test_gpu_rms_norm import reference as norm_reference

pytestmark = pytest.mark.gpu


def test_int8_logits_past_two_to_the_31_elements():
    n, V, K = 17000, 129280, 64                      # 2.2e9 logits
    xq, xs, wq, ws = operands(n, V, K, 1)
    out = torch.empty(n, V, dtype=torch.bfloat16, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.dspark_lm_head_int8(xq, xs, wq, ws, out_logits=out, dev_status=st)
    torch.cuda.synchronize()
    for a, b in ((0, 3), (8300, 8310), (16600, 16615), (16990, 17000)):
        want = (xq[a:b].double() @ wq.double().T) * xs[a:b, None].double() * ws.double()
        assert ((out[a:b].double() - want).abs() <= (2.0 ** -8 + 3 * 2.0 ** -24) * 1.01 * want.abs()).all()


def test_norm_past_two_to_the_31_elements():
    n, d = 140000, 16384
    x = torch.randn(4096, d, device="cuda").bfloat16().repeat(35, 1)[:n]
    w = torch.randn(d, device="cuda").bfloat16()
    q = torch.empty(n, d, dtype=torch.int8, device="cuda")
    s = torch.empty(n, device="cuda")
    B.dspark_rms_norm_quant(x, w, 1e-6, out_q=q, out_scale=s)
    torch.cuda.synchronize()
    for a in (0, 65530, 131070, n - 8):
        _, rq, rs, _ = norm_reference(x[a: a + 8], None, w, 1e-6)
        assert torch.equal(q[a: a + 8], rq)
        assert ((s[a: a + 8].double() - rs).abs() <= 48 * 2.0 ** -24 * rs).all()


def test_int8_many_rows():
    check_int8(*operands(70001, 65, 48, 2), torch.bfloat16, live=69999)


def test_loss_of_wide_rows():
    check_loss(*make(3, 700, 9000, 3))
    check_loss(*make(150, 500, 8200, 4))


def test_loss_over_a_very_large_vocabulary():
    check_loss(*make(5, 2_000_003, 24, 5))


def test_loss_of_many_rows():
    check_loss(*make(66000, 300, 40, 6, ignored=0.2))


def test_what_the_python_layer_refuses():
    x = torch.zeros(4, 64, dtype=torch.bfloat16, device="cuda")
    q, s = torch.empty(4, 64, dtype=torch.int8, device="cuda"), torch.empty(4, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    w = x[0].contiguous()

    def norm(**kw):
        a = dict(x=x, weight=w, eps=1e-6, out_q=q, out_scale=s)
        a.update(kw)
        B.dspark_rms_norm_quant(**a)

    norm()
    for bad in (dict(x=x.half()), dict(x=x.t()), dict(x=x[0]), dict(weight=w.float()), dict(weight=w[:32]), dict(out_q=q.int()), dict(out_q=q[:3]),
                dict(out_q=q[:, :63]), dict(out_scale=s[:3]), dict(out_scale=s.double()), dict(residual=x.float()), dict(residual=x[:, :32]),
                dict(n_live=torch.ones(1, dtype=torch.int64, device="cuda")), dict(n_live=torch.ones(1, dtype=torch.int32)), dict(out_q=None),
                dict(out_norm=x.expand(4, 64)[:2]), dict(x=x[:1].expand(4, 64))):
        with pytest.raises(B.DsparkError):
            norm(**bad)

    logits = torch.empty(4, 10, device="cuda")
    wq, sw = torch.empty(10, 64, dtype=torch.int8, device="cuda"), torch.empty(10, device="cuda")

    def head(**kw):
        a = dict(x_q=q, x_scale=s, w_q=wq, w_scale=sw, out_logits=logits, dev_status=st)
        a.update(kw)
        B.dspark_lm_head_int8(**a)

    head()
    for bad in (dict(x_q=q.to(torch.uint8)), dict(w_q=wq[:, :48]), dict(x_scale=s[:2]), dict(out_logits=logits.half()), dict(out_logits=logits[:, :9]),
                dict(out_logits=logits[:3]), dict(dev_status=None), dict(out_logits=logits.t().contiguous().t()), dict(x_q=q[:, 1:], w_q=wq[:, 1:])):
        with pytest.raises(B.DsparkError):
            head(**bad)

    weight = torch.zeros(10, 64, dtype=torch.bfloat16, device="cuda")
    labels = torch.zeros(4, dtype=torch.int32, device="cuda")
    ws = B.workspace(B.dspark_lm_head_loss_workspace_bytes(4, 10, 64))

    def loss(**kw):
        a = dict(hidden=x, weight=weight, labels=labels, out_loss=s.clone(), out_lse=s.clone(), dev_status=st, workspace=ws)
        a.update(kw)
        B.dspark_lm_head_loss(**a)

    loss()
    for bad in (dict(hidden=x.float()), dict(weight=weight.float()), dict(weight=weight[:, :32]), dict(labels=labels.long()), dict(labels=labels[:2]),
                dict(out_loss=s.double()), dict(workspace=ws[:256]), dict(workspace=None), dict(weight=weight[:, 1:], hidden=x[:, 1:]),
                dict(labels=torch.zeros(8, dtype=torch.int32, device="cuda")[::2]), dict(hidden=x.cpu())):
        with pytest.raises(B.DsparkError):
            loss(**bad)
