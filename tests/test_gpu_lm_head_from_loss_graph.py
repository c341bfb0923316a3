"""A training step of the vocabulary projection whose backward is given the loss, captured once and replayed on other inputs,
on a side stream, with a workspace sized for a larger batch: the bits of the eager calls."""
import pytest
import torch

from paper_2607_05147_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N,V,d", [(60, 900, 72), (300, 2100, 136)])
def test_captured_and_replayed(N, V, d):
    g = torch.Generator(device="cuda").manual_seed(N)

    def inputs(scale):
        w = (torch.randn(V, d, generator=g, device="cuda") * scale / d ** 0.5).bfloat16()
        labels = torch.randint(-1, V, (N,), generator=g, device="cuda", dtype=torch.int32)
        h = (torch.randn(N, d, generator=g, device="cuda") + 4 * w[labels.clamp(min=0).long()].float()).bfloat16()
        return h, w, labels, torch.rand(N, generator=g, device="cuda")

    ws = B.workspace(B.dspark_lm_head_loss_workspace_bytes(4 * N, V, d)).fill_(0xFF)
    st = torch.zeros(1, dtype=torch.int32, device="cuda")

    def step(h, w, labels, gl, out):
        loss, lse, dh, dw = out
        B.dspark_lm_head_loss(h, w, labels, out_loss=loss, out_lse=lse, dev_status=st, workspace=ws)
        B.dspark_lm_head_loss_backward(h, w, labels, lse, gl, loss=loss, out_grad_hidden=dh, out_grad_weight=dw, dev_status=st, workspace=ws)

    def outputs():
        return (torch.empty(N, device="cuda"), torch.empty(N, device="cuda"), torch.empty(N, d, dtype=torch.bfloat16, device="cuda"),
                torch.empty(V, d, dtype=torch.bfloat16, device="cuda"))

    data, out = list(inputs(2.5)), outputs()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*data, out)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step(*data, out)
    torch.cuda.current_stream().wait_stream(side)
    for scale in (2.5, 1.0, 6.0):
        fresh, want = inputs(scale), outputs()
        step(*fresh, want)
        for a, b in zip(data, fresh):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
    assert int(st) == 0
