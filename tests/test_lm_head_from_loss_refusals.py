"""What dspark_lm_head_loss_backward_from_loss refuses beside what dspark_lm_head_loss_backward does (host, no GPU)."""
import pytest

from paper_2607_05147_b200 import binding as B

P = 0x10000
INVALID, SHAPE, ALIGN, WORKSPACE = 1, 2, 3, 4


@pytest.mark.parametrize("kw,code", [(dict(loss=None), INVALID), (dict(lse=None), INVALID), (dict(g=None), INVALID), (dict(dh=None, dw=None), INVALID),
                                     (dict(N=0), INVALID), (dict(N=(1 << 20) + 1), SHAPE), (dict(loss=P + 2), ALIGN), (dict(lse=P + 1), ALIGN),
                                     (dict(n=100), WORKSPACE), (dict(wsp=P + 128), ALIGN)])
def test_refusals(kw, code):
    a = dict(lse=P, loss=P, g=P, N=8, dh=P, dw=P, wsp=P, n=B.dspark_lm_head_loss_workspace_bytes(8, 100, 64))
    a.update(kw)
    assert B.lib().dspark_lm_head_loss_backward_from_loss(P, 64, P, 64, P, a["lse"], a["loss"], a["g"], a["N"], 100, 64, a["dh"], 64, a["dw"], 64,
                                                          P, a["wsp"], a["n"], None) == code
