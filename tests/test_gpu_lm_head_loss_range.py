"""The vocabulary loss where it passes the range of fp32."""
import pytest
import torch

from paper_2607_05147_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N", [1, 140])
def test_a_loss_beyond_fp32_is_reported(N):
    # two logits of 3.2e38 and -3.2e38: the loss of the second is 6.4e38, an infinity in fp32
    h = torch.full((N, 1), 1.8e19, device="cuda").bfloat16()
    w = torch.zeros(2, 8, dtype=torch.bfloat16, device="cuda")[:, :1]
    w[0], w[1] = 1.8e19, -1.8e19
    labels = torch.zeros(N, dtype=torch.int32, device="cuda")
    loss, lse, st = torch.empty(N, device="cuda"), torch.empty(N, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = B.workspace(B.dspark_lm_head_loss_workspace_bytes(N, 2, 1))
    B.dspark_lm_head_loss(h, w, labels, out_loss=loss, out_lse=lse, dev_status=st, workspace=ws)
    assert int(st) == 0 and (loss == 0).all() and torch.isfinite(lse).all()
    labels[N - 1] = 1
    B.dspark_lm_head_loss(h, w, labels, out_loss=loss, out_lse=lse, dev_status=st, workspace=ws)
    assert int(st) == B.DEV_BAD_ROW and torch.isinf(loss[N - 1]) and (loss[: N - 1] == 0).all()
