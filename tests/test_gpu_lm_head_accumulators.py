"""The sums of the statistics' logits are cut into runs that are added up rounded, because the tensor cores cut an accumulator
off after every product: on operands of one sign, where every cut goes the same way, a long sum shows it.

Tolerances.  h and w positive, so partial sums rise to the logit S.  A product of 16 terms loses at most 2^-23 of the run's
sum: a run of t terms t / 16 x 2^-23 of its own sum, all runs together t / 16 x 2^-23 S (t = 256 for up to 128 rows, 512
beyond).  The runs are added up rounded, d / t additions of 2^-24 S each.  lse is off by that, the loss also by the label's
logit, summed in fp32 by 256 partial sums: (d / 256 + 8) 2^-24 S; both by 8 roundings of their own size.  One accumulator
for all of d loses about half a unit of the running sum at each of its products and more: 20, 211 and 557 x 2^-23 S measured
at d = 2 048, 8 192 and 16 384, above the 32 to 48 allowed here."""
import pytest
import torch

from paper_2607_05147_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N", [1, 64, 129, 200])
@pytest.mark.parametrize("d", [8192, 16384])
@pytest.mark.parametrize("V", [300, 5000])
def test_long_sums_of_one_sign(N, d, V):
    g = torch.Generator(device="cuda").manual_seed(N + d + V)
    h = (torch.rand(N, d, generator=g, device="cuda") + 0.5).bfloat16()
    w = ((torch.rand(V, d, generator=g, device="cuda") + 0.5) * (15.0 / d)).bfloat16()       # logits of about 15
    labels = torch.randint(0, V, (N,), generator=g, device="cuda", dtype=torch.int32)
    z = h.double() @ w.double().T
    S = float(z.max())
    want_lse = torch.logsumexp(z, 1)
    want_loss = want_lse - z.gather(1, labels.long()[:, None])[:, 0]
    loss, lse, st = torch.empty(N, device="cuda"), torch.empty(N, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = B.workspace(B.dspark_lm_head_loss_workspace_bytes(N, V, d))
    B.dspark_lm_head_loss(h, w, labels, out_loss=loss, out_lse=lse, dev_status=st, workspace=ws)
    torch.cuda.synchronize()
    assert int(st) == 0
    t = 256 if N <= 128 else 512
    of_z = (t / 16 * 2.0 ** -23 + d / t * 2.0 ** -24) * S
    of_label = (d / 256 + 8) * 2.0 ** -24 * S
    # the label's logit weighs in lse with its probability, here below 2 / V
    assert ((lse.double() - want_lse).abs() <= of_z + 2 / V * of_label + 8 * 2.0 ** -24 * want_lse).all()
    assert ((loss.double() - want_loss).abs() <= of_z + of_label + 8 * 2.0 ** -24 * (want_lse + want_loss.abs())).all()
