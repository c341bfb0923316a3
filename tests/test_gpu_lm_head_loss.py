"""dspark_lm_head_loss and its backward against the formulas in 64 bits and against differences.

Tolerances.  A logit is a sum of d exact products in fp32, added 16 at a time; a partial sum is at most A = sum |h w|, so
the logit is off by at most dz = (d / 16 + 8) 2^-23 A.  Loss and lse: that, plus 8 roundings of their own size.
Gradients: the exponent z - lse is off by dz on either side and by what fp32 holds of lse: up to 8 x 2^-24 |lse| as above,
then the product with log2 e, that constant and the subtraction (3 x 2^-24 |lse|), together dx = 2 dz + 11 x 2^-24 |lse|.
An entry of G is p g (1 +- dx +- 2^-20), rounded to bf16 (half a step, 2^-8), so a sum over entries is off by at most
(2^-8 + dx + 2^-20) sum |G| |W| (with the two terms of the label's entry taken apart), plus the fp32 sum of its terms
and the rounding of the result.  An entry of G (or p) below the smallest normal number is taken as zero: 2^-126 each."""
import pytest
import torch

from paper_2607_05147_b200 import binding as B

pytestmark = pytest.mark.gpu

H = 2.0 ** -8


def make(N, V, d, seed, ignored=0.0, pad=0, lift=6.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    pitch = -(-d // 8) * 8 + 8 * pad
    w = (torch.randn(V, pitch, generator=g, device="cuda") * (2.5 / d ** 0.5)).bfloat16()[:, :d]
    labels = torch.randint(0, V, (N,), generator=g, device="cuda", dtype=torch.int32)
    h = torch.randn(N, d + 3 * pad, generator=g, device="cuda")[:, :d]
    h = (h + torch.rand(N, 1, generator=g, device="cuda") * (lift / 6.25) * w[labels.long()].float()).bfloat16()
    if pad:                                     # a row pitch that is not a multiple of 8
        h = torch.cat([h, h[:, : 3 * pad]], 1)[:, :d]
    drop = torch.rand(N, generator=g, device="cuda") < ignored
    labels[drop] = -1
    gl = torch.rand(N, generator=g, device="cuda") / N
    return h, w, labels, gl


def forward(h, w, labels):
    N, d = h.shape
    loss = torch.full((N,), -5.0, device="cuda")
    lse = torch.full((N,), -5.0, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = B.workspace(B.dspark_lm_head_loss_workspace_bytes(N, w.shape[0], d)).fill_(0xFF)
    B.dspark_lm_head_loss(h, w, labels, out_loss=loss, out_lse=lse, dev_status=st, workspace=ws)
    torch.cuda.synchronize()
    return loss, lse, int(st)


def backward(h, w, labels, lse, gl, want=(True, True), pads=(0, 0)):
    N, d = h.shape
    V = w.shape[0]
    dh = torch.full((N, d + pads[0]), 9.0, dtype=torch.bfloat16, device="cuda")
    dw = torch.full((V, d + pads[1]), 9.0, dtype=torch.bfloat16, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = B.workspace(B.dspark_lm_head_loss_workspace_bytes(N, V, d)).fill_(0xFF)
    B.dspark_lm_head_loss_backward(h, w, labels, lse, gl, out_grad_hidden=dh[:, :d] if want[0] else None,
                                   out_grad_weight=dw[:, :d] if want[1] else None, dev_status=st, workspace=ws)
    torch.cuda.synchronize()
    assert (dh[:, d:] == 9).all() and (dw[:, d:] == 9).all()
    return dh[:, :d], dw[:, :d], int(st)


def reference(h, w, labels, gl):
    live = (labels >= 0) & (labels < w.shape[0])
    hd = torch.where(live[:, None], h.double(), 0.0)
    wd = w.double()
    z = hd @ wd.T
    lse = torch.logsumexp(z, 1)
    at = labels.clamp(0, w.shape[0] - 1).long()[:, None]
    loss = lse - z.gather(1, at)[:, 0]
    p = (z - lse[:, None]).exp()
    g = torch.where(live, gl.double(), 0.0)[:, None]
    one = torch.zeros_like(p).scatter_(1, at, 1.0)
    G, Gabs = (p - one) * g, (p + one) * g.abs()
    dz = (h.shape[1] / 16 + 8) * 2.0 ** -23 * float((hd.abs() @ wd.abs().T).max())
    out = dict(loss=torch.where(live, loss, 0.0), lse=torch.where(live, lse, 0.0), dh=G @ wd, dw=G.T @ hd)
    dx = 2 * dz + 11 * 2.0 ** -24 * float(out["lse"].abs().max()) + 2.0 ** -20
    rel = H + dx
    tol = dict(loss=2 * dz + 8 * 2.0 ** -24 * (lse.abs() + loss.abs()), lse=dz + 8 * 2.0 ** -24 * lse.abs(),
               dh=rel * (Gabs @ wd.abs()) + H * out["dh"].abs() + 2.0 ** -126 * (1 + wd.abs().sum(0)),
               dw=rel * (Gabs.T @ hd.abs()) + H * out["dw"].abs() + 2.0 ** -126 * (1 + hd.abs().sum(0)))
    # what an entry of G is off by before its rounding, carried through the products
    tol["dh_exact"] = dx * (Gabs @ wd.abs())
    tol["dw_exact"] = dx * (Gabs.T @ hd.abs())
    return out, tol


def check(h, w, labels, gl, pads=(0, 0)):
    out, tol = reference(h, w, labels, gl)
    loss, lse, st = forward(h, w, labels)
    assert st == 0
    assert ((loss.double() - out["loss"]).abs() <= tol["loss"]).all()
    assert ((lse.double() - out["lse"]).abs() <= tol["lse"]).all()
    dh, dw, st = backward(h, w, labels, lse, gl, pads=pads)
    assert st == 0
    assert ((dh.double() - out["dh"]).abs() <= tol["dh"] * 1.01).all()
    assert ((dw.double() - out["dw"]).abs() <= tol["dw"] * 1.01).all()
    dead = labels < 0
    assert (loss[dead] == 0).all() and (lse[dead] == 0).all() and (dh[dead] == 0).all()
    # as a whole the error is that of the roundings, which do not add up: half a step of bf16 is 2^-8, uniformly spread
    # 2^-8 / sqrt(3) of the value; two of them side by side (G's and the result's) stay below 2^-8
    for name, got in (("dh", dh), ("dw", dw)):
        assert (got.double() - out[name]).norm() <= H * out[name].norm() + tol[name + "_exact"].norm()
    return loss, lse, dh, dw


@pytest.mark.parametrize("N,V,d", [(1, 1, 1), (1, 2, 8), (1, 1000, 64), (2, 256, 16), (5, 257, 63), (64, 1000, 128), (65, 513, 200), (127, 300, 72),
                                   (128, 2048, 256), (129, 4100, 257), (200, 10007, 500), (300, 777, 1024), (520, 5000, 320)])
def test_sizes(N, V, d):
    check(*make(N, V, d, N + V + d), pads=(1, 2))


@pytest.mark.parametrize("ignored", [0.3, 0.9])
def test_ignored_rows(ignored):
    check(*make(333, 2000, 136, 7, ignored=ignored))


def test_row_pitches():
    check(*make(150, 700, 100, 8, pad=1), pads=(4, 8))


@pytest.mark.parametrize("d", [64, 33, 34, 500, 511])
@pytest.mark.parametrize("pad", [0, 1, 2, 6, 16])
def test_pitches_of_the_weight_gradient(d, pad):
    # whole sectors, pairs and single elements; the last row of the last tile of 32
    check(*make(40, 333, d, 21), pads=(pad, pad))


@pytest.mark.parametrize("V", [18944, 28417, 33153, 40001, 76000])
def test_narrower_tiles_of_the_statistics(V):
    # vocabularies for which few rows take tiles of 128 (all whole), 224, 256, 160 (one entry in the last) and 192 entries
    check(*make(90, V, 72, 23, ignored=0.1))


def test_every_row_ignored():
    h, w, labels, gl = make(70, 600, 64, 9)
    labels[:] = -1
    h[3] = float("nan")
    loss, lse, st = forward(h, w, labels)
    dh, dw, st2 = backward(h, w, labels, lse, gl)
    assert st == 0 and st2 == 0
    for t in (loss, lse, dh, dw):
        assert (t == 0).all()


@pytest.mark.parametrize("kind", ["one label", "two labels", "neighbours", "ends"])
def test_labels_that_many_rows_share(kind):
    h, w, labels, gl = make(300, 1500, 200, 19, ignored=0.1)
    live = labels >= 0
    some = {"one label": [777], "two labels": [255, 256], "neighbours": list(range(512, 530)), "ends": [0, 1499]}[kind]
    labels[live] = torch.tensor(some, device="cuda", dtype=torch.int32)[torch.arange(300, device="cuda") % len(some)][live]
    check(h, w, labels, gl)


@pytest.mark.parametrize("V,d", [(900, 100), (300, 257), (5000, 64)])
def test_runs_of_every_length(V, d):
    # neighbouring entries that are the label of 1, 2, ... 40 rows: runs a lane adds up alone (up to 16) and ones that the
    # warp shares, of whole and of broken groups of eight rows, at the edge of a tile of 128 entries
    first = 110
    labels = torch.repeat_interleave(torch.arange(first, first + 40), torch.arange(1, 41))
    N = labels.numel()
    h, w, _, gl = make(N, V, d, 22)
    labels = labels[torch.randperm(N, generator=torch.Generator().manual_seed(3))].int().cuda()
    gl.fill_(1.0 + 2.0 ** -8 - 2.0 ** -12)              # every label's entry of G rounded to the same side
    check(h, w, labels, gl, pads=(0, 16 - d % 16))


def test_equal_weights_whose_rounding_is_the_same_for_every_row():
    # g = 1.00390625 - tiny: every label's entry of G, about -g, loses almost half a step of bf16 on the same side
    h, w, labels, gl = make(260, 3000, 128, 20, lift=0.0)
    gl.fill_(1.0 + 2.0 ** -8 - 2.0 ** -12)
    out, _ = reference(h, w, labels, gl)
    _, lse, _ = forward(h, w, labels)
    dh, dw, _ = backward(h, w, labels, lse, gl)
    # the result's rounding (2^-8 / sqrt 3 as a norm) and the little that the entries beside the labels' add
    for got, want in ((dh, out["dh"]), (dw, out["dw"])):
        assert (got.double() - want).norm() <= 0.7 * H * want.norm()


def test_what_an_ignored_row_holds_reaches_nothing():
    h, w, labels, gl = make(200, 900, 64, 10, ignored=0.3)
    a = check(h, w, labels, gl)
    dead = labels < 0
    h2, gl2 = h.clone(), gl.clone()
    h2[dead] = float("nan")
    h2[dead.nonzero()[0, 0]] = float("inf")
    gl2[dead] = float("nan")
    loss, lse, st = forward(h2, w, labels)
    lse[dead] = float("nan")
    dh, dw, st2 = backward(h2, w, labels, lse, gl2)
    assert st == 0 and st2 == 0
    assert torch.equal(loss, a[0]) and torch.equal(dh, a[2]) and torch.equal(dw, a[3])


def test_labels_outside_the_vocabulary():
    h, w, labels, gl = make(40, 300, 64, 11)
    labels[5], labels[6] = 300, 2 ** 31 - 1
    loss, lse, st = forward(h, w, labels)
    assert st == B.DEV_BAD_TOKEN and float(loss[5]) == 0 and float(lse[6]) == 0
    dh, dw, st = backward(h, w, labels, lse, gl)
    assert st == B.DEV_BAD_TOKEN and (dh[5:7] == 0).all()
    labels[5:7] = -1
    dh2, dw2, _ = backward(h, w, labels, lse, gl)
    assert torch.equal(dh, dh2) and torch.equal(dw, dw2)


def test_a_row_that_cannot_be_normalised_is_reported_and_stays_alone():
    h, w, labels, gl = make(140, 1000, 64, 12)
    good = forward(h, w, labels)
    h2 = h.clone()
    h2[17, 3] = float("nan")
    loss, lse, st = forward(h2, w, labels)
    assert st == B.DEV_BAD_ROW and torch.isnan(loss[17])
    keep = torch.arange(140, device="cuda") != 17
    assert torch.equal(loss[keep], good[0][keep])


def test_large_logits():
    # logits of several hundred: the softmax is one entry, the loss the distance to it
    h, w, labels, gl = make(60, 800, 64, 13)
    check((h.float() * 64).bfloat16(), w, labels, gl)


@pytest.mark.parametrize("N,pad", [(1, 0), (2, 0), (100, 1), (200, 0)])
def test_rows_that_are_sure_of_their_label(N, pad):
    """Losses of 5e-3 at d = 16 384: softmax - 1 at the label is small against what a long sum that is cut off loses.

    A loss is log(1 + e^-z[label] sum e^z), so it is off by what the exponents are (2 dz) and the exponentials (2^-20), all
    relative to its size; lse is rounded once, and the label's entry e^(z - lse) - 1 sees that and the 11 roundings of lse as
    above, and the loss's own error.  It is rounded to bf16 in two parts.  Every other entry is a probability, off by its
    exponent and half a step."""
    V, d = 2000, 16384
    g = torch.Generator(device="cuda").manual_seed(77 + N)
    w = (torch.randn(V, d, generator=g, device="cuda") * (0.2 / d ** 0.5)).bfloat16()
    labels = torch.randperm(V, generator=g, device="cuda")[:N].int()
    h = (torch.rand(N, d, generator=g, device="cuda") + 0.5) * w[labels.long()].float().sign()
    z = (h.double() * w[labels.long()].double()).sum(1, keepdim=True)
    h = h * (12.9 / z).float()
    h = torch.cat([h, h[:, :pad]], 1).bfloat16()[:, :d]
    gl = torch.ones(N, device="cuda")
    hd, wd, at = h.double(), w.double(), labels.long()[:, None]
    z = hd @ wd.T
    lse = torch.logsumexp(z, 1, keepdim=True)
    want = (z.scatter(1, at, float("-inf")) - lse).exp().sum(1, keepdim=True)       # 1 - softmax at the label
    loss = -torch.log1p(-want)
    assert float(loss.min()) > 2e-3 and float(loss.max()) < 2e-2
    dz = (d / 16 + 8) * 2.0 ** -23 * float((hd.abs() @ wd.abs().T).max())            # of any logit, summed in one piece
    p = (z - lse).exp().scatter(1, at, 0.0)
    G = p.scatter(1, at, -want)
    one = torch.zeros_like(p).scatter_(1, at, 1.0)
    got = forward(h, w, labels)
    assert got[2] == 0
    assert ((got[0].double() - loss[:, 0]).abs() <= (2 * dz + 2.0 ** -19) * loss[:, 0]).all()
    dh, dw, st = backward(h, w, labels, got[1], gl)
    assert st == 0
    rel = H + 2 * dz + 11 * 2.0 ** -24 * float(lse.max()) + 2.0 ** -20
    off = rel * p + (11 * 2.0 ** -24 * lse.max() + (2 * dz + 2.0 ** -19 + H * H) * want) * one
    assert ((dh.double() - G @ wd).abs() <= off @ wd.abs() + H * (G @ wd).abs() + 2.0 ** -20 * (G.abs() @ wd.abs())).all()
    assert ((dw.double() - G.T @ hd).abs() <= off.T @ hd.abs() + H * (G.T @ hd).abs() + 2.0 ** -20 * (G.abs().T @ hd.abs())).all()


@pytest.mark.parametrize("N", [1, 130])
@pytest.mark.parametrize("size", [0.5, -200.0, 200.0])
def test_a_vocabulary_of_one_entry(N, size):
    # nothing but the label: the loss is the logarithm of one, whatever the logit
    d = 64
    h = torch.full((N, d), size, device="cuda").bfloat16()
    w = torch.full((1, d), 0.5, device="cuda").bfloat16()
    labels = torch.zeros(N, dtype=torch.int32, device="cuda")
    loss, lse, st = forward(h, w, labels)
    assert st == 0 and (loss == 0).all() and (lse == d * 0.5 * size).all()
    dh, dw, st = backward(h, w, labels, lse, torch.ones(N, device="cuda"))
    assert st == 0 and (dh == 0).all() and (dw == 0).all()


@pytest.mark.parametrize("N", [3, 200])
def test_labels_far_below_the_largest_logit(N):
    # losses of several hundred, and a label whose own logit is far below what e^x holds
    h, w, labels, gl = make(N, 700, 128, 21, lift=-60.0)
    check((h.float() * 16).bfloat16(), w, labels, gl)


def test_equal_logits():
    h = torch.zeros(30, 40, dtype=torch.bfloat16, device="cuda")
    w = torch.randn(1000, 40, device="cuda").bfloat16()
    labels = torch.arange(30, dtype=torch.int32, device="cuda") * 33
    loss, lse, _ = forward(h, w, labels)
    want = torch.log(torch.tensor(1000.0, dtype=torch.float64))
    assert ((loss.double().cpu() - want).abs() <= 8 * 2.0 ** -24 * want).all()


def test_one_gradient_without_the_other():
    args = make(150, 1500, 96, 14, ignored=0.2)
    h, w, labels, gl = args
    _, lse, _ = forward(h, w, labels)
    dh, dw, _ = backward(h, w, labels, lse, gl)
    dh1, dw1, _ = backward(h, w, labels, lse, gl, want=(True, False))
    dh2, dw2, _ = backward(h, w, labels, lse, gl, want=(False, True))
    assert torch.equal(dh, dh1) and (dw1 == 9).all() and torch.equal(dw, dw2) and (dh2 == 9).all()


def test_the_same_inputs_give_the_same_bits():
    h, w, labels, gl = make(400, 3001, 300, 15, ignored=0.1)
    first = [*forward(h, w, labels)[:2]]
    first += [*backward(h, w, labels, first[1], gl)[:2]]
    for _ in range(3):
        again = [*forward(h, w, labels)[:2]]
        again += [*backward(h, w, labels, again[1], gl)[:2]]
        assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_several_pieces_of_the_vocabulary():
    # 20 000 rows: a piece of G is the smallest kept (2 048 entries), so a vocabulary of 5 000 takes three pieces, the
    # last of them ragged
    h, w, labels, gl = make(20000, 5000, 64, 16, ignored=0.5)
    check(h, w, labels, gl)


@pytest.mark.parametrize("N,V,d", [(20000, 12001, 64), (100, 70000, 4096), (1500, 60001, 72)])
def test_many_pieces(N, V, d):
    # six, five and six pieces: the fourth overwrites the first one's G; with pairs of CTAs and without
    h, w, labels, gl = make(N, V, d, 18, ignored=0.1)
    check(h, w, labels, gl)


def test_full_vocabulary():
    h, w, labels, gl = make(70, 129280, 256, 17)
    check(h, w, labels, gl)


def test_gradients_against_differences():
    # hidden states and weights that are multiples of 1/64 below 2: a step of 1/64 either way is exact in bf16.
    # d loss / d epsilon = <gradient, direction>; the central difference is off by epsilon^2 / 6 times the third
    # derivative, at most (sum |direction| |w|)^3 -- computed below -- and by the two losses' fp32 roundings.
    torch.manual_seed(3)
    N, V, d = 12, 50, 24
    step = 1 / 64
    h = (torch.randint(-60, 61, (N, d), device="cuda") * step).bfloat16()
    w = (torch.randint(-60, 61, (V, d), device="cuda") * step).bfloat16()
    labels = torch.randint(0, V, (N,), device="cuda", dtype=torch.int32)
    gl = torch.rand(N, device="cuda") + 0.5
    _, lse, _ = forward(h, w, labels)
    dh, dw, _ = backward(h, w, labels, lse, gl)
    _, tol = reference(h, w, labels, gl)

    def total(hh, ww):
        return float((forward(hh, ww, labels)[0].double() * gl.double()).sum())

    for _ in range(6):
        n, k, v = (int(torch.randint(0, x, (1,))) for x in (N, d, V))
        for which in ("h", "w"):
            hp, hm, wp, wm = h.clone(), h.clone(), w.clone(), w.clone()
            if which == "h":
                hp[n, k] += step
                hm[n, k] -= step
                got, t, reach = float(dh[n, k]), float(tol["dh"][n, k]), float(w[:, k].float().abs().max())
                weight = float(gl[n])
            else:
                wp[v, k] += step
                wm[v, k] -= step
                got, t, reach = float(dw[v, k]), float(tol["dw"][v, k]), float(h[:, k].float().abs().max())
                weight = float(gl.sum())
            diff = (total(hp, wp) - total(hm, wm)) / (2 * step)
            third = weight * (2 * reach) ** 3 * step ** 2 / 6
            rounding = float((gl.double() * tol["loss"]).sum()) / step
            assert abs(got - diff) <= t + third + rounding
