"""dspark_lm_head_int8 and dspark_lm_head_quantize against the formula in 64 bits.

Tolerances.  The integer sum is exact; turning it into fp32 and the two products round once each (3 x 2^-24), the output
once more (half a step of its type)."""
import pytest
import torch

from paper_2607_05147_b200 import binding as B

pytestmark = pytest.mark.gpu


def operands(n, V, K, seed, pad=None):
    g = torch.Generator(device="cuda").manual_seed(seed)
    pitch = -(-K // 16) * 16 + (16 if pad else 0)
    xq = torch.randint(-127, 128, (n, pitch), generator=g, device="cuda", dtype=torch.int8)
    wq = torch.randint(-127, 128, (V, pitch), generator=g, device="cuda", dtype=torch.int8)
    xs = torch.rand(n, generator=g, device="cuda") + 0.1
    ws = torch.rand(V, generator=g, device="cuda") * 1e-3 + 1e-4
    return xq[:, :K], xs, wq[:, :K], ws


def check(xq, xs, wq, ws, dtype, out_pad=0, live=None, out_offset=0):
    n, V = xq.shape[0], wq.shape[0]
    rows = n if live is None else min(max(live, 0), n)
    full = torch.full((n, V + out_pad + out_offset), 123.0, dtype=dtype, device="cuda")
    out = full[:, out_offset: out_offset + V]
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.dspark_lm_head_int8(xq, xs, wq, ws, out_logits=out, dev_status=st,
                          n_live=None if live is None else torch.tensor([live], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert int(st) == 0
    want = (xq[:rows].double() @ wq.double().T) * xs[:rows, None].double() * ws.double()
    tol = (torch.finfo(dtype).eps / 2 + 3 * 2.0 ** -24) * 1.01
    assert ((out[:rows].double() - want).abs() <= tol * want.abs() + 1e-38).all()
    assert (out[rows:] == 123).all() and (full[:, :out_offset] == 123).all() and (full[:, out_offset + V:] == 123).all()
    return out


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,V,K", [(1, 1, 1), (1, 128, 128), (3, 129, 127), (31, 1000, 64), (32, 257, 1001), (33, 5, 2048), (64, 4096, 256),
                                   (65, 10007, 130), (128, 1024, 16), (255, 300, 512), (256, 130, 4096), (257, 999, 333), (600, 2000, 1024)])
def test_sizes(dtype, n, V, K):
    check(*operands(n, V, K, n + V + K), dtype, out_pad=3)


@pytest.mark.parametrize("n,V,K", [(700, 20001, 900), (1482, 9000, 1001), (300, 60000, 768), (130, 129280, 767)])
def test_pairs_by_the_size_of_the_product(n, V, K):
    # on either side of the rule that gives rows of up to 1 024 entries to pairs of CTAs
    check(*operands(n, V, K, n + V + K), torch.bfloat16, out_pad=1)


@pytest.mark.parametrize("live", [0, 1, 31, 256, 257, 300, 1000])
def test_rows_behind_the_last_one_are_left(live):
    check(*operands(300, 700, 200, 3), torch.bfloat16, live=live)


@pytest.mark.parametrize("n", [2, 17, 130, 200, 257, 300, 352, 511, 513, 700])
@pytest.mark.parametrize("K", [512, 4096])
def test_row_tiles_that_are_moved_back(n, K):
    # single CTAs and pairs; tiles whose boxes would reach past the last row; with and without a smaller live count
    ops = operands(n, 390, K, n + K)
    for live in (None, n - 1, n // 2 + 1):
        check(*ops, torch.bfloat16, live=live)
        check(*ops, torch.float32, live=live, out_pad=1)


def test_row_pitches_offsets_and_odd_strides():
    ops = operands(70, 333, 100, 4, pad=True)
    for pad, off in ((0, 0), (1, 0), (0, 1), (5, 3)):
        check(*ops, torch.bfloat16, out_pad=pad, out_offset=off)
        check(*ops, torch.float32, out_pad=pad, out_offset=off)


def test_columns_between_the_width_and_the_pitch_do_not_count():
    xq, xs, wq, ws = operands(40, 200, 100, 5)
    a = check(xq, xs, wq, ws, torch.float32).clone()
    xq._base[:, 100:] = 127
    wq._base[:, 100:] = -127
    assert torch.equal(check(xq, xs, wq, ws, torch.float32), a)


def test_the_largest_sums():
    K = 65536
    xq = torch.full((2, K), 127, dtype=torch.int8, device="cuda")
    wq = torch.full((3, K), -127, dtype=torch.int8, device="cuda")
    wq[1] = 127
    check(xq, torch.ones(2, device="cuda"), wq, torch.ones(3, device="cuda"), torch.float32)


def test_a_scale_of_nan_gives_a_row_of_nan():
    xq, xs, wq, ws = operands(5, 300, 64, 6)
    xs[2] = float("nan")
    xq[2] = 0
    out = torch.empty(5, 300, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    B.dspark_lm_head_int8(xq, xs, wq, ws, out_logits=out, dev_status=st)
    assert torch.isnan(out[2]).all() and torch.isfinite(out[[0, 1, 3, 4]]).all()


@pytest.mark.parametrize("V,K", [(1, 1), (5, 1001), (300, 64), (40, 4096)])
def test_quantised_weight(V, K):
    W = torch.randn(V, K + 3, device="cuda").bfloat16()[:, :K]
    if V > 2:
        W[1] = 0
        W[2, K - 1] = float("inf")
    q = torch.full((V, K + 5), 77, dtype=torch.int8, device="cuda")
    s = torch.empty(V, device="cuda")
    B.dspark_lm_head_quantize(W, q[:, :K], s)
    top = W.double().abs().amax(1, keepdim=True)
    want = torch.nan_to_num(torch.round(W.double() * 127 / top), nan=0.0)
    ok = torch.isfinite(top[:, 0])
    want[~ok] = 0
    assert torch.equal(q[:, :K], want.to(torch.int8)) and (q[:, K:] == 77).all()
    assert ((s.double() - top[:, 0] / 127).abs()[ok] <= 2.0 ** -23 * top[ok, 0]).all()
    assert torch.isnan(s[~ok]).all()
