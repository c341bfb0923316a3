"""NaN and infinities among V's rows of a long prompt: they reach the rows that see them, and nothing else, without holding up the call
until its waits run out."""
import math

import pytest
import torch

import tree_helpers as T

pytestmark = pytest.mark.gpu


def chunk(n, others, kind, d, first=50):
    cache = T.Cache([first + n] + [9] * others, 64, 1, d, kind)
    g = T.gen(n)
    for c in (cache.k, cache.v):
        if kind == "bf16":
            c.normal_(generator=g)
        else:
            # (above 464 the conversion to e4m3 gives NaN: of half a million numbers one or two are beyond 4.64 standard deviations)
            c.copy_((torch.randn(c.shape, generator=g, device="cuda") * 100).clamp(-448, 448).to(c.dtype))
    for s in (cache.ks, cache.vs):
        if s is not None:
            s.fill_(0.01)
    q = torch.randn(n + others, 1, d, generator=g, device="cuda").bfloat16()
    return cache, q, T.i32([first] + [8] * others), T.offsets([n] + [1] * others)


def put(cache, node, component, what, first=50):
    pg, at = cache.slots(0, [first + node])
    if cache.kind == "bf16":
        cache.v[0, pg, at, 0, component] = what
    else:
        cache.v.view(torch.uint8)[0, pg, at, 0, component] = 0x7f


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("others", [0, 200])                  # 200 single tokens beside: the kernel for few rows
@pytest.mark.parametrize("parents", [False, True])
def test_a_long_prompt(kind, others, parents):
    n, d = 8192, 64
    cache, q, first, off = chunk(n, others, kind, d)
    par = T.i32([-1] + list(range(n - 1)) + [-1] * others) if parents else None
    clean, _, st = T.run_attention(cache, q, first, off, par, 0.1)
    assert st == 0 and bool(clean.isfinite().all())
    put(cache, 5, 3, math.inf)
    put(cache, 6000, 3, -math.inf)
    put(cache, 4000, 40, math.nan)
    put(cache, 8191, 63, math.inf)
    got, _, st = T.run_attention(cache, q, first, off, par, 0.1)
    assert st == 0
    want = clean.clone()
    want[5:n, 0, 3] = math.inf if kind == "bf16" else math.nan
    want[6000:n, 0, 3] = math.nan
    want[4000:n, 0, 40] = math.nan
    want[8191, 0, 63] = math.inf if kind == "bf16" else math.nan
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(7.0, 8.0, 9.0), want.nan_to_num(7.0, 8.0, 9.0))


@pytest.mark.parametrize("what", [math.inf, math.nan])
def test_a_prompt_full_of_them(what):
    n, d = 4096, 32
    cache, q, first, off = chunk(n, 0, "bf16", d)
    cache.v.fill_(what)
    cache.v[0, cache.table[0, 0].long(), :50] = 1.0           # not those before the step
    got, lse, st = T.run_attention(cache, q, first, off, None, 0.1)
    assert st == 0 and bool(lse.isfinite().all())
    assert bool((got.isnan() if math.isnan(what) else got == math.inf).all())


def test_a_very_long_prompt():
    n, d = 60000, 16
    cache, q, first, off = chunk(n, 0, "bf16", d)
    clean, _, st = T.run_attention(cache, q, first, off, None, 0.1)
    put(cache, 0, 2, math.inf)
    put(cache, 31000, 9, -math.inf)
    got, _, st2 = T.run_attention(cache, q, first, off, None, 0.1)
    assert st == st2 == 0
    clean[:, 0, 2] = math.inf
    clean[31000:, 0, 9] = -math.inf
    assert torch.equal(got, clean)
