"""What the tree step's entry points refuse, on the host before anything is launched (no GPU needed: the addresses are never
used)."""
import ctypes as C

import pytest
import torch

from paper_2607_05147_b200 import binding as B

P = 0x10000          # an aligned address; every call below is refused before it would be used
INVALID, SHAPE, ALIGN, WORKSPACE = 1, 2, 3, 4


def cache(**kw):
    a = dict(k=P, v=P, k_scale=None, v_scale=None, dtype=B.DSPARK_BF16, n_layers=2, n_pages=4, page_size=16, kv_heads=2, head_dim=64,
             layer_stride=4 * 16 * 128, page_stride=16 * 128, token_stride=128, head_stride=64, block_table=P, block_table_stride=8, max_pages=8)
    a.update(kw)
    return B.KvCacheStruct(**a)


BAD_CACHES = [
    (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(block_table=None), INVALID), (dict(dtype=B.DSPARK_F32), INVALID), (dict(dtype=9), INVALID),
    (dict(dtype=B.DSPARK_I8), INVALID), (dict(dtype=B.DSPARK_E4M3, k_scale=P), INVALID), (dict(n_layers=0), INVALID), (dict(n_pages=0), INVALID),
    (dict(page_size=0), INVALID), (dict(kv_heads=0), INVALID), (dict(head_dim=0), INVALID), (dict(max_pages=0), INVALID), (dict(max_pages=9), INVALID),
    (dict(page_stride=-8), INVALID), (dict(token_stride=56), INVALID), (dict(head_stride=32), INVALID), (dict(page_stride=0), INVALID),
    (dict(layer_stride=0), INVALID),
    (dict(page_size=12), SHAPE), (dict(page_size=4), SHAPE), (dict(page_size=(1 << 20) + 1), SHAPE), (dict(head_dim=72, head_stride=72, token_stride=144), SHAPE),
    (dict(head_dim=272, head_stride=272, token_stride=544), SHAPE), (dict(kv_heads=1025), SHAPE), (dict(n_layers=1025), SHAPE),
    (dict(n_pages=(1 << 28) + 1), SHAPE),
    (dict(k=P + 8), ALIGN), (dict(v=P + 2), ALIGN), (dict(head_stride=68), ALIGN), (dict(token_stride=132), ALIGN), (dict(block_table=P + 2), ALIGN),
    (dict(dtype=B.DSPARK_I8, k_scale=P, v_scale=P, head_stride=72), ALIGN), (dict(dtype=B.DSPARK_I8, k_scale=P + 1, v_scale=P), ALIGN)]


def write(c, **kw):
    a = dict(layer=0, k=P, v=P, row=128, head=64, first=P, off=P, R=2, n=4, st=P)
    a.update(kw)
    return B.lib().dspark_kv_write(C.byref(c) if c is not None else None, a["layer"], a["k"], a["v"], a["row"], a["head"], a["first"], a["off"], a["R"],
                                   a["n"], a["st"], None)


def read(c, **kw):
    a = dict(layer=0, k=P, v=P, dtype=B.DSPARK_BF16, row=128, head=64, first=P, off=P, R=2, n=4, st=P)
    a.update(kw)
    return B.lib().dspark_kv_read(C.byref(c) if c is not None else None, a["layer"], a["first"], a["off"], a["R"], a["n"], a["k"], a["v"], a["dtype"],
                                  a["row"], a["head"], a["st"], None)


def commit(c, **kw):
    a = dict(first=P, off=P, R=2, n=4, acc=P, path=P, out=P + 4, st=P)
    a.update(kw)
    return B.lib().dspark_kv_commit(C.byref(c) if c is not None else None, a["first"], a["off"], a["R"], a["n"], a["acc"], a["path"], a["out"], a["st"], None)


def attend(c, **kw):
    a = dict(layer=0, q=P, qr=256, qh=64, hq=4, first=P, off=P, par=P, R=2, n=4, scale=0.1, out=P, outr=256, outh=64, lse=P, st=P, ws=P, size=None)
    a.update(kw)
    size = B.dspark_tree_attention_workspace_bytes(4, 4, 2, 64) if a["size"] is None else a["size"]
    return B.lib().dspark_tree_attention(C.byref(c) if c is not None else None, a["layer"], a["q"], a["qr"], a["qh"], a["hq"], a["first"], a["off"], a["par"],
                                         a["R"], a["n"], a["scale"], a["out"], a["outr"], a["outh"], a["lse"], a["st"], a["ws"], size, None)


@pytest.mark.parametrize("call", [write, read, commit, attend])
@pytest.mark.parametrize("kw,code", BAD_CACHES)
def test_caches(call, kw, code):
    assert call(cache(**kw)) == code


@pytest.mark.parametrize("call", [write, read, commit, attend])
@pytest.mark.parametrize("kw,code", [(dict(first=None), INVALID), (dict(off=None), INVALID), (dict(R=0), INVALID), (dict(n=0), INVALID), (dict(st=None), INVALID),
                                     (dict(R=(1 << 20) + 1), SHAPE), (dict(n=(1 << 24) + 1), SHAPE), (dict(first=P + 1), ALIGN), (dict(off=P + 2), ALIGN),
                                     (dict(st=P + 2), ALIGN)])
def test_steps(call, kw, code):
    assert call(cache(), **kw) == code
    assert call(None) == INVALID


@pytest.mark.parametrize("kw,code", [(dict(layer=2), INVALID), (dict(layer=-1), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(row=-8), INVALID),
                                     (dict(head=56), INVALID), (dict(row=56), INVALID), (dict(row=132), ALIGN), (dict(head=68), ALIGN), (dict(k=P + 8), ALIGN)])
def test_write(kw, code):
    assert write(cache(), **kw) == code


@pytest.mark.parametrize("kw,code", [(dict(layer=2), INVALID), (dict(k=None, v=None), INVALID), (dict(dtype=B.DSPARK_I8), INVALID), (dict(row=56), INVALID),
                                     (dict(row=132), ALIGN), (dict(dtype=B.DSPARK_F32, row=130), ALIGN), (dict(v=P + 8), ALIGN)])
def test_read(kw, code):
    assert read(cache(), **kw) == code


@pytest.mark.parametrize("kw,code", [(dict(acc=None), INVALID), (dict(path=None), INVALID), (dict(out=P), INVALID), (dict(acc=P + 1), ALIGN), (dict(path=P + 2), ALIGN),
                                     (dict(out=P + 2), ALIGN)])
def test_commit(kw, code):
    assert commit(cache(), **kw) == code


@pytest.mark.parametrize("kw,code", [
    (dict(layer=2), INVALID), (dict(q=None), INVALID), (dict(out=None), INVALID), (dict(hq=0), INVALID), (dict(hq=3), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(scale=float("inf")), INVALID), (dict(qr=56), INVALID), (dict(qh=-8), INVALID), (dict(outh=56), INVALID), (dict(outr=260), ALIGN), (dict(qh=68), ALIGN),
    (dict(q=P + 8), ALIGN), (dict(out=P + 8), ALIGN), (dict(par=P + 2), ALIGN), (dict(lse=P + 1), ALIGN), (dict(outr=512), INVALID),
    (dict(hq=258, qr=258 * 64, outr=258 * 64), SHAPE), (dict(ws=None), WORKSPACE), (dict(size=8), WORKSPACE), (dict(ws=P + 128), ALIGN)])
def test_attention(kw, code):
    assert attend(cache(), **kw) == code


def test_attention_is_for_heads_of_up_to_128():
    c = cache(head_dim=144, head_stride=144, token_stride=288, page_stride=16 * 288, layer_stride=4 * 16 * 288)
    assert attend(c, qr=4 * 144, qh=144, outr=4 * 144, outh=144) == SHAPE
    assert B.dspark_tree_attention_workspace_bytes(0, 4, 2, 64) == 0


@pytest.mark.parametrize("kw,code", [
    (dict(p=None), INVALID), (dict(tok=None), INVALID), (dict(par=None), INVALID), (dict(off=None), INVALID), (dict(u=None), INVALID), (dict(ul=None), INVALID),
    (dict(acc=None), INVALID), (dict(out=None), INVALID), (dict(st=None), INVALID), (dict(V=0), INVALID), (dict(R=0), INVALID), (dict(n=0), INVALID),
    (dict(ps=99), INVALID), (dict(qs=99), INVALID), (dict(V=(1 << 24) + 1, ps=1 << 25, qs=1 << 25), SHAPE), (dict(R=(1 << 20) + 1), SHAPE),
    (dict(n=(1 << 24) + 1), SHAPE), (dict(p=P + 2), ALIGN), (dict(q=P + 1), ALIGN), (dict(path=P + 2), ALIGN), (dict(u=P + 2), ALIGN)])
def test_verify(kw, code):
    a = dict(p=P, ps=100, q=P, qs=100, V=100, tok=P, par=P, off=P, R=2, n=8, u=P, ul=P, acc=P, out=P, path=P, st=P)
    a.update(kw)
    assert B.lib().dspark_verify_tree(a["p"], a["ps"], a["q"], a["qs"], a["V"], a["tok"], a["par"], a["off"], a["R"], a["n"], a["u"], a["ul"], a["acc"],
                                      a["out"], a["path"], a["st"], None) == code


def test_the_binding_refuses_cpu_tensors():
    k = torch.zeros(2, 8, 1, 16, dtype=torch.bfloat16)
    with pytest.raises(B.DsparkError):
        B.KvCache(k, k, torch.zeros(1, 2, dtype=torch.int32))
    p = torch.zeros(2, 4)
    with pytest.raises(B.DsparkError):
        B.dspark_verify_tree(p, None, None, None, None, None, None, accepted_len=None, out_tokens=None, dev_status=None)
