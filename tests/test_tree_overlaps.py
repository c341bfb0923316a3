"""Outputs of the tree step's calls that share memory with another array: refused on the host before anything is launched (no GPU
needed: the addresses are never used)."""
import ctypes as C

import pytest

from paper_2607_05147_b200 import binding as B

INVALID = 1
V, R, ROWS = 100, 2, 8
# arrays of a call to dspark_verify_tree, a page apart, and their sizes in bytes
VERIFY = {"p": ROWS * V * 4, "q": ROWS * V * 4, "tok": ROWS * 4, "par": ROWS * 4, "off": (R + 1) * 4, "u": ROWS * 4, "ul": R * 4, "acc": R * 4,
          "out": ROWS * 4, "path": ROWS * 4, "st": 4}
VERIFY_OUT = ("acc", "out", "path", "st")


def verify(a):
    return B.lib().dspark_verify_tree(a["p"], V, a["q"], V, V, a["tok"], a["par"], a["off"], R, ROWS, a["u"], a["ul"], a["acc"], a["out"],
                                      a["path"], a["st"], None)


def places(sizes):
    return {name: 0x100000 * (i + 1) for i, name in enumerate(sizes)}


@pytest.mark.parametrize("other", VERIFY)
@pytest.mark.parametrize("out", VERIFY_OUT)
def test_verify(out, other):
    if out == other:
        return
    for at in (0, VERIFY[other] - 4, 4 - VERIFY[out]):        # the same place, the other's last entry, this one's last entry
        a = places(VERIFY)
        a[out] = a[other] + at
        assert verify(a) == INVALID


COMMIT = {"first": R * 4, "off": (R + 1) * 4, "acc": R * 4, "path": ROWS * 4, "st": 4}


@pytest.mark.parametrize("other", COMMIT)
def test_commit(other):
    c = B.KvCacheStruct(k=0x1000000, v=0x2000000, dtype=B.DSPARK_BF16, n_layers=2, n_pages=4, page_size=16, kv_heads=2, head_dim=64,
                        layer_stride=4 * 16 * 128, page_stride=16 * 128, token_stride=128, head_stride=64, block_table=0x3000000,
                        block_table_stride=8, max_pages=8)
    a = places(COMMIT)
    for at in (0, COMMIT[other] - 4, 4 - R * 4):
        assert B.lib().dspark_kv_commit(C.byref(c), a["first"], a["off"], R, ROWS, a["acc"], a["path"], a[other] + at, a["st"], None) == INVALID
