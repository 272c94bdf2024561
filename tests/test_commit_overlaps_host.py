"""Where the new lengths of a commit may not lie, without a GPU: on nothing that the same call still reads.  (One workgroup of a
sequence stores its length; the others may read the count, the path or the table after that.)"""
import ctypes

import pytest

B, N, BLOCKS, AT = 3, 4, 8, 0x100000             # lens_out is [AT, AT + 12)


@pytest.fixture(scope="module")
def hg():
    from paper_2507_03153_amd import build, hgca
    build.build(force=False)
    hgca.lib()
    return hgca


def commit(hg, first=None, path=None, cnt=None, table=None, first_block=None):
    rows = 0x10000000
    view = hg.KvView(rows, rows, None, table, 64, 16 if table else 0, BLOCKS if table else 0, first_block)
    shape = hg.Shape(hg.BF16, B, 8, 2, 128, 0.1)
    return hg.lib().hgca_kv_commit(ctypes.byref(shape), ctypes.byref(view), first, 0x20000000, 0x20000000, N, path, cnt, AT, None, None)


@pytest.mark.parametrize("off", [0, 4, 8, -4, -8])
def test_lengths_over_what_the_call_reads(hg, off):
    for name in ("first", "path", "cnt"):
        assert commit(hg, **{name: AT + off}) == hg.ERR_INVALID_ARG, name
    assert commit(hg, table=0x30000000, first_block=AT + off) == hg.ERR_INVALID_ARG
    assert commit(hg, table=AT + off) == hg.ERR_INVALID_ARG


def test_the_ends_of_path_and_table(hg):
    assert commit(hg, path=AT - 4 * (B * N - 1)) == hg.ERR_INVALID_ARG
    assert commit(hg, table=AT - 4 * (B * BLOCKS - 1)) == hg.ERR_INVALID_ARG
