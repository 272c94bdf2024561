"""Overlaps of hgca_kv_write where the slots are not whole blocks, without a GPU: the heads of a block lie one behind the other, so its rows reach
to the block's end however few of its slots count."""
from test_serve_host import at, hg, shape, view, write  # noqa: F401


def test_rows_reach_to_the_end_of_the_last_block(hg):  # noqa: F811
    I, U = hg.ERR_INVALID_ARG, hg.ERR_UNSUPPORTED
    # 2 heads of 128 in bf16: 512 bytes a slot; a contiguous tier of 2 x 64 and one of blocks of 16
    for kv, n_slots, rows in ((dict(), 40, 64), (dict(), 100, 128), (dict(table=1 << 20, bs=16, mb=4), 40, 48), (dict(table=1 << 20, bs=16, mb=4), 1, 16)):
        tier = view(hg, k=at(3), v=at(4), **kv)
        assert write(hg, kv=tier, n_slots=n_slots, k=at(3) + 512 * rows - 16) == I
        assert write(hg, kv=tier, n_slots=n_slots, v=at(4) + 512 * rows - 16) == I
        assert write(hg, kv=view(hg, k=at(3), v=at(3) + 512 * rows - 16, **kv), n_slots=n_slots) == I
    assert write(hg, n_slots=(1 << 31)) in (I, U)
