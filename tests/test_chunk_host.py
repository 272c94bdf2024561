"""Flags of packed chunks (hgca_chunk_attn), without a GPU: what is accepted ends at the missing workspace."""
from test_serve_host import chunk, hg  # noqa: F401


def test_flags(hg):  # noqa: F811
    assert (hg.CHUNK_CAUSAL, hg.CHUNK_ONE_PART_P) == (1, 4)
    for flags in (0, 1, 4, 5):
        assert chunk(hg, flags=flags, ws=None) == hg.ERR_WORKSPACE
    for flags in (2, 3, 6, 8, 9, -1):
        assert chunk(hg, flags=flags, ws=None) == hg.ERR_INVALID_ARG
