"""Which tensors the norm with rotation takes as rows of tokens, without a GPU: the distance of tokens that the library is given is
that of the tensor's own storage."""
import pytest
import torch

B, n, H, d = 4, 5, 8, 128


@pytest.fixture(scope="module")
def hg():
    from paper_2507_03153_amd import hgca
    return hgca


@pytest.mark.parametrize("batch,tokens", [(1, n), (B, 1), (B, n)])
def test_a_row_that_stands_for_many_is_refused(hg, batch, tokens):
    """An expanded token has a distance of 0, which the library takes as rows one behind the other."""
    one = torch.zeros(1, 1, H, d, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="side by side"):
        hg._token_stride("q", one.expand(batch, tokens, H, d))


def test_rows_that_overlap_are_refused(hg):
    x = torch.zeros(B * n * H * d)
    for step in (d, (H - 1) * d):
        with pytest.raises(ValueError, match="side by side"):
            hg._token_stride("q", x.as_strided((1, n, H, d), (0, step, d, 1)))
        with pytest.raises(ValueError, match="side by side"):
            hg._token_stride("q", x.as_strided((B, 1, H, d), (step, 0, d, 1)))


def test_only_one_of_two_dimensions_is_expanded(hg):
    x = torch.zeros(1, n, H, d)
    with pytest.raises(ValueError, match="side by side"):
        hg._token_stride("q", x.expand(B, n, H, d))
    with pytest.raises(ValueError, match="side by side"):
        hg._token_stride("q", x.transpose(0, 1)[:B].expand(B, n, H, d))


def test_what_is_taken(hg):
    dense = torch.zeros(B, n, H, d)
    assert hg._token_stride("q", dense) == H * d
    assert hg._token_stride("q", dense[:, :1]) == n * H * d                    # one token of each sequence
    assert hg._token_stride("q", torch.zeros(1, 1, H, d).expand(1, 1, H, d)) == H * d
    assert hg._token_stride("q", torch.zeros(B, n, 3 * H * d)[..., :H * d].unflatten(-1, (H, d))) == 3 * H * d
    assert hg._token_stride("k", torch.zeros(B, n, 1, d)) == d
    assert hg._token_stride("q", torch.zeros(1, 1, H, d).expand(B, 0, H, d)) >= 0          # no rows at all
