"""What comes out of the verification of drafted tokens (hgca_verify_drafts) is distributed as the target's samples where the call says so, and is not
where it says so.  20 000 draws: counts within 5 standard deviations for each of 8 tokens (one in 10^5 by chance), or one of them
beyond 10."""
import numpy as np
import pytest

from test_gpu_verify import call, gpu, softmax  # noqa: F401

pytestmark = pytest.mark.gpu
B, V = 20000, 8


def first_token(gpu, p, q, tokens, rng):  # noqa: F811
    """Counts of the token that follows the root, all others being its children; q None: without draft rows."""
    n = tokens.shape[1]
    rows = lambda x: None if x is None else np.broadcast_to(x, (B, n, V)).astype(np.float32)
    path, cnt, nxt = call(gpu, rows(p), rows(q), tokens, rng.random((B, n)), rng.random(B), np.zeros((B, n), np.int64))
    first = np.where(cnt > 1, tokens[np.arange(B), np.maximum(path[:, 1], 0)], nxt)
    counts, expect = np.bincount(first, minlength=V), p * B
    print("\n[counts]", counts, expect.round(), flush=True)
    return np.abs(counts - expect) / np.sqrt(expect * (1 - p))


def distributions(seed):
    rng = np.random.default_rng(seed)
    return rng, softmax(rng.standard_normal(V)), softmax(1.5 * rng.standard_normal(V))


def ranked(q, n):
    """The root and the n likeliest tokens, the same ones for every sequence."""
    return np.tile(np.concatenate([[0], np.argsort(-q)[:n]]), (B, 1))


@pytest.mark.parametrize("children", [1, 2, 4, 8])
def test_likeliest_tokens_without_draft_rows(gpu, children):  # noqa: F811
    rng, p, q = distributions(children)
    assert (first_token(gpu, p, None, ranked(q, children), rng) <= 5).all()


@pytest.mark.parametrize("children", [1, 3, 6])
def test_draws_with_replacement_and_draft_rows(gpu, children):  # noqa: F811
    rng, p, q = distributions(children)
    assert (first_token(gpu, p, q, rng.choice(V, size=(B, children + 1), p=q), rng) <= 5).all()


def test_likeliest_tokens_with_their_row_are_biased(gpu):  # noqa: F811
    rng, p, q = distributions(2)
    assert first_token(gpu, p, q, ranked(q, 3), rng).max() > 10
