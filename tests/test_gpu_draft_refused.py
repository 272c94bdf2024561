"""Draft steps that a sequence has no room for: what the device leaves out has no result and is not committed."""
import numpy as np
import pytest

import draft_oracle as do
from test_gpu_draft_checks import B, BS, drafts, make
from test_gpu_tree import bounds, gpu, i32, put  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("given", [True, False])
@pytest.mark.parametrize("pool8", [True, False])
def test_a_sequence_at_the_end_of_its_table_row(gpu, pool8, given):
    """The first sequence fills its 64 positions and is refused from then on; the second one goes on as if alone, and so does the
    first one with as few drafts as it has room for."""
    torch, hgca = gpu
    rng = np.random.default_rng(5)
    C = make(torch, pool8)
    host = lambda t: t.float().cpu().numpy().astype(np.float64)
    rows, refused = [[], []], 0
    sizes = [9] * 8 + [1, 9] if given else [18, 18, 18, 18, 1]
    for n in sizes:
        q, k, v, masks, mask, path = drafts(torch, rng, n)
        cnt = [n, min(2, n)] if given else [n, n]
        C.draft_step(q, k, v, mask)
        torch.cuda.synchronize()
        room = [len(x) + n <= 4 * BS for x in rows]
        o, lse = C.o_draft.double().cpu().numpy(), C.lse_draft.double().cpu().numpy()
        qh, kh, vh, pool = host(q), host(k), host(v), C.pool_lens.tolist()
        for b in range(B):
            if not room[b]:
                refused += 1
                assert (o[b] == 0).all() and np.isneginf(lse[b]).all()
                continue
            K, V = (np.stack([x[j] for x in rows[b]] + [y[b, i] for i in range(n)], 1)[None] for j, y in ((0, kh), (1, vh)))
            if pool8 and pool[b]:
                for x in (K, V):
                    x[:, :, :pool[b]] = do.decode(*do.encode(x[:, :, :pool[b]]))
            T = K.shape[2]
            O, L = do.rows_attention(qh[b:b + 1], K, V, [T], 0.125, masks[b:b + 1])
            tol_o, tol_l = bounds(qh[b:b + 1], K, V, [T], 0.125, T)
            # the append stage's weights have two parts, 2^-17 each; a merge of two parts adds 8 roundings, counted by `bounds`
            assert np.abs(o[b:b + 1] - O).max() <= tol_o + 2.0 ** -16 * np.abs(V).max() and np.abs(lse[b:b + 1] - L).max() <= tol_l
        before = [x.clone() for x in (C.k_blocks, C.v_blocks)]
        C.commit(k, v, path, i32(torch, cnt) if given else None, beta=1.0)
        torch.cuda.synchronize()
        for b in range(B):
            if room[b]:
                rows[b] += [(kh[b, i], vh[b, i]) for i in range(cnt[b])]
            else:
                blocks = C.block_table[b].long()
                assert all(torch.equal(x[blocks], y[blocks]) for x, y in zip((C.k_blocks, C.v_blocks), before))
        assert (C.win_lens + C.pool_lens).tolist() == [len(x) for x in rows]
        assert bool(C.status.item() & hgca.CACHE_CONTEXT_FULL) == (refused > 0)
    assert refused >= 2 and len(rows[0]) > 54


def test_captured_steps_with_a_full_sequence(gpu):
    """A graph of a draft step and its commit, replayed until one sequence is full and beyond."""
    torch, hgca = gpu
    rng = np.random.default_rng(7)
    n, G, E = 5, make(torch, True), make(torch, True)
    q, k, v, _, mask, path = drafts(torch, rng, n)
    cnt = i32(torch, [5, 1])

    def step(C):
        C.draft_step(q, k, v, mask)
        C.commit(k, v, path, cnt, 1.0)
    step(G), step(E)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(G)
    for r in range(18):
        for t in (q, k, v):
            t.copy_(put(torch, rng.standard_normal(t.shape), "bf16"))
        graph.replay()
        step(E)
        torch.cuda.synchronize()
        assert torch.equal(G.o_draft, E.o_draft) and torch.equal(G.lse_draft, E.lse_draft)
        assert torch.equal(G.win_lens, E.win_lens) and torch.equal(G.pool_lens, E.pool_lens)
    assert (G.win_lens + G.pool_lens).tolist() == [60, 19] and (G.lse_draft[0] == -float("inf")).all()
