"""Verification of drafted tokens against the target's probabilities (hgca_verify_drafts).  The results are whole numbers and have to be equal; the
oracle says by what margin its closest decision was taken, relative to the sums: 1e-12 and more is far from what the order of fp64 sums
does (a sum of 2^17 terms is off by 2^17 * 2^-53 = 1.5e-11 of itself at the very most, by 1e-14 as a rule), so inputs are taken as
they come."""
import numpy as np
import pytest

import serve_oracle as so

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def gpu():
    import torch
    assert torch.cuda.is_available(), "these tests need the MI355X"
    from paper_2507_03153_amd import hgca
    hgca.lib()
    return torch, hgca


def i32(torch, a):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(DEV)


def softmax(x):
    e = np.exp(x - x.max(-1, keepdims=True))
    return e / e.sum(-1, keepdims=True)


def bf16(x):
    from draft_oracle import to_bf16
    return to_bf16(x)


def call(gpu, target, draft, tokens, u, u_next, parents=None, dtype="f32", wide=0, stream=None):
    """Numpy in, numpy out; wide: elements between the rows (a padded vocabulary)."""
    torch, hgca = gpu
    B, n, V = target.shape
    dt = torch.float32 if dtype == "f32" else torch.bfloat16

    def put(x):
        if x is None:
            return None
        t = torch.full((B, n, V + wide), float("nan"), dtype=dt, device=DEV)
        t[..., :V] = torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(DEV).to(dt)
        return t[..., :V]

    path, cnt, nxt = (torch.full(s, -77, dtype=torch.int32, device=DEV) for s in ((B, n), (B,), (B,)))
    ws = hgca.verify_workspace(B, V, DEV)
    ws.fill_(0xff)
    f = lambda x: torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(DEV)
    hgca.verify_drafts(put(target), put(draft), i32(torch, tokens), f(u), f(u_next), path, cnt, nxt, ws, parents=i32(torch, parents))
    torch.cuda.synchronize()
    return path.cpu().numpy(), cnt.cpu().numpy(), nxt.cpu().numpy()


def drafted(rng, B, n, V, tree, dtype, sharp=2.5):
    logits = sharp * rng.standard_normal((B, n, V))
    target = softmax(logits + 0.7 * rng.standard_normal((B, n, V))).astype(np.float32)
    draft = softmax(logits).astype(np.float32)
    if dtype == "bf16":
        target, draft = bf16(target), bf16(draft)
    parents = None
    if tree:
        parents = np.zeros((B, n), np.int64)
        for j in range(1, n):
            parents[:, j] = np.maximum(j - 1 - rng.integers(0, min(j, 5), B), 0)
    tokens = np.zeros((B, n), np.int64)
    for b in range(B):
        for j in range(1, n):
            row = draft[b, j - 1 if parents is None else parents[b, j]].astype(np.float64)
            tokens[b, j] = rng.choice(V, p=row / row.sum())
    return target, draft, tokens, parents, rng.random((B, n)).astype(np.float32), rng.random(B).astype(np.float32)


@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("with_q", [True, False])
@pytest.mark.parametrize("dtype,B,n,V,wide", [("f32", 3, 1, 7, 0), ("f32", 16, 5, 100, 0), ("f32", 40, 9, 2049, 3), ("bf16", 16, 6, 5001, 7),
                                              ("f32", 4, 64, 2048, 0), ("bf16", 5, 17, 4096, 0), ("f32", 3, 8, 131071, 1)])
def test_against_64_bits(gpu, dtype, B, n, V, wide, with_q, tree):
    rng = np.random.default_rng(B * 1000 + n + V)
    target, draft, tokens, parents, u, u_next = drafted(rng, B, n, V, tree, dtype)
    if n > 3:                                    # a few that are in no tree
        tokens[0, n - 1], tokens[1, 1], tokens[2, 2] = -1, V, 2 ** 31 - 1
        if parents is not None:
            parents[3 % B, 2], parents[1, 3] = 2, -1
    draft = draft if with_q else None
    want = so.verify(target, draft, tokens, u, u_next, parents)
    got = call(gpu, target, draft, tokens, u, u_next, parents, dtype, wide)
    print(f"\n[case] {dtype} B={B} n={n} V={V} q={with_q} tree={tree}: accepted {want[1].mean():.2f} of {n}, margin {want[3]:.1e}", flush=True)
    for a, b in zip(got, want):
        assert np.array_equal(a, b)


@pytest.mark.parametrize("with_q", [True, False])
def test_many_refusals_at_one_node(gpu, with_q):
    """Eleven children of the root whose random numbers refuse nearly all of them, the same token among them more than once."""
    rng = np.random.default_rng(11)
    B, n, V = 24, 12, 700
    target, draft, tokens, _, u, u_next = drafted(rng, B, n, V, True, "f32", sharp=1.0)
    parents = np.zeros((B, n), np.int64)
    tokens[:, 1:] = np.argsort(-target[:, 0], -1)[:, :n - 1]
    tokens[::3, 5] = tokens[::3, 2]
    u[:, 1:] = 0.9 + 0.0999 * u[:, 1:]
    draft = draft if with_q else None
    want = so.verify(target, draft, tokens, u, u_next, parents)
    got = call(gpu, target, draft, tokens, u, u_next, parents)
    print(f"\n[case] refusals: cnt {want[1].tolist()}, margin {want[3]:.1e}", flush=True)
    for a, b in zip(got, want):
        assert np.array_equal(a, b)


def test_edges_of_the_random_numbers(gpu):
    """u = 0 accepts whatever has probability and refuses what has none; u_next = 0 is the first token that has any, the largest number below 1
    the last or nearly; numbers of 1 and more, which are not asked for, still give a token."""
    V, n = 3000, 3
    target, draft = np.zeros((6, n, V), np.float32), np.zeros((6, n, V), np.float32)
    target[:, :, 10:2990] = 1 / 2980
    draft[:, :, :] = 1 / V
    tokens = np.array([[0, 20, 30], [0, 20, 5], [0, 5, 30], [0, 20, 30], [0, 20, 30], [0, 5, 30]])
    u = np.zeros((6, n), np.float32)
    u_next = np.array([0, 0, 0, 1 - 2.0 ** -24, 1.0, 3.0], np.float32)
    want = so.verify(target, draft, tokens, u, u_next)
    got = call(gpu, target, draft, tokens, u, u_next)
    for a, b in zip(got, want):
        assert np.array_equal(a, b)
    assert got[1].tolist() == [3, 2, 1, 3, 3, 1] and got[2][:3].tolist() == [10, 10, 10] and got[2][4:].tolist() == [2989, 2989]


def test_rows_without_mass(gpu):
    """A row of zeros, of negative numbers, NaN or infinities has no token; a residual without mass is the target itself."""
    V, n = 2500, 2
    target = np.zeros((5, n, V), np.float32)
    target[1] = -1.0
    target[2] = np.nan
    target[3] = np.inf
    target[4, :, [7, 2400]] = 0.5
    draft = np.full((5, n, V), 1 / V, np.float32)
    draft[4] = 1.0                               # larger than the target everywhere: the first refusal leaves nothing
    tokens = np.array([[0, 7]] * 5)
    u, u_next = np.full((5, n), 0.75, np.float32), np.full(5, 0.6, np.float32)
    for q in (draft, None):
        want = so.verify(target, q, tokens, u, u_next)
        got = call(gpu, target, q, tokens, u, u_next)
        for a, b in zip(got, want):
            assert np.array_equal(a, b)
        assert got[2][:4].tolist() == [-1] * 4 and got[2][4] == 2400


def test_samples_are_the_targets(gpu):
    """Speculative sampling leaves the target's distribution as it is: over 20 000 draws of the first token after the root, by a chain and by three children of
    the root, counts are within 5 standard deviations of the target's for each of 8 tokens (16 counts: one in 10^5 by chance)."""
    rng = np.random.default_rng(0)
    B, V = 20000, 8
    p, q = softmax(rng.standard_normal(V)), softmax(1.5 * rng.standard_normal(V))
    for n, parents in ((2, None), (4, np.zeros((B, 4), np.int64))):
        target, draft = np.broadcast_to(p, (B, n, V)).astype(np.float32), np.broadcast_to(q, (B, n, V)).astype(np.float32)
        tokens = rng.choice(V, size=(B, n), p=q)
        path, cnt, nxt = call(gpu, target, draft, tokens, rng.random((B, n)), rng.random(B), parents)
        first = np.where(cnt > 1, tokens[np.arange(B), np.maximum(path[:, 1], 0)], nxt)
        counts, expect = np.bincount(first, minlength=V), p * B
        print("[counts]", counts, expect.round(), flush=True)
        assert (np.abs(counts - expect) <= 5 * np.sqrt(expect * (1 - p))).all()


def test_strides_and_a_vocabulary_of_one(gpu):
    torch, hgca = gpu
    one = np.ones((2, 3, 1), np.float32)
    got = call(gpu, one, one, np.zeros((2, 3)), np.full((2, 3), 0.5), np.full(2, 0.5))
    assert got[0].tolist() == [[0, 1, 2]] * 2 and got[2].tolist() == [0, 0]
    # the distributions of every second sequence and of the first tokens of a longer tensor
    rng = np.random.default_rng(8)
    target, draft, tokens, parents, u, u_next = drafted(rng, 3, 4, 900, True, "f32")
    big = torch.full((6, 9, 900), float("nan"), device=DEV)
    big[::2, :4] = torch.from_numpy(target).to(DEV)
    path, cnt, nxt = (torch.empty(s, dtype=torch.int32, device=DEV) for s in ((3, 4), (3,), (3,)))
    hgca.verify_drafts(big[::2, :4], torch.from_numpy(draft).to(DEV), i32(torch, tokens), torch.from_numpy(u).to(DEV),
                       torch.from_numpy(u_next).to(DEV), path, cnt, nxt, hgca.verify_workspace(3, 900, DEV), parents=i32(torch, parents))
    want = so.verify(target, draft, tokens, u, u_next, parents)
    for a, b in zip((path, cnt, nxt), want):
        assert np.array_equal(a.cpu().numpy(), b)


def test_captured_and_replayed(gpu):
    """One graph, other distributions and random numbers at every replay, eager work between them."""
    torch, hgca = gpu
    B, n, V = 5, 7, 5000
    bufs = dict(target=torch.zeros(B, n, V, device=DEV), draft=torch.zeros(B, n, V, device=DEV), tokens=torch.zeros(B, n, dtype=torch.int32, device=DEV),
                u=torch.zeros(B, n, device=DEV), u_next=torch.zeros(B, device=DEV), path_out=torch.zeros(B, n, dtype=torch.int32, device=DEV),
                cnt_out=torch.zeros(B, dtype=torch.int32, device=DEV), next_out=torch.zeros(B, dtype=torch.int32, device=DEV),
                ws=hgca.verify_workspace(B, V, DEV), parents=torch.zeros(B, n, dtype=torch.int32, device=DEV))
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    for turn in range(5):
        target, draft, tokens, parents, u, u_next = drafted(np.random.default_rng(turn), B, n, V, True, "f32")
        for k, x in (("target", target), ("draft", draft), ("u", u), ("u_next", u_next), ("tokens", tokens.astype(np.int32)), ("parents", parents.astype(np.int32))):
            bufs[k].copy_(torch.from_numpy(x))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            if turn == 0:
                hgca.verify_drafts(**bufs)
            else:
                if turn == 1:
                    with torch.cuda.graph(graph, stream=side):
                        hgca.verify_drafts(**bufs)
                graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((bufs["path_out"], bufs["cnt_out"], bufs["next_out"]), so.verify(target, draft, tokens, u, u_next, parents)):
            assert np.array_equal(a.cpu().numpy(), b)
        bufs["target"].sum()
        torch.cuda.synchronize()


@pytest.mark.parametrize("with_q", [True, False])
@pytest.mark.parametrize("dtype,B", [("f32", 5), ("bf16", 20)])
def test_refusals_over_a_large_vocabulary(gpu, dtype, B, with_q):
    """Rows of more than 65536 elements: four children of every node, with random numbers that refuse none, one, ... all of them, here and at the
    accepted child, the same token twice; from no pass over the rows but the last to more than there are launches for."""
    rng = np.random.default_rng(B)
    n, V = 13, 66003
    target, draft, tokens, _, u, u_next = drafted(rng, B, n, V, True, dtype, sharp=1.5)
    parents = np.tile(np.array([0, 0, 0, 0, 0, 1, 1, 1, 3, 3, 3, 9, 9]), (B, 1))
    for j in range(1, n):
        tokens[:, j] = [np.argsort(-target[b, parents[b, j]])[(3 * j + b) % 7] for b in range(B)]
    tokens[::2, 4] = tokens[::2, 2]
    for b in range(B):
        u[b, 1:1 + b % 5] = 0.9999                                             # the root's first b % 5 children are refused
        u[b, 1 + b % 5:5] = 1e-9
        u[b, 5:8] = u[b, 8:] = 0.9999 if b % 3 else 1e-9
    draft = draft if with_q else None
    want = so.verify(target, draft, tokens, u, u_next, parents)
    got = call(gpu, target, draft, tokens, u, u_next, parents, dtype, 5)
    print(f"\n[case] {dtype} B={B} q={with_q}: cnt {want[1].tolist()}, margin {want[3]:.1e}", flush=True)
    for a, b in zip(got, want):
        assert np.array_equal(a, b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [2, 3, 4, 5, 7, 8, 9, 250, 1022, 1023, 1024, 1025, 1027, 2050, 33001, 66005])
def test_ends_of_rows_and_odd_elements(gpu, dtype, V):
    """Rows of every alignment, ends inside a load, elements that do not count among them; draws from the first to the last token of the row, with a chain
    that stops anywhere in it."""
    rng = np.random.default_rng(V)
    B, n = 24, 4
    target, draft, tokens, _, u, u_next = drafted(rng, B, n, V, False, dtype, sharp=1.0)
    for x in (target, draft):
        where = rng.random(x.shape) < min(0.1, 20 / V)
        x[where] = rng.choice(np.array([-1.0, -0.0, np.inf, -np.inf, np.nan, -1e-30], np.float32), int(where.sum()))
    target[:, :, -1] = 0.25                      # drawn by the numbers near 1
    u[:, 1:] = np.where(rng.random((B, n - 1)) < 0.5, 0.999, u[:, 1:])
    u_next[:8] = 1 - 2.0 ** -np.arange(1, 9)
    u_next[8] = 0
    for q in (draft, None):
        want = so.verify(target, q, tokens, u, u_next)
        got = call(gpu, target, q, tokens, u, u_next, None, dtype, wide=int(rng.integers(0, 4)))
        print(f"\n[case] V={V} {dtype}: cnt {np.bincount(want[1]).tolist()}, last token {int((want[2] == V - 1).sum())}, margin {want[3]:.1e}", flush=True)
        for a, b in zip(got, want):
            assert np.array_equal(a, b)
