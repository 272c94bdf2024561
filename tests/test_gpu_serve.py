"""The calls of a server's step as they are used together: blocks planned, rows written, packed chunks attended to, drafts attended to, verified and
committed, blocks given back; eagerly, in a captured graph, on another stream; and what the binding refuses."""
import numpy as np
import pytest

import draft_oracle as do
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
    return torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(DEV)


class Server:
    """One layer's paged cache of B requests, on the GPU and as plain rows."""

    def __init__(self, gpu, B=3, Hq=8, Hkv=2, d=64, bs=16, row=20, n_blocks=70, most=256):
        torch, hgca = gpu
        self.torch, self.hgca, self.B, self.Hq, self.Hkv, self.d, self.bs = torch, hgca, B, Hq, Hkv, d, bs
        self.rng = np.random.default_rng(0)
        self.scale = float(np.float32(d ** -0.5))
        z = lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEV)
        self.state = hgca.BlockState(torch.full((B, row), -1, dtype=torch.int32, device=DEV), z(B), z(B), torch.randperm(n_blocks).to(torch.int32).to(DEV),
                                     torch.tensor([n_blocks], dtype=torch.int32, device=DEV), bs, status=z(1))
        kv = lambda: torch.full((n_blocks, Hkv, bs, d), float("nan"), dtype=torch.bfloat16, device=DEV)
        self.tier = hgca.Tier(kv(), kv(), row * bs, self.state.lens, self.state.block_table, bs)
        self.shape = hgca.Shape(hgca.BF16, B, Hq, Hkv, d, self.scale)
        self.cu, self.pos, self.slots = z(B + 1), z(most), z(most)
        self.most = most
        self.ws = hgca.chunk_workspace(self.shape, most, row * bs, DEV)
        self.o = torch.zeros(most, Hq, d, device=DEV)
        self.lse = torch.zeros(most, Hq, device=DEV)
        self.q, self.k, self.v = (torch.zeros(most, h, d, dtype=torch.bfloat16, device=DEV) for h in (Hq, Hkv, Hkv))
        self.n_new = z(B)
        self.K = [np.zeros((Hkv, 0, d)) for _ in range(B)]       # the plain side: rows of every request
        self.V = [np.zeros((Hkv, 0, d)) for _ in range(B)]

    def launch(self, stream=None, **opt):
        h = self.hgca
        h.kv_plan(self.state, self.n_new, self.cu, self.pos, self.slots, stream=stream)
        h.kv_write(self.shape, self.tier, self.slots, self.k, self.v, stream=stream)
        h.chunk_attn(self.shape, self.q, self.cu, self.tier, self.o, self.lse, self.ws, cap=30.0, stream=stream, **opt)

    def inputs(self, counts):
        T, r = sum(counts), lambda h: do.to_bf16(self.rng.standard_normal((self.most, h, self.d)))
        self.host = [r(self.Hq), r(self.Hkv), r(self.Hkv)]
        for t, a in zip((self.q, self.k, self.v), self.host):
            t.copy_(self.torch.from_numpy(a))
        self.n_new.copy_(i32(self.torch, counts))

    def check(self, counts):
        at = 0
        for b, n in enumerate(counts):
            self.K[b] = np.concatenate([self.K[b], self.host[1][at:at + n].transpose(1, 0, 2)], 1)
            self.V[b] = np.concatenate([self.V[b], self.host[2][at:at + n].transpose(1, 0, 2)], 1)
            at += n
        lens = [k.shape[1] for k in self.K]
        assert self.state.lens.tolist() == lens and int(self.state.status) == 0
        cap = max(lens + [1])
        K, V = (np.stack([np.pad(x, ((0, 0), (0, cap - x.shape[1]), (0, 0))) for x in y]) for y in (self.K, self.V))
        cu = np.concatenate([[0], np.cumsum(counts)])
        assert self.cu.tolist() == cu.tolist()
        O, L = so.chunk(self.host[0][:at], cu, K, V, lens, self.scale, cap=30.0)
        # fp32 results of bf16 rows: as in the tests of the attention itself, 2e-6 of the output and twice what the cap adds
        o = self.o[:at].double().cpu().numpy()
        assert np.linalg.norm(o - O) <= (2e-6 + 2 * 30 * 4.9e-7) * max(np.linalg.norm(O), 1e-30)
        assert np.abs(self.lse[:at].double().cpu().numpy() - L).max(initial=0) <= 1e-4


def test_requests_of_different_size(gpu):
    torch, hgca = gpu
    S = Server(gpu)
    for counts in ([40, 0, 17], [1, 64, 1], [1, 1, 1], [130, 1, 1], [0, 0, 0], [1, 1, 60]):
        S.inputs(counts)
        S.launch()
        torch.cuda.synchronize()
        S.check(counts)


def test_a_captured_step_replayed(gpu):
    """Plan, write and attention in one graph, replayed with other counts and rows between eager steps and synchronizations: the lengths live on the
    device, so each replay goes on where the last step ended."""
    torch, hgca = gpu
    S, E = Server(gpu), Server(gpu)
    E.state.free_blocks.copy_(S.state.free_blocks)
    side = torch.cuda.Stream()
    steps = [[5, 1, 30], [1, 1, 1], [33, 2, 1], [1, 100, 0], [7, 7, 7], [1, 1, 1]]
    graph = torch.cuda.CUDAGraph()
    for i, counts in enumerate(steps):
        for x in (S, E):
            x.rng = np.random.default_rng(100 + i)
            x.inputs(counts)
        if i == 0:                               # the first step eagerly, as a warm-up
            with torch.cuda.stream(side):
                S.launch()
        elif i == 1:
            with torch.cuda.stream(side):
                with torch.cuda.graph(graph, stream=side):
                    S.launch()
                graph.replay()
        else:
            graph.replay()
        E.launch()
        torch.cuda.synchronize()
        S.check(counts)
        T = sum(counts)
        assert torch.equal(S.o[:T], E.o[:T]) and torch.equal(S.slots, E.slots) and torch.equal(S.pos, E.pos)
        torch.ones(1 << 20, device=DEV).sum()    # other work between the replays
        torch.cuda.synchronize()


def test_on_another_stream(gpu):
    """Everything on a stream that is not the current one: the results are there once that stream has been waited for."""
    torch, hgca = gpu
    S = Server(gpu)
    side = torch.cuda.Stream()
    for counts in ([40, 3, 17], [1, 1, 1]):
        S.inputs(counts)
        torch.cuda.synchronize()
        S.launch(stream=side)
        side.synchronize()
        S.check(counts)


def test_a_step_with_drafts(gpu):
    """A prompt, then rounds of drafts: their rows are planned and written like any other, tree attention sees them, verification picks the path, the commit
    moves the accepted ones together, the release gives back what is behind.  The cache always holds what the accepted tokens' rows are."""
    torch, hgca = gpu
    S = Server(gpu)
    B, n, V, rng = S.B, 6, 300, np.random.default_rng(9)
    counts = [33, 16, 5]
    S.inputs(counts)
    S.launch()
    torch.cuda.synchronize()
    S.check(counts)
    parents = np.array([[0, 0, 0, 1, 1, 3]] * B)
    masks = [0] * n
    for i in range(n):
        masks[i] = (masks[parents[0][i]] if i else 0) | 1 << i
    mask = torch.tensor([masks] * B, dtype=torch.int64, device=DEV)
    path, cnt, nxt = (torch.zeros(s, dtype=torch.int32, device=DEV) for s in ((B, n), (B,), (B,)))
    o, lse = torch.zeros(B, n, S.Hq, S.d, device=DEV), torch.zeros(B, n, S.Hq, device=DEV)
    ws_tree, ws = hgca.tree_workspace(S.shape, n, S.tier.cap, DEV), hgca.verify_workspace(B, V, DEV)
    first = torch.zeros(B, dtype=torch.int32, device=DEV)
    for turn in range(5):
        q, k, v = (do.to_bf16(rng.standard_normal((B, n, h, S.d))) for h in (S.Hq, S.Hkv, S.Hkv))
        target, draft = (rng.dirichlet(np.full(V, 0.1), (B, n)).astype(np.float32) for _ in range(2))
        draft = (0.5 * draft + 0.5 * target).astype(np.float32)
        tokens = np.stack([[rng.choice(V, p=draft[b, parents[b][i]].astype(np.float64) / draft[b, parents[b][i]].astype(np.float64).sum()) for i in range(n)]
                           for b in range(B)])
        u, un = rng.random((B, n)).astype(np.float32), rng.random(B).astype(np.float32)
        put = lambda x: torch.from_numpy(x).to(DEV).to(torch.bfloat16)
        kt, vt = put(k), put(v)
        first.copy_(S.state.lens)
        S.n_new.fill_(n)
        hgca.kv_plan(S.state, S.n_new, S.cu, S.pos, S.slots)
        hgca.kv_write(S.shape, S.tier, S.slots[:B * n], kt.view(B * n, S.Hkv, S.d), vt.view(B * n, S.Hkv, S.d))
        hgca.tree_attn(S.shape, put(q), S.tier, mask, o, lse, ws_tree)
        f = lambda x: torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(DEV)
        hgca.verify_drafts(f(target), f(draft), i32(torch, tokens), f(u), f(un), path, cnt, nxt, ws, parents=i32(torch, parents))
        hgca.kv_commit(S.shape, S.tier, first, kt, vt, S.state.lens, path=path, cnt=cnt)
        hgca.kv_release(S.state, S.state.lens)
        torch.cuda.synchronize()
        want = so.verify(target, draft, tokens, u, un, parents)
        for a, b in zip((path, cnt, nxt), want):
            assert np.array_equal(a.cpu().numpy(), b)
        lens = [x.shape[1] for x in S.K]
        Kd, Vd = (np.stack([np.pad(np.concatenate([x, new.transpose(1, 0, 2)], 1), ((0, 0), (0, 400 - x.shape[1] - n), (0, 0))) for x, new in zip(old, rows)])
                  for old, rows in ((S.K, k), (S.V, v)))
        O, _ = do.rows_attention(q, Kd, Vd, [x + n for x in lens], S.scale, [masks] * B)
        assert np.linalg.norm(o.double().cpu().numpy() - O) <= 2e-6 * np.linalg.norm(O)
        for b in range(B):
            take = [int(x) for x in want[0][b] if x >= 0]
            S.K[b] = np.concatenate([S.K[b], k[b, take].transpose(1, 0, 2)], 1)
            S.V[b] = np.concatenate([S.V[b], v[b, take].transpose(1, 0, 2)], 1)
        lens = [x.shape[1] for x in S.K]
        assert S.state.lens.tolist() == lens and S.state.held.tolist() == [-(-x // S.bs) for x in lens]
        assert int(S.state.free_count) + sum(S.state.held.tolist()) == S.state.free_blocks.numel()
    # a token each reads it all back
    counts = [1, 1, 1]
    S.inputs(counts)
    S.launch()
    torch.cuda.synchronize()
    S.check(counts)


def test_two_calls_at_once(gpu):
    """Two streams with states and workspaces of their own."""
    torch, hgca = gpu
    X, Y = Server(gpu), Server(gpu)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    Y.rng = np.random.default_rng(5)
    for counts, other in (([100, 50, 20], [3, 90, 64]), ([1, 1, 1], [1, 0, 2])):
        X.inputs(counts)
        Y.inputs(other)
        torch.cuda.synchronize()
        X.launch(stream=a)
        Y.launch(stream=b)
        torch.cuda.synchronize()
        X.check(counts)
        Y.check(other)


def test_the_binding_refuses(gpu):
    torch, hgca = gpu
    S = Server(gpu)
    S.inputs([2, 2, 2])
    z = lambda *s: torch.zeros(*s, dtype=torch.int32, device=DEV)
    bad = [lambda: hgca.kv_plan(S.state, z(4), S.cu, S.pos, S.slots), lambda: hgca.kv_plan(S.state, z(3).long(), S.cu, S.pos, S.slots),
           lambda: hgca.kv_plan(S.state, S.n_new, z(3), S.pos, S.slots), lambda: hgca.kv_plan(S.state, S.n_new, S.cu, S.pos, S.slots[:-1]),
           lambda: hgca.kv_plan(S.state, S.n_new.cpu(), S.cu, S.pos, S.slots), lambda: hgca.kv_release(S.state, z(2)),
           lambda: hgca.kv_write(S.shape, S.tier, S.slots[:6], S.k[:5], S.v[:6]), lambda: hgca.kv_write(S.shape, S.tier, S.slots[:6], S.k[:6].float(), S.v[:6]),
           lambda: hgca.kv_write(S.shape, S.tier, S.slots[:6], S.k[:6].transpose(0, 1).contiguous().transpose(0, 1), S.v[:6]),
           lambda: hgca.chunk_attn(S.shape, S.q, S.cu[:3], S.tier, S.o, S.lse, S.ws), lambda: hgca.chunk_attn(S.shape, S.q[:9], S.cu, S.tier, S.o, S.lse, S.ws),
           lambda: hgca.chunk_attn(S.shape, S.q, S.cu, S.tier, S.o, S.lse, S.ws, slopes=torch.zeros(3, device=DEV)),
           lambda: hgca.chunk_attn(S.shape, S.q, S.cu, S.tier, S.o, S.lse, S.ws, prefix_lens=z(4)),
           lambda: hgca.chunk_attn(S.shape, S.q, S.cu, S.tier, S.o, S.lse, S.ws, first=z(3))]
    P = torch.full((2, 3, 50), 0.02, device=DEV)
    v = dict(target=P, draft=P, tokens=z(2, 3), u=torch.zeros(2, 3, device=DEV), u_next=torch.zeros(2, device=DEV), path_out=z(2, 3), cnt_out=z(2), next_out=z(2),
             ws=hgca.verify_workspace(2, 50, DEV))
    for k, x in (("draft", P.bfloat16()), ("draft", P[:, :2]), ("tokens", z(2, 4)), ("u", torch.zeros(2, 3, device=DEV).double()), ("u_next", torch.zeros(3, device=DEV)),
                 ("path_out", z(3, 2)), ("cnt_out", z(3)), ("next_out", z(1)), ("target", P[:1].expand(2, 3, 50)), ("target", P.transpose(1, 2).contiguous().transpose(1, 2)),
                 ("target", P.cpu())):
        bad.append(lambda k=k, x=x: hgca.verify_drafts(**{**v, k: x}))
    for f in bad:
        with pytest.raises(ValueError):
            f()
    for f in (lambda: hgca.chunk_attn(S.shape, S.q, S.cu, S.tier, S.o, S.lse, S.ws[:64]), lambda: hgca.chunk_attn(S.shape, S.q, S.cu, S.tier, S.o, S.lse, S.ws, window=-1),
              lambda: hgca.verify_drafts(**{**v, "ws": v["ws"][:8]})):
        with pytest.raises(hgca.HgcaError):
            f()
    torch.cuda.synchronize()
