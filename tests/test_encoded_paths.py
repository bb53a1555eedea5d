"""Attention over position-encoded keys by the way its rows are shared out: the single-token kernel and the tiled one, whole, in two
parts that the last workgroup joins, in more that a launch joins; on both sides of the rule between the kernels.  Each case names the plan
it is meant for, which the library's own planner confirms; tokens at random places are held against 64 bits, by the bound of the kernel
that ran."""
import ctypes

import pytest
import torch

import paper_2603_23516_amd as msa
import plain64 as P
from probe_build import build_probe

PAIRS, SINGLE = 2.0 ** -16, 2.0 ** -8          # softmax weights as bf16 (hi, lo) pairs, or as one bf16


@pytest.fixture(scope="module")
def plan():
    fn = ctypes.CDLL(build_probe(force=False)).probe_encoded_plan
    i, ll = ctypes.c_int, ctypes.c_longlong
    fn.argtypes, fn.restype = [i, i, i, i, i, ll, i, ll, i], i
    return fn


# parts: of the single-token kernel, negative: of the tiled kernel
WINDOW = [                                     # Hq, Hkv, d, B, M, L, W, S, parts
    (32, 8, 128, 8, 3, 4096, 4096, 0, 2),      # fewer than four tokens: one by one
    (32, 8, 128, 8, 4, 4096, 4096, 0, -13),    # four: together
    (32, 8, 128, 8, 9, 4096, 4090, 2, -8),
    (32, 8, 128, 2, 5, 4096, 4096, 4, -32),
    (32, 8, 128, 1, 13, 2048, 2048, 0, 4),     # just below the rule's border ...
    (32, 8, 128, 1, 14, 2048, 2048, 0, -16),   # ... and above
    (8, 8, 64, 1, 13, 2048, 2048, 0, 4),
    (8, 8, 64, 1, 31, 2048, 1500, 7, -13),
    (32, 8, 128, 16, 8, 200, 200, 3, -1),      # thin tiles, whole
    (8, 8, 64, 40, 7, 100, 90, 3, -1),
    (24, 8, 64, 40, 4, 200, 200, 3, -1),
    (24, 8, 64, 16, 8, 600, 600, 3, -2),       # thin tiles in two parts
    (16, 2, 128, 64, 13, 600, 600, 3, -2),
    (6, 2, 64, 1, 20, 500, 400, 3, 3),         # 20 tokens one by one: weights in pairs
    (24, 8, 64, 1, 700, 700, 100, 0, -1),      # three heads to a group, whole
    (24, 8, 64, 1, 300, 900, 900, 0, -2),
]
ATTEND4 = [                                    # Hq, Hkv, d, B, M, k, G, L, scope, parts (shared selections)
    (32, 8, 128, 16, 8, 2, 8, 200, 0, -1),
    (24, 8, 64, 16, 13, 5, 33, 100, 1, -1),
    (32, 8, 128, 16, 31, 4, 64, 0, 0, -1),
    (24, 8, 64, 16, 20, 8, 64, 100, 1, -2),
    (32, 8, 128, 8, 9, 9, 33, 1000, 0, -7),
    (16, 8, 64, 10, 16, 5, 64, 700, 1, -6),
    (8, 1, 64, 5, 24, 20, 100, 1800, 0, -24),
    (32, 8, 128, 1, 8, 6, 100, 2000, 0, 4),    # eight tokens one by one
    (8, 2, 64, 1, 31, 6, 33, 200, 1, 1),       # 31, whole
    (32, 8, 128, 1, 300, 6, 64, 300, 1, -2),   # documents, two parts joined by the last workgroup
    (16, 8, 64, 2, 512, 8, 128, 512, 0, -2),
    (24, 8, 64, 1, 700, 7, 100, 100, 1, -2),
    (32, 8, 128, 1, 100, 8, 128, 100, 0, -6),
    (32, 8, 128, 3, 400, 2, 30, 50, 1, -1),
]


def _window_parts(plan, Hq, Hkv, d, B, M, L, W, S):
    return plan(Hq, Hkv, d, B, M, 0, 0, min(W + S, L), L)


def _attend4_parts(plan, Hq, Hkv, d, B, M, k, G, L, pool=1):
    return plan(Hq, Hkv, d, B, M, k * G, pool, L, L)


def test_plans_are_those_the_cases_are_meant_for(plan):
    got = [_window_parts(plan, *c[:8]) for c in WINDOW], [_attend4_parts(plan, *c[:8]) for c in ATTEND4]
    assert got == ([c[8] for c in WINDOW], [c[9] for c in ATTEND4])


@pytest.mark.parametrize("Hq, Hkv, d", [(32, 8, 128), (8, 1, 64), (8, 8, 64), (24, 8, 64)])
def test_more_rows_stay_with_the_tiled_kernel(plan, Hq, Hkv, d):
    """Once a number of tokens goes through the tiled kernel it does with more documents, a longer context or a longer window."""
    for B, M in ((1, 4), (1, 8), (2, 9), (8, 8), (8, 31), (40, 16)):
        for L in (0, 500, 3297, 3360):
            tiled = [plan(Hq, Hkv, d, B, M, rows, 1, L, L) < 0 for rows in range(1, 20000, 13)]
            assert tiled == sorted(tiled), (B, M, L)
        tiled = [plan(Hq, Hkv, d, B, M, 0, 0, L, L) < 0 for L in range(1, 20000, 13)]
        assert tiled == sorted(tiled), (B, M)


def _normal(g, *shape):
    return torch.randn(shape, generator=g).to(torch.bfloat16)


def _positions(g, B, M, L, pos0):
    """The last tokens of every sequence, of different lengths; some anywhere, some that see nothing, one past the cache."""
    last = torch.randint(max(L - max(L // 3, 1), 0), max(L, 1), (B, 1), generator=g)
    p = last - M + 1 + torch.arange(M)
    p = torch.where(torch.rand((B, M), generator=g) < 0.1, torch.randint(-4, L + 9, (B, M), generator=g), p)
    p[0, 0], p[-1, -1] = -1, L + 5
    return (p + pos0).clamp_min(-1).to(torch.int32)


def _places(g, B, M, n):
    at = {(0, 0), (B - 1, M - 1), (B - 1, 0), (0, M - 1)}
    while len(at) < min(n, B * M):
        at.add((int(torch.randint(0, B, (1,), generator=g)), int(torch.randint(0, M, (1,), generator=g))))
    return sorted(at)


def _behind(x, q_pos, pos0, value):
    x = x.clone()
    for b in range(x.shape[0]):
        x[b, :, max(0, int(q_pos[b].max()) - pos0 + 1):] = value
    return x


def _same_again(call, out, lse, turns=3):
    for _ in range(turns):                     # whichever workgroup joins the parts: the same bits
        o, y = call()
        assert torch.equal(o, out) and torch.equal(y, lse)


@pytest.mark.gpu
@pytest.mark.parametrize("case", WINDOW, ids=str)
def test_window(plan, case):
    Hq, Hkv, d, B, M, L, W, S, parts = case
    assert _window_parts(plan, *case[:8]) == parts
    g = torch.Generator().manual_seed(sum(case[:8]))
    q, K, V, pos0 = _normal(g, B, M, Hq, d), _normal(g, B, Hkv, L, d), _normal(g, B, Hkv, L, d), 11
    q_pos = _positions(g, B, M, L, pos0)
    cfg = msa.MsaConfig(1, 1, 1, Hq, Hkv, d, 1e4)
    args = [t.cuda() for t in (q, _behind(K, q_pos, pos0, float("nan")), _behind(V, q_pos, pos0, float("inf")), q_pos)]
    ws = torch.full((msa.window_attend_workspace_bytes(cfg, B, M, L, W, S),), 0xA5, dtype=torch.uint8, device="cuda")

    def call():
        return msa.msa_window_attend(cfg, *args, W, sinks=S, local_pos0=pos0, workspace=ws)

    out, lse = call()
    _same_again(call, out, lse)
    at, t, r = _places(g, B, M, 24), torch.arange(L), Hq // Hkv
    ref = P.Attended((len(at), Hq), d)
    for i, (b, m) in enumerate(at):
        p = int(q_pos[b, m]) - pos0
        seen = (t <= p) & ((p - t < W) | (t < S))
        rows = [(x[b][:, seen].double()) for x in (K, V)]
        for h in range(Hq):
            ref.put((i, h), P.attend(q[b, m, h].double(), rows[0][h // r], rows[1][h // r], seen[seen]))
    pick = tuple(torch.tensor(at).T)
    ref.check(out.cpu()[pick], lse.cpu()[pick], PAIRS if parts > 0 else SINGLE)


class _Four:
    """A bank in four bits with documents of their own lengths, selections with pads and ids outside, and the call."""

    def __init__(self, case, pool=1, seed=0):
        Hq, Hkv, d, B, M, k, G, L, scope, _ = case
        g = self.g = torch.Generator().manual_seed(sum(case[:8]) + seed)
        N, self.pos0 = 40, G
        self.case, self.pool, self.N = case, pool, N
        K, V = _normal(g, N, Hkv, G, d), _normal(g, N, Hkv, G, d)
        self.lens = torch.randint(0, G + 2, (N,), generator=g, dtype=torch.int32)
        self.cfg = msa.MsaConfig(N, G, 1, Hq, Hkv, d, 1e4, bank_keys_rotated=1, select_scope=scope, token_pool=pool,
                                 doc_lens=self.lens.cuda())
        self.bank = msa.msa_pack_kv4(self.cfg.replace(doc_lens=None), K.cuda(), V.cuda())
        self.kept = [P.unpack4(self.bank[i].cpu(), self.bank[i + 1].cpu()) for i in (0, 2)]
        self.q, self.Kl, self.Vl = _normal(g, B, M, Hq, d), _normal(g, B, Hkv, L, d), _normal(g, B, Hkv, L, d)
        self.q_pos = _positions(g, B, M, L, G)
        self.idx = self.selection()
        self.dev = [t.cuda() for t in (self.q, self.idx, _behind(self.Kl, self.q_pos, G, float("nan")),
                                       _behind(self.Vl, self.q_pos, G, float("inf")), self.q_pos)]
        size = msa.sparse_attend4_workspace_bytes(self.cfg, B, M, k, L)
        self.ws = torch.full((size,), 0xA5, dtype=torch.uint8, device="cuda")

    def selection(self):
        Hq, Hkv, d, B, M, k, G, L, scope, _ = self.case
        idx = torch.randint(-1, self.N, (B, 1 if self.pool else M, 1 if scope else Hkv, k), generator=self.g, dtype=torch.int32)
        idx[0, 0, 0, k // 2] = self.N
        idx[-1, 0, -1] = -1                    # no document at all
        return idx

    def call(self, **kw):
        q, idx, Kl, Vl, q_pos = self.dev
        near = (Kl, Vl) if Kl.shape[2] else (None, None)
        return msa.msa_sparse_attend4(self.cfg, q, self.bank, idx, *near, self.pos0, q_pos, **kw)

    def check(self, out, lse, weights, n=24, without=None):
        Hq, Hkv, d, B, M, k, G, L, scope, _ = self.case
        at, r = [x for x in _places(self.g, B, M, n) if without is None or not without[x]], Hq // Hkv
        ref = P.Attended((len(at), Hq), d)
        for i, (b, m) in enumerate(at):
            near = torch.arange(L) + self.pos0 <= int(self.q_pos[b, m])
            for h0 in range(Hkv):
                docs = [int(x) for x in self.idx[b, 0 if self.pool else m, 0 if scope else h0] if 0 <= int(x) < self.N]
                n_of = [min(max(int(self.lens[x]), 1), G) for x in docs]
                rows = [torch.cat([x[j, h0, :c] for j, c in zip(docs, n_of)] + [y[b, h0][near].double()])
                        for x, y in zip(self.kept, (self.Kl, self.Vl))]
                seen = torch.ones(rows[0].shape[0], dtype=torch.bool)
                for h in range(h0 * r, h0 * r + r):
                    ref.put((i, h), P.attend(self.q[b, m, h].double(), *rows, seen))
        pick = tuple(torch.tensor(at).T)
        ref.check(out.cpu()[pick], lse.cpu()[pick], weights)


@pytest.mark.gpu
@pytest.mark.parametrize("case", ATTEND4, ids=str)
def test_attend4(plan, case):
    parts = case[9]
    assert _attend4_parts(plan, *case[:8]) == parts
    f = _Four(case)
    out, lse = f.call(workspace=f.ws)
    _same_again(lambda: f.call(workspace=f.ws), out, lse)
    f.check(out, lse, PAIRS if parts > 0 else SINGLE)


@pytest.mark.gpu
@pytest.mark.parametrize("M", [9, 40])
def test_selections_of_their_own_keep_pairs(plan, M):
    """Tokens whose selections are their own go one by one, however many they are."""
    case = (8, 2, 128, 2, M, 5, 33, 60, 0, None)
    assert _attend4_parts(plan, *case[:8], pool=0) > 0
    f = _Four(case, pool=0)
    f.check(*f.call(workspace=f.ws), PAIRS)


@pytest.mark.gpu
@pytest.mark.parametrize("case", [c for c in ATTEND4 if c[4] in (8, 9, 300, 700)], ids=str)
def test_queries_that_are_no_numbers_stay_by_themselves(case):
    """The padding of a batch holds anything; where its tokens see shared documents their own outputs do too, and no others."""
    f = _Four(case)
    B, M = case[3], case[4]
    bad = torch.rand((B, M), generator=f.g) < 0.4
    bad[0, 0], bad[-1, -1] = True, True
    bad[0, 1] = bad[-1, 0] = bad[0, M - 1] = False
    f.dev[0][bad.cuda()] = float("nan")
    out, lse = f.call(workspace=f.ws)
    assert bool(out.cpu()[~bad].isfinite().all()) and not bool(lse.cpu()[~bad].isnan().any())
    f.check(out, lse, PAIRS if case[9] > 0 else SINGLE, without=bad)


@pytest.mark.gpu
@pytest.mark.parametrize("case", [c for c in ATTEND4 if c[9] < 0 and c[4] in (8, 9, 20, 300, 100)], ids=str)
def test_graphs_of_expanded_documents(case):
    """A captured call that expands its documents, replayed on other selections and queries, with eager work in between."""
    f = _Four(case)
    B, M, Hq = case[3], case[4], case[0]
    out, lse = torch.empty_like(f.dev[0]), torch.empty((B, M, Hq), dtype=torch.float32, device="cuda")
    f.call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f.call(out=out, lse=lse, workspace=f.ws)
    for turn in range(4):
        f.idx = f.selection()
        f.q = _normal(f.g, *f.q.shape)
        f.dev[0].copy_(f.q)
        f.dev[1].copy_(f.idx)
        for t in (out, lse):
            t.fill_(3.0)
        graph.replay()
        o, y = f.call()
        torch.cuda.synchronize()
        assert torch.equal(o, out) and torch.equal(y, lse), turn
    f.check(out, lse, SINGLE, n=6)


@pytest.mark.gpu
def test_single_token_offsets_past_32_bits():
    """The single-token kernel at the far end of a cache of 2.2 billion elements, and of a bank whose codes alone are 2.3 GB, by
    the bound of its weights."""
    g = torch.Generator().manual_seed(3)
    B, Hq, Hkv, L, d = 2, 8, 4, 2_150_000, 128
    K, V = (torch.zeros((B, Hkv, L, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q, Ks, Vs = _normal(g, B, 1, Hq, d), _normal(g, B, Hkv, 300, d), _normal(g, B, Hkv, 300, d)
    K[:, :, L - 300:], V[:, :, L - 300:] = Ks.cuda(), Vs.cuda()
    q_pos = torch.full((B, 1), L - 1, dtype=torch.int32)
    out, lse = msa.msa_window_attend(msa.MsaConfig(1, 1, 1, Hq, Hkv, d, 1e4), q.cuda(), K, V, q_pos.cuda(), 200)
    P.window_attend(q.double(), Ks.double(), Vs.double(), q_pos - (L - 300), 200, 0, 0).check(out, lse, PAIRS)
    del K, V
    torch.cuda.empty_cache()
    N, G, k = 9000, 512, 3
    cfg = msa.MsaConfig(N, G, 1, Hq, 8, d, 1e4, bank_keys_rotated=1)
    bank = tuple(torch.zeros_like(t) for t in msa.alloc_kv4(cfg))
    bank[1].fill_(127), bank[3].fill_(127)
    small = msa.msa_pack_kv4(cfg.replace(n_docs=4), _normal(g, 4, 8, G, d).cuda(), _normal(g, 4, 8, G, d).cuda())
    for t, x in zip(bank, small):
        t[N - 4:] = x
    idx = torch.tensor([N - 1, N - 3, N - 4], dtype=torch.int32).reshape(1, 1, 1, k).expand(1, 1, 8, k).contiguous()
    q1, Kl, Vl = _normal(g, 1, 1, Hq, d), _normal(g, 1, 8, 9, d), _normal(g, 1, 8, 9, d)
    q_pos = torch.full((1, 1), G + 8, dtype=torch.int32)
    out, lse = msa.msa_sparse_attend4(cfg, q1.cuda(), bank, idx.cuda(), Kl.cuda(), Vl.cuda(), G, q_pos.cuda())
    kept = [P.unpack4(small[i].cpu(), small[i + 1].cpu()) for i in (0, 2)]
    P.sparse_attend4(q1.double(), *kept, idx - (N - 4), None, Kl.double(), Vl.double(), q_pos, G).check(out, lse, PAIRS)


@pytest.mark.gpu
@pytest.mark.parametrize("d, M", [(64, 1), (128, 2), (64, 5)])
def test_a_captured_decode_step(d, M):
    """One step of a program -- norms and append, a local layer, a routed layer, and the new document packed and unpacked -- captured
    once and replayed for token after token, positions and projections changing between: the bits of the same steps run eagerly."""
    B, Hq, Hkv, N, G, L, k = 3, 8, 2, 12, 24, 64, 4
    g = torch.Generator().manual_seed(d + M)
    cfg = msa.MsaConfig(N, G, 1, Hq, Hkv, d, 1e4, bank_keys_rotated=1, token_pool=int(M > 1))
    K, V = (_normal(g, N, Hkv, G, d).cuda() for _ in range(2))
    bank = msa.msa_pack_kv4(cfg, K, V)
    idx = torch.randint(-1, N, (B, 1, Hkv, k), generator=g, dtype=torch.int32).cuda()
    w = [(1 + 0.2 * torch.randn(d, generator=g)).to(torch.bfloat16).cuda() for _ in range(2)]
    fused = torch.empty((B, M, Hq + 2 * Hkv, d), dtype=torch.bfloat16, device="cuda")
    pos = torch.empty((B, M), dtype=torch.int32, device="cuda")

    class Step:
        def __init__(self):
            self.Kl, self.Vl = (torch.full((B, Hkv, L, d), 0.5, dtype=torch.bfloat16, device="cuda") for _ in range(2))
            self.q, self.a, self.b = (torch.empty((B, M, Hq, d), dtype=torch.bfloat16, device="cuda") for _ in range(3))
            self.la, self.lb = (torch.empty((B, M, Hq), dtype=torch.float32, device="cuda") for _ in range(2))
            self.bank, self.back = tuple(t.clone() for t in bank), [torch.zeros_like(K) for _ in range(2)]
            self.wa = torch.full((msa.window_attend_workspace_bytes(cfg, B, M, L, 20, 3),), 0xA5, dtype=torch.uint8, device="cuda")
            self.wb = torch.full((msa.sparse_attend4_workspace_bytes(cfg, B, M, k, L),), 0xA5, dtype=torch.uint8, device="cuda")

        def run(self):
            msa.msa_norm_rotate(cfg, fused[:, :, :Hq], fused[:, :, Hq:Hq + Hkv], fused[:, :, Hq + Hkv:], pos, self.Kl, self.Vl, *w,
                                local_pos0=G, q_out=self.q)
            msa.msa_pack_kv4(cfg, K, V, N - 2, 2, self.bank)
            msa.msa_window_attend(cfg, self.q, self.Kl, self.Vl, pos, 20, sinks=3, local_pos0=G, out=self.a, lse=self.la, workspace=self.wa)
            msa.msa_sparse_attend4(cfg, self.q, self.bank, idx, self.Kl, self.Vl, G, pos, out=self.b, lse=self.lb, workspace=self.wb)
            msa.msa_unpack_kv4(cfg, self.bank, N - 2, 2, *self.back)

        def results(self):
            return [self.Kl, self.Vl, self.q, self.a, self.la, self.b, self.lb, *self.bank, *self.back]

    def feed(step):
        fused.copy_(_normal(g, *fused.shape))
        pos.copy_((G + step * M + torch.arange(M)).expand(B, M) - torch.arange(B)[:, None] * (step > 1))
        K[N - 2:].copy_(_normal(g, 2, Hkv, G, d))

    feed(0)
    Step().run()                               # (warm)
    torch.cuda.synchronize()
    played, eager, graph = Step(), Step(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        played.run()
    for step in range(6):
        feed(step)
        graph.replay()
        eager.run()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(played.results(), eager.results())), step
