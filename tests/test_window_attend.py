"""msa_window_attend against the plain definition in 64 bits: windows, first tokens, positions in any order, empty rows."""
import ctypes
import itertools
import threading

import pytest
import torch

import paper_2603_23516_amd as msa
import plain64 as P

FEW = 2.0 ** -16      # softmax weights of few tokens: bf16 (hi, lo) pairs
MANY = 2.0 ** -8      # of many: bf16


def _cfg(Hq=8, Hkv=2, d=64):
    return msa.MsaConfig(1, 1, 1, Hq, Hkv, d, 1e4)


@pytest.fixture(scope="module")
def lib():
    return msa.load_library()


def _call(lib, cfg, **kw):
    p = ctypes.c_void_p(0x10000)
    a = dict(q=p, B=1, M=1, K=p, V=p, L=64, pos0=0, W=16, S=0, q_pos=p, out=p, lse=p, ws=p, bytes=1 << 40)
    a.update(kw)
    return lib.msa_window_attend(ctypes.byref(cfg), a["q"], a["B"], a["M"], a["K"], a["V"], a["L"], a["pos0"], a["W"], a["S"],
                                 a["q_pos"], a["out"], a["lse"], a["ws"], a["bytes"], None)


@pytest.mark.parametrize("kw, status", [
    (dict(q=None), -1), (dict(K=None), -1), (dict(V=None), -1), (dict(q_pos=None), -1), (dict(out=None), -1), (dict(ws=None), -1),
    (dict(B=0), -1), (dict(M=0), -1), (dict(L=0), -1), (dict(W=0), -1), (dict(S=-1), -1), (dict(pos0=-1), -1),
    (dict(B=65536), -2), (dict(B=1 << 13, M=1 << 13), -2),
    (dict(B=65536, M=32), -2), (dict(L=(1 << 28) + 1), -2), (dict(bytes=255), -3),
    (dict(q=ctypes.c_void_p(0x10008)), -4), (dict(K=ctypes.c_void_p(0x10002)), -4), (dict(q_pos=ctypes.c_void_p(0x10002)), -4),
    (dict(lse=ctypes.c_void_p(0x10002)), -4), (dict(ws=ctypes.c_void_p(0x10010 + 4)), -4),
])
def test_refusals(lib, kw, status):
    assert _call(lib, _cfg(), **kw) == status


def test_workspace_sizes(lib):
    c = _cfg(32, 8, 128)
    for B, M, L, W, S in ((1, 1, 1, 1, 0), (1, 1, 1 << 20, 1 << 20, 4), (40, 1, 8192, 4096, 4), (1, 8192, 8192, 4096, 4), (1, 8, 65536, 65536, 0)):
        n = msa.window_attend_workspace_bytes(c, B, M, L, W, S)
        assert n >= 256 and n % 256 == 0
        assert _call(lib, c, B=B, M=M, L=L, W=W, S=S, bytes=n - 1) == msa.MSA_ERR_WORKSPACE
    assert msa.window_attend_workspace_bytes(c, 1, 1, 0, 4, 0) == 0
    assert msa.window_attend_workspace_bytes(c, 1, 1, 8, 0, 0) == 0
    assert msa.window_attend_workspace_bytes(c, 1, 70000, 8, 2 ** 40, 2 ** 40) == msa.window_attend_workspace_bytes(c, 1, 70000, 8, 8, 0)
    for bad in (dict(M=2 ** 32 + 1), dict(Lloc=2 ** 31), dict(window=-2 ** 40), dict(sinks=-2 ** 33)):
        with pytest.raises(ValueError):
            msa.window_attend_workspace_bytes(c, **{**dict(B=1, M=1, Lloc=8, window=4, sinks=0), **bad})
    # a longer cache or window never asks for less
    for cfg, B, M in itertools.product((c, _cfg(8, 1, 64)), (1, 3, 40), (1, 2, 5, 9, 31, 32, 509)):
        sizes = [msa.window_attend_workspace_bytes(cfg, B, M, L, W, S) for L, W, S in (
                (1, 1, 0), (100, 50, 0), (100, 50, 40), (1000, 50, 40), (1000, 500, 40), (2500, 2000, 40), (9000, 8000, 40), (70000, 66000, 40))]
        assert sizes == sorted(sizes), (B, M)


def _make(B, M, Hq, Hkv, d, L, seed=0):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(s, generator=g).to(torch.bfloat16) for s in ((B, M, Hq, d), (B, Hkv, L, d), (B, Hkv, L, d))]


def _check(Hq, Hkv, d, q, K, V, q_pos, W, S, pos0, **kw):
    B, M = q.shape[:2]
    cfg = _cfg(Hq, Hkv, d)
    ws = torch.full((msa.window_attend_workspace_bytes(cfg, B, M, K.shape[2], W, S),), 0xA5, dtype=torch.uint8, device="cuda")
    Kd, Vd = K.clone(), V.clone()
    for b in range(B):          # what lies behind every token of a sequence has no effect
        behind = max(0, int(q_pos[b].max()) - pos0 + 1)
        Kd[b, :, behind:] = float("nan")
        Vd[b, :, behind:] = float("inf")
    out, lse = msa.msa_window_attend(cfg, q.cuda(), Kd.cuda(), Vd.cuda(), q_pos.cuda(), W, sinks=S, local_pos0=pos0,
                                     workspace=ws, **kw)
    torch.cuda.synchronize()
    P.window_attend(q.double(), K.double(), V.double(), q_pos, W, S, pos0).check(out, lse, FEW if M < 8 else MANY)
    return out, lse


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 3, 8, 45])
@pytest.mark.parametrize("Hq, Hkv, d", [(4, 4, 64), (4, 2, 128), (6, 2, 64), (4, 1, 64), (8, 1, 128), (5, 1, 128)])
@pytest.mark.parametrize("L, W, S", [(1, 1, 0), (50, 1, 0), (50, 7, 3), (97, 32, 33), (130, 200, 4), (161, 33, 0)])
def test_against_64_bits(M, Hq, Hkv, d, L, W, S):
    q, K, V = _make(2, M, Hq, Hkv, d, L, M + L)
    pos0 = 5
    last = torch.tensor([[L - 1], [max(L // 2, 0)]]) + pos0
    q_pos = (last - M + 1 + torch.arange(M)).to(torch.int32)      # the first tokens may lie in front of the cache: they see nothing
    _check(Hq, Hkv, d, q, K, V, q_pos, W, S, pos0)


@pytest.mark.gpu
@pytest.mark.parametrize("M", [2, 40])
def test_positions_in_any_order(M):
    """Padding, positions past the cache's end, the same position twice, tokens far apart in one tile."""
    g = torch.Generator().manual_seed(2)
    q, K, V = _make(3, M, 4, 2, 64, 300, 1)
    q_pos = torch.randint(-3, 340, (3, M), generator=g, dtype=torch.int32)
    q_pos[0, 0], q_pos[1, 1], q_pos[2] = -2 ** 31, 2 ** 31 - 1, -1
    for W, S in ((16, 4), (400, 0), (1, 0), (2 ** 31 - 1, 2 ** 31 - 1), (60, 100)):
        _check(4, 2, 64, q, K, V, q_pos, W, S, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("M, L, W, S", [(1, 3000, 2500, 9), (4, 2100, 2100, 0), (9, 2500, 2500, 0), (20, 1700, 900, 70)])
def test_split_rows(M, L, W, S):
    """Long windows with few tokens: the rows are shared out and the parts joined."""
    q, K, V = _make(1, M, 4, 1, 128, L, 4)
    q_pos = (L - M + torch.arange(M)).reshape(1, M).to(torch.int32)
    _check(4, 1, 128, q, K, V, q_pos, W, S, 0)
    q_pos[0, 0] = 31                                              # one of them sees a single step: most parts of it are empty
    _check(4, 1, 128, q, K, V, q_pos, W, S, 0)


@pytest.mark.gpu
def test_large_scores():
    """Scores of hundreds: one row takes all; and equal scores: the mean."""
    q, K, V = _make(1, 12, 4, 2, 64, 200, 5)
    q_pos = (188 + torch.arange(12)).reshape(1, 12).to(torch.int32)
    for M in (12, 2):
        _check(4, 2, 64, (q[:, :M] * 30).to(torch.bfloat16), (K * 10).to(torch.bfloat16), V, q_pos[:, :M].contiguous(), 100, 3, 0)
        _check(4, 2, 64, torch.zeros_like(q[:, :M]), K, V, q_pos[:, :M].contiguous(), 100, 3, 0)


@pytest.mark.gpu
def test_tokens_do_not_depend_on_their_neighbours():
    """A prompt in one call and in chunks, and a second sequence beside it: the same results within the weights' rounding."""
    q, K, V = _make(2, 300, 8, 2, 128, 300, 6)
    cfg = _cfg(8, 2, 128)
    q, K, V = q.cuda(), K.cuda(), V.cuda()
    q_pos = torch.arange(300, dtype=torch.int32, device="cuda").expand(2, 300).contiguous()
    out, lse = msa.msa_window_attend(cfg, q, K, V, q_pos, 64, sinks=4)
    for m0, m1 in ((0, 100), (100, 300), (299, 300)):
        o, y = msa.msa_window_attend(cfg, q[:1, m0:m1].contiguous(), K[:1].contiguous(), V[:1].contiguous(), q_pos[:1, m0:m1].contiguous(), 64, sinks=4)
        assert float((o.float() - out[:1, m0:m1].float()).abs().max()) <= 2.0 ** -5      # |V| < 5: 2^-8 of it twice, bf16 steps
        assert float((y - lse[:1, m0:m1]).abs().max()) <= 1e-4


@pytest.mark.gpu
@pytest.mark.parametrize("M, L, Hq, Hkv", [(1, 2000, 8, 1), (12, 700, 8, 1), (40, 3000, 8, 1), (256, 2100, 64, 8)])
def test_graph_replays_and_streams(M, L, Hq, Hkv):
    """A captured call, replayed on new inputs with other work between, on a stream of its own, with split rows: one token,
    tokens one by one, tiles whose many parts a launch joins, tiles whose few parts the last workgroup joins."""
    cfg = _cfg(Hq, Hkv, 128)
    q, K, V = (t.cuda() for t in _make(1, M, Hq, Hkv, 128, L, 7))
    q_pos = (L - M + torch.arange(M)).reshape(1, M).to(torch.int32).cuda()
    ws = torch.full((msa.window_attend_workspace_bytes(cfg, 1, M, L, L, 0),), 0xFF, dtype=torch.uint8, device="cuda")
    out, lse = torch.empty_like(q), torch.empty((1, M, Hq), dtype=torch.float32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        msa.msa_window_attend(cfg, q, K, V, q_pos, L, out=out, lse=lse, workspace=ws)
    for i in range(4):
        q.copy_(torch.randn_like(q.float()).to(torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        o, y = msa.msa_window_attend(cfg, q, K, V, q_pos, L)
        torch.cuda.synchronize()
        assert torch.equal(o, out) and torch.equal(y, lse), i
    with torch.cuda.stream(side):
        o2, y2 = msa.msa_window_attend(cfg, q, K, V, q_pos, L, workspace=ws)
    side.synchronize()
    assert torch.equal(o2, out) and torch.equal(y2, lse)


@pytest.mark.gpu
def test_python_refusals():
    cfg = _cfg()
    q, K, V = (t.cuda() for t in _make(2, 3, 8, 2, 64, 9))
    pos = torch.zeros((2, 3), dtype=torch.int32, device="cuda")
    for bad in (dict(q=q[:1]), dict(q=q.transpose(1, 2)), dict(Kloc=K[:, :, :5]), dict(Vloc=V.float()), dict(q_pos=pos[:, :2]),
                dict(q_pos=pos.long()), dict(out=q[:1])):
        a = dict(q=q, Kloc=K, Vloc=V, q_pos=pos, window=4)
        a.update(bad)
        with pytest.raises(ValueError):
            msa.msa_window_attend(cfg, **a)
    with pytest.raises(msa.MsaError):
        msa.msa_window_attend(cfg, q, K, V, pos, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("M", [3, 40])
def test_queries_of_padding_may_be_anything(M):
    """Tokens that see nothing give zeros and -inf whatever their queries hold, and do not touch their neighbours."""
    q, K, V = _make(2, M, 4, 2, 64, 60, 9)
    q_pos = (60 - M + torch.arange(M)).expand(2, M).contiguous().to(torch.int32)
    q_pos[:, ::2] = -1
    cfg = _cfg(4, 2, 64)
    bad = q.clone()
    bad[:, ::2] = float("nan")
    a = msa.msa_window_attend(cfg, q.cuda(), K.cuda(), V.cuda(), q_pos.cuda(), 30, sinks=2)
    b = msa.msa_window_attend(cfg, bad.cuda(), K.cuda(), V.cuda(), q_pos.cuda(), 30, sinks=2)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert float(b[0][:, ::2].abs().max()) == 0.0 and bool(torch.isinf(b[1][:, ::2]).all())


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 33])
def test_offsets_past_32_bits(M):
    """A cache of 2.2 billion elements: the last rows of the last head are found."""
    B, Hkv, L, d = 2, 4, 2_150_000, 128
    cfg = _cfg(8, Hkv, d)
    K, V = (torch.zeros((B, Hkv, L, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q, Ks, Vs = _make(B, M, 8, Hkv, d, 300, 10)
    K[:, :, L - 300:], V[:, :, L - 300:] = Ks.cuda(), Vs.cuda()
    q_pos = (L - M + torch.arange(M)).expand(B, M).contiguous().to(torch.int32)
    out, lse = msa.msa_window_attend(cfg, q.cuda(), K, V, q_pos.cuda(), 200)
    torch.cuda.synchronize()
    P.window_attend(q.double(), Ks.double(), Vs.double(), q_pos - (L - 300), 200, 0, 0).check(out, lse, MANY)
    del K, V
    torch.cuda.empty_cache()


@pytest.mark.gpu
def test_two_streams_at_once():
    """Calls that run side by side with workspaces of their own, and one whose workspace comes from the binding."""
    cfg = _cfg(8, 1, 128)
    sets = [[t.cuda() for t in _make(1, 1, 8, 1, 128, 4000, 20 + i)] for i in range(3)]
    pos = torch.full((1, 1), 3999, dtype=torch.int32, device="cuda")
    want = [msa.msa_window_attend(cfg, *s, pos, 4000) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(20):
        got = [msa.msa_window_attend(cfg, *s, pos, 4000, stream=st) for s, st in zip(sets, streams)]
        for st in streams:
            st.synchronize()
        assert all(torch.equal(a, c) and torch.equal(b, d) for (a, b), (c, d) in zip(want, got))


@pytest.mark.gpu
def test_one_by_one_and_together_agree():
    """The same tokens below and above the number that goes through the tiled kernel."""
    q, K, V = _make(1, 32, 8, 2, 64, 500, 30)
    q_pos = (468 + torch.arange(32)).reshape(1, 32).to(torch.int32)
    a, la = _check(8, 2, 64, q, K, V, q_pos, 77, 5, 0)
    b, lb = _check(8, 2, 64, q[:, :31].contiguous(), K, V, q_pos[:, :31].contiguous(), 77, 5, 0)
    assert float((a[:, :31].float() - b.float()).abs().max()) <= 2.0 ** -5 and float((la[:, :31] - lb).abs().max()) <= 1e-4


@pytest.mark.gpu
@pytest.mark.parametrize("B, M, Hq, Hkv, d, L, W, S", [
    (1, 256, 64, 8, 128, 2100, 2100, 0),       # two parts to a tile
    (4, 509, 16, 8, 64, 1500, 1000, 16),       # two, of 64 dims
    (1, 40, 8, 1, 128, 3000, 2500, 3),         # many, joined by a launch
    (1, 700, 24, 8, 64, 900, 900, 0),          # none: r = 3
])
def test_many_tokens_at_random_places(B, M, Hq, Hkv, d, L, W, S):
    """Chunks of prompts large enough for every way of sharing their rows out; tokens at random places in 64 bits."""
    q, K, V = _make(B, M, Hq, Hkv, d, L, M)
    last = torch.tensor([[L - 1 - 97 * b] for b in range(B)])
    q_pos = (last - M + 1 + torch.arange(M)).to(torch.int32)
    args = (_cfg(Hq, Hkv, d), q.cuda(), K.cuda(), V.cuda(), q_pos.cuda(), W)
    out, lse = msa.msa_window_attend(*args, sinks=S)
    for _ in range(3):        # whichever workgroup is the last to join the parts: the same bits
        again = msa.msa_window_attend(*args, sinks=S)
        assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    g = torch.Generator().manual_seed(1)
    n = 60
    at = torch.stack([torch.randint(0, B, (n,), generator=g), torch.randint(0, M, (n,), generator=g)], 1).tolist() + [[0, 0], [B - 1, M - 1]]
    ref = P.Attended((len(at), Hq), d)
    t = torch.arange(L)
    for i, (b, m) in enumerate(at):
        p = int(q_pos[b, m])
        seen = (t <= p) & ((p - t < W) | (t < S))
        for h in range(Hq):
            ref.put((i, h), P.attend(q[b, m, h].double(), K[b, h * Hkv // Hq].double(), V[b, h * Hkv // Hq].double(), seen))
    pick = tuple(torch.tensor(at).T)
    ref.check(out.cpu()[pick], lse.cpu()[pick], MANY)


def _some_tokens(out, lse, q, K, V, q_pos, W, S, at):
    ref = P.Attended((len(at), q.shape[2]), q.shape[3])
    t = torch.arange(K.shape[2])
    for i, m in enumerate(at):
        p = int(q_pos[0, m])
        seen = (t <= p) & ((p - t < W) | (t < S))
        for h in range(q.shape[2]):
            ref.put((i, h), P.attend(q[0, m, h].double(), K[0, 0, seen].double(), V[0, 0, seen].double(), seen[seen]))
    ref.check(out[0, at].cpu(), lse[0, at].cpu(), MANY)


@pytest.mark.gpu
def test_a_prompt_of_more_than_65535_tokens():
    M, W, S = 70001, 300, 5
    q, K, V = _make(1, M, 2, 1, 64, M, 40)
    q_pos = torch.arange(M, dtype=torch.int32).reshape(1, M)
    out, lse = msa.msa_window_attend(_cfg(2, 1, 64), q.cuda(), K.cuda(), V.cuda(), q_pos.cuda(), W, sinks=S)
    _some_tokens(out, lse, q, K, V, q_pos, W, S, [0, 1, 299, 300, 306, 40000, 65534, 65535, 65536, 65600, M - 65, M - 1])


@pytest.mark.gpu
@pytest.mark.parametrize("M", [2, 40])
def test_sizes_past_32_bits(M):
    """A window, or a number of first tokens, past 32 bits sees everything; what would be cut off is refused."""
    cfg = _cfg(2, 1, 64)
    q, K, V = (t.cuda() for t in _make(1, M, 2, 1, 64, 90, 41))
    pos = (90 - M + torch.arange(M)).reshape(1, M).to(torch.int32).cuda()
    want = msa.msa_window_attend(cfg, q, K, V, pos, 90)
    for W, S in ((2 ** 31, 0), (2 ** 32 + 5, 0), (3, 2 ** 32), (2 ** 31 - 1, 0)):
        got = msa.msa_window_attend(cfg, q, K, V, pos, W, sinks=S)
        assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
    for bad in (dict(local_pos0=2 ** 32), dict(window=-2 ** 32 + 9), dict(sinks=-2 ** 32)):
        with pytest.raises(ValueError):
            msa.msa_window_attend(cfg, q, K, V, pos, **{**dict(window=9), **bad})


@pytest.mark.gpu
def test_two_graphs_share_a_workspace():
    """Graphs of different layouts of one workspace, replayed in turn, with eager calls through it in between."""
    cfg = _cfg(32, 8, 128)
    sets = []
    for M, L in ((1, 3000), (256, 2100), (48, 3000), (2, 1500)):      # parts of single tokens, of tiles (two, more), again
        q, K, V = (t.cuda() for t in _make(1, M, 32, 8, 128, L, 50 + M))
        sets.append((q, K, V, (L - M + torch.arange(M)).reshape(1, M).to(torch.int32).cuda(), L))
    want = [msa.msa_window_attend(cfg, *s) for s in sets]
    size = max(msa.window_attend_workspace_bytes(cfg, 1, s[0].shape[1], s[4], s[4]) for s in sets)
    ws = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")
    outs = [(torch.empty_like(a), torch.empty_like(b)) for a, b in want]
    torch.cuda.synchronize()
    side, graphs = torch.cuda.Stream(), []
    for s, (o, l) in zip(sets, outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            msa.msa_window_attend(cfg, *s, out=o, lse=l, workspace=ws, stream=side)
    for turn in range(4):
        for i in (0, 1, 2, 3, 1, 0):
            for t in outs[i]:
                t.fill_(3.0)
            graphs[i].replay()
            again = msa.msa_window_attend(cfg, *sets[(i + turn) % 4], workspace=ws)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(outs[i], want[i])), (turn, i)
            assert all(torch.equal(a, b) for a, b in zip(again, want[(i + turn) % 4])), (turn, i)


@pytest.mark.gpu
def test_calls_from_two_threads():
    cfg = _cfg(8, 2, 64)
    sets = []
    for i, M in enumerate((1, 100)):
        q, K, V = (t.cuda() for t in _make(1, M, 8, 2, 64, 1000, 60 + i))
        sets.append((q, K, V, (1000 - M + torch.arange(M)).reshape(1, M).to(torch.int32).cuda(), 1000))
    want = [msa.msa_window_attend(cfg, *s) for s in sets]
    torch.cuda.synchronize()
    bad = []

    def work(i):
        stream = torch.cuda.Stream()
        for _ in range(50):
            got = msa.msa_window_attend(cfg, *sets[i], stream=stream)
            stream.synchronize()
            if not all(torch.equal(a, b) for a, b in zip(got, want[i])):
                bad.append(i)

    threads = [threading.Thread(target=work, args=(i,)) for i in (0, 1, 0, 1)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad
