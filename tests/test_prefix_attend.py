"""msa_prefix_attend against the plain definition in 64 bits: shared prefixes of any length, parts of them, empty rows."""
import ctypes
import itertools

import pytest
import torch

import paper_2603_23516_amd as msa
import plain64_cache as C


def _cfg(Hq=8, Hkv=2, d=64):
    return msa.MsaConfig(1, 1, 1, Hq, Hkv, d, 1e4)


@pytest.fixture(scope="module")
def lib():
    return msa.load_library()


def _call(lib, cfg, **kw):
    p = ctypes.c_void_p(0x10000)
    a = dict(q=p, B=1, M=1, Kp=p, Vp=p, P=64, lens=p, K=p, V=p, L=64, pos0=0, q_pos=p, out=p, lse=p, ws=p, bytes=1 << 40)
    a.update(kw)
    return lib.msa_prefix_attend(ctypes.byref(cfg), a["q"], a["B"], a["M"], a["Kp"], a["Vp"], a["P"], a["lens"], a["K"], a["V"],
                                 a["L"], a["pos0"], a["q_pos"], a["out"], a["lse"], a["ws"], a["bytes"], None)


@pytest.mark.parametrize("kw, status", [
    (dict(q=None), -1), (dict(Kp=None), -1), (dict(Vp=None), -1), (dict(K=None), -1), (dict(V=None), -1), (dict(q_pos=None), -1),
    (dict(out=None), -1), (dict(ws=None), -1), (dict(B=0), -1), (dict(M=0), -1), (dict(P=-1), -1), (dict(L=-1), -1),
    (dict(P=0, L=0), -1), (dict(pos0=-1), -1),
    (dict(B=65536), -2), (dict(B=1 << 13, M=1 << 13), -2), (dict(P=(1 << 28) + 1), -2), (dict(L=(1 << 28) + 1), -2),
    (dict(bytes=255), -3),
    (dict(q=ctypes.c_void_p(0x10008)), -4), (dict(Kp=ctypes.c_void_p(0x10002)), -4), (dict(V=ctypes.c_void_p(0x10004)), -4),
    (dict(lens=ctypes.c_void_p(0x10002)), -4), (dict(q_pos=ctypes.c_void_p(0x10001)), -4), (dict(lse=ctypes.c_void_p(0x10002)), -4),
    (dict(ws=ctypes.c_void_p(0x10010 + 4)), -4),
])
def test_refusals(lib, kw, status):
    assert _call(lib, _cfg(), **kw) == status


def test_workspace_sizes(lib):
    for cfg, B, M in itertools.product((_cfg(32, 8, 128), _cfg(8, 1, 64), _cfg(24, 8, 64)), (1, 3, 40, 500), (1, 2, 5, 16, 33, 128, 700)):
        sizes = [msa.prefix_attend_workspace_bytes(cfg, B, M, P, L) for P, L in
                 ((0, 1), (1, 1), (50, 1), (50, 100), (700, 100), (700, 3000), (9000, 3000), (70000, 3000), (70000, 30000))]
        assert sizes == sorted(sizes) and sizes[0] >= 256 and all(n % 256 == 0 for n in sizes), (B, M, sizes)
        assert _call(lib, cfg, B=B, M=M, P=9000, L=3000, bytes=sizes[6] - 1) == msa.MSA_ERR_WORKSPACE
    for bad in (dict(B=2 ** 32 + 1), dict(Lpre=2 ** 31), dict(Lloc=-2 ** 40)):
        with pytest.raises(ValueError):
            msa.prefix_attend_workspace_bytes(cfg, **{**dict(B=1, M=1, Lpre=8, Lloc=8), **bad})


def _make(B, M, Hq, Hkv, d, n_pre, L, seed=0):
    g = torch.Generator().manual_seed(seed)
    shapes = ((B, M, Hq, d), (Hkv, n_pre, d), (Hkv, n_pre, d), (B, Hkv, L, d), (B, Hkv, L, d))
    return [torch.randn(s, generator=g).to(torch.bfloat16) for s in shapes]


def _check(Hq, Hkv, d, q, Kp, Vp, K, V, q_pos, pos0, lens=None, **kw):
    B, M = q.shape[:2]
    n_pre, L = Kp.shape[1], K.shape[2]
    cfg = _cfg(Hq, Hkv, d)
    ws = torch.full((msa.prefix_attend_workspace_bytes(cfg, B, M, n_pre, L),), 0xA5, dtype=torch.uint8, device="cuda")
    bad = [t.clone() for t in (Kp, Vp, K, V)]
    if lens is not None:        # rows of the prefix that nobody sees, and what lies behind every token of a sequence
        most = max(0, int(lens.max()))
        bad[0][:, most:], bad[1][:, most:] = float("nan"), float("inf")
    for b in range(B):
        behind = max(0, int(q_pos[b].max()) - pos0 + 1)
        bad[2][b, :, behind:], bad[3][b, :, behind:] = float("nan"), float("inf")
    bad = [t.cuda() if t.numel() else None for t in bad]
    out, lse = msa.msa_prefix_attend(cfg, q.cuda(), *bad, q_pos.cuda(), local_pos0=pos0,
                                     prefix_lens=None if lens is None else lens.cuda(), workspace=ws, **kw)
    torch.cuda.synchronize()
    C.prefix_attend(q.double(), Kp.double(), Vp.double(), lens, K.double(), V.double(), q_pos, pos0).check(out, lse, 2.0 ** -8)
    return out, lse


def _ends(B, M, L, pos0):
    """Sequences of different lengths; the first tokens of some lie in front of their cache and see the prefix alone."""
    last = torch.tensor([[L - 1 - (b * 13) % max(L, 1)] for b in range(B)])
    return (pos0 + last - M + 1 + torch.arange(M)).to(torch.int32)


@pytest.mark.gpu
@pytest.mark.parametrize("B, M", [(1, 1), (5, 1), (3, 3), (2, 17), (1, 45), (40, 1)])
@pytest.mark.parametrize("Hq, Hkv, d", [(4, 4, 64), (4, 2, 128), (6, 2, 64), (8, 1, 128), (5, 1, 128)])
@pytest.mark.parametrize("n_pre, L", [(1, 1), (31, 40), (32, 7), (97, 65), (200, 33)])
def test_against_64_bits(B, M, Hq, Hkv, d, n_pre, L):
    x = _make(B, M, Hq, Hkv, d, n_pre, L, M + L)
    _check(Hq, Hkv, d, *x, _ends(B, M, L, n_pre), n_pre)


@pytest.mark.gpu
@pytest.mark.parametrize("B, M", [(6, 1), (4, 9), (3, 50)])
def test_parts_of_the_prefix(B, M):
    """Sequences that share a part of the prefix, none of it, or more than there is; of some tokens nothing is left at all."""
    x = _make(B, M, 4, 2, 64, 130, 70, 5)
    lens = torch.tensor([0, 130, -3, 64, 500, 33][:B], dtype=torch.int32)
    q_pos = _ends(B, M, 70, 130)
    q_pos[:, 0] = -1                    # the prefix alone, or nothing
    if M > 8:
        q_pos[1, 3], q_pos[0, 8] = 2 ** 31 - 1, -2 ** 31
    out, lse = _check(4, 2, 64, *x, q_pos, 130, lens)
    assert bool(torch.isinf(lse[0, 0]).all()) and float(out[0, 0].abs().max()) == 0.0
    lens = torch.zeros(B, dtype=torch.int32)
    _check(4, 2, 64, *x, q_pos, 130, lens)


@pytest.mark.gpu
@pytest.mark.parametrize("B, M", [(3, 1), (3, 20), (1, 40)])
def test_without_prefix_or_cache(B, M):
    q, Kp, Vp, K, V = _make(B, M, 8, 2, 64, 75, 50, 6)
    _check(8, 2, 64, q, Kp[:, :0], Vp[:, :0], K, V, _ends(B, M, 50, 0), 0)
    _check(8, 2, 64, q, Kp, Vp, K[:, :, :0], V[:, :, :0], _ends(B, M, 50, 0), 0)


@pytest.mark.gpu
@pytest.mark.parametrize("B, M, n_pre, L", [(2, 1, 3000, 500), (9, 1, 2100, 1), (33, 1, 1700, 2), (1, 1, 40, 3000), (2, 16, 2500, 700),
                                            (1, 70, 1500, 71)])
def test_long_rows(B, M, n_pre, L):
    """Long prefixes and caches with few tokens: the rows are shared out and the parts joined."""
    x = _make(B, M, 4, 1, 128, n_pre, L, 4)
    _check(4, 1, 128, *x, _ends(B, M, L, n_pre), n_pre)
    lens = torch.tensor([n_pre - 40 * b for b in range(B)], dtype=torch.int32)
    lens[0] = 5                          # one of them sees a single step: most parts of it are empty
    _check(4, 1, 128, *x, _ends(B, M, L, n_pre), n_pre, lens)


@pytest.mark.gpu
def test_large_scores():
    """Scores of hundreds: one row takes all; and equal scores: the mean."""
    for B, M in ((3, 1), (2, 40)):
        q, Kp, Vp, K, V = _make(B, M, 4, 2, 64, 150, 60, 5)
        q_pos = _ends(B, M, 60, 150)
        _check(4, 2, 64, (q * 30).to(torch.bfloat16), (Kp * 10).to(torch.bfloat16), Vp, (K * 10).to(torch.bfloat16), V, q_pos, 150)
        _check(4, 2, 64, torch.zeros_like(q), Kp, Vp, K, V, q_pos, 150)


@pytest.mark.gpu
def test_is_window_attend_over_both():
    """A prefix copied into every cache and attended by msa_window_attend gives the same within the weights' rounding."""
    B, M, Hq, Hkv, d, n_pre, L = 3, 4, 8, 2, 128, 300, 90
    q, Kp, Vp, K, V = (t.cuda() for t in _make(B, M, Hq, Hkv, d, n_pre, L, 8))
    q_pos = _ends(B, M, L, n_pre).cuda()
    cfg = _cfg(Hq, Hkv, d)
    out, lse = msa.msa_prefix_attend(cfg, q, Kp, Vp, K, V, q_pos, local_pos0=n_pre)
    both = [torch.cat([p.expand(B, Hkv, n_pre, d), t], 2).contiguous() for p, t in ((Kp, K), (Vp, V))]
    o, y = msa.msa_window_attend(cfg, q, *both, q_pos, n_pre + L)
    assert float((o.float() - out.float()).abs().max()) <= 2.0 ** -5      # |V| < 5: 2^-8 of it twice, bf16 steps
    assert float((y - lse).abs().max()) <= 1e-4


@pytest.mark.gpu
@pytest.mark.parametrize("B, M", [(3, 1), (2, 40)])
def test_queries_of_padding_may_be_anything(B, M):
    """A token whose query is no number does not touch its neighbours."""
    q, Kp, Vp, K, V = (t.cuda() for t in _make(B, M, 4, 2, 64, 60, 40, 9))
    q_pos = _ends(B, M, 40, 60).cuda()
    bad = q.clone()
    bad[:1, ::2] = float("nan")
    a = msa.msa_prefix_attend(_cfg(4, 2, 64), q, Kp, Vp, K, V, q_pos, local_pos0=60)
    b = msa.msa_prefix_attend(_cfg(4, 2, 64), bad, Kp, Vp, K, V, q_pos, local_pos0=60)
    keep = torch.ones((B, M), dtype=torch.bool)
    keep[:1, ::2] = False
    assert torch.equal(a[0][keep], b[0][keep]) and torch.equal(a[1][keep], b[1][keep])


@pytest.mark.gpu
@pytest.mark.parametrize("B, M, n_pre, L, Hq, Hkv", [(1, 1, 2000, 100, 8, 1), (40, 1, 900, 60, 8, 2), (24, 5, 1500, 77, 4, 2),
                                                     (3, 40, 3000, 90, 8, 1), (4, 128, 700, 300, 8, 2)])
def test_graph_replays_and_streams(B, M, n_pre, L, Hq, Hkv):
    """A captured call, replayed on new inputs with other work between, and on a stream of its own: the same bits."""
    cfg = _cfg(Hq, Hkv, 128)
    q, Kp, Vp, K, V = (t.cuda() for t in _make(B, M, Hq, Hkv, 128, n_pre, L, 7))
    q_pos = _ends(B, M, L, n_pre).cuda()
    ws = torch.full((msa.prefix_attend_workspace_bytes(cfg, B, M, n_pre, L),), 0xFF, dtype=torch.uint8, device="cuda")
    out, lse = torch.empty_like(q), torch.empty((B, M, Hq), dtype=torch.float32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        msa.msa_prefix_attend(cfg, q, Kp, Vp, K, V, q_pos, local_pos0=n_pre, out=out, lse=lse, workspace=ws)
    for i in range(4):
        q.copy_(torch.randn_like(q.float()).to(torch.bfloat16))
        q_pos.sub_(i % 2)
        graph.replay()
        torch.cuda.synchronize()
        o, y = msa.msa_prefix_attend(cfg, q, Kp, Vp, K, V, q_pos, local_pos0=n_pre)
        torch.cuda.synchronize()
        assert torch.equal(o, out) and torch.equal(y, lse), i
    with torch.cuda.stream(side):
        o2, y2 = msa.msa_prefix_attend(cfg, q, Kp, Vp, K, V, q_pos, local_pos0=n_pre, workspace=ws)
    side.synchronize()
    assert torch.equal(o2, out) and torch.equal(y2, lse)


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 40])
def test_offsets_past_32_bits(M):
    """A prefix of 2.2 billion elements and caches of as many: the last rows of the last head are found."""
    B, Hkv, n, d = 2, 4, 4_300_000, 128
    cfg = _cfg(8, Hkv, d)
    q, Ks, Vs, Kt, Vt = _make(B, M, 8, Hkv, d, 40, 60, 10)
    lens = torch.tensor([n, n], dtype=torch.int32)
    # everything but the last rows scores far below them
    Kp, Vp = (torch.zeros((Hkv, n, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    big = torch.full((B, M, 8, d), 4.0, dtype=torch.bfloat16)
    Kp[:, n - 40:], Vp[:, n - 40:] = (Ks + 8).to(torch.bfloat16).cuda(), Vs.cuda()
    out, lse = msa.msa_prefix_attend(cfg, big.cuda(), Kp, Vp, Kt.cuda(), Vt.cuda(), torch.full((B, M), -1, dtype=torch.int32, device="cuda"),
                                     prefix_lens=lens.cuda())
    torch.cuda.synchronize()
    C.prefix_attend(big.double(), (Ks + 8).to(torch.bfloat16).double(), Vs.double(), None, Kt.double(), Vt.double(),
                    torch.full((B, M), -1), 0).check(out, lse)
    del Kp, Vp
    L = 2_150_000
    K, V = (torch.zeros((B, Hkv, L, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    K[:, :, L - 60:], V[:, :, L - 60:] = (Kt + 8).to(torch.bfloat16).cuda(), Vt.cuda()
    q_pos = torch.full((B, M), L - 1, dtype=torch.int32)
    out, lse = msa.msa_prefix_attend(cfg, big.cuda(), None, None, K, V, q_pos.cuda())
    torch.cuda.synchronize()
    C.prefix_attend(big.double(), Ks[:, :0].double(), Vs[:, :0].double(), None, (Kt + 8).to(torch.bfloat16).double(), Vt.double(),
                    torch.full((B, M), 59), 0).check(out, lse)
    del K, V
    torch.cuda.empty_cache()


@pytest.mark.gpu
def test_two_streams_at_once():
    cfg = _cfg(8, 1, 128)
    sets = [[t.cuda() for t in _make(6, 1, 8, 1, 128, 3000, 400, 20 + i)] for i in range(3)]
    pos = torch.full((6, 1), 3399, dtype=torch.int32, device="cuda")
    want = [msa.msa_prefix_attend(cfg, *s, pos, local_pos0=3000) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(20):
        got = [msa.msa_prefix_attend(cfg, *s, pos, local_pos0=3000, stream=st) for s, st in zip(sets, streams)]
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.gpu
def test_python_refusals():
    cfg = _cfg()
    q, Kp, Vp, K, V = (t.cuda() for t in _make(2, 3, 8, 2, 64, 9, 7))
    pos, lens = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((2, 3), (2,)))
    good = dict(q=q, Kpre=Kp, Vpre=Vp, Kloc=K, Vloc=V, q_pos=pos)
    msa.msa_prefix_attend(cfg, **good, prefix_lens=lens)
    for bad in (dict(q=q[:1]), dict(q=q.transpose(1, 2)), dict(Kpre=Kp[None]), dict(Vpre=Vp[:, :5]), dict(Vpre=None), dict(Kloc=None),
                dict(Kloc=K[:, :, :5]), dict(Vloc=V.float()), dict(q_pos=pos.long()), dict(prefix_lens=lens[:1]), dict(out=q[:1]),
                dict(workspace=torch.zeros(256, device="cuda"))):
        with pytest.raises(ValueError):
            msa.msa_prefix_attend(cfg, **{**good, **bad})
    with pytest.raises(msa.MsaError):
        msa.msa_prefix_attend(cfg, q, None, None, None, None, pos)
