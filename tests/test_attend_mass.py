"""msa_attend_mass against the plain definition in 64 bits: windows, first tokens, padding, old weights that fade."""
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
    a = dict(q=p, B=1, M=1, K=p, L=64, pos0=0, W=16, S=0, q_pos=p, lse=p, mass=p, decay=1.0, out=p, ws=p, bytes=1 << 40)
    a.update(kw)
    return lib.msa_attend_mass(ctypes.byref(cfg), a["q"], a["B"], a["M"], a["K"], a["L"], a["pos0"], a["W"], a["S"], a["q_pos"],
                               a["lse"], a["mass"], a["decay"], a["out"], a["ws"], a["bytes"], None)


@pytest.mark.parametrize("kw, status", [
    (dict(q=None), -1), (dict(K=None), -1), (dict(q_pos=None), -1), (dict(lse=None), -1), (dict(out=None), -1), (dict(ws=None), -1),
    (dict(B=0), -1), (dict(M=0), -1), (dict(L=0), -1), (dict(W=0), -1), (dict(S=-1), -1), (dict(pos0=-1), -1),
    (dict(decay=-0.1), -1), (dict(decay=1.5), -1), (dict(decay=float("nan")), -1),
    (dict(B=65536), -2), (dict(B=1 << 13, M=1 << 13), -2), (dict(L=(1 << 28) + 1), -2), (dict(bytes=255), -3),
    (dict(B=4, L=1 << 28), -2), (dict(B=4, M=100, L=1 << 28), -2),      # 2^24 blocks of 128 rows
    (dict(q=ctypes.c_void_p(0x10008)), -4), (dict(K=ctypes.c_void_p(0x10002)), -4), (dict(q_pos=ctypes.c_void_p(0x10002)), -4),
    (dict(lse=ctypes.c_void_p(0x10002)), -4), (dict(mass=ctypes.c_void_p(0x10002)), -4), (dict(out=ctypes.c_void_p(0x10002)), -4),
    (dict(ws=ctypes.c_void_p(0x10010 + 4)), -4),
])
def test_refusals(lib, kw, status):
    assert _call(lib, _cfg(), **kw) == status


def test_workspace_sizes(lib):
    for cfg, B, M, L in itertools.product((_cfg(32, 8, 128), _cfg(8, 1, 64)), (1, 3), (1, 40, 700, 9000), (1, 500, 9000)):
        n = msa.attend_mass_workspace_bytes(cfg, B, M, L, L, 0)
        assert n >= 256 and n % 256 == 0
        assert _call(lib, cfg, B=B, M=M, L=L, W=L, bytes=n - 1) == msa.MSA_ERR_WORKSPACE
    for cfg, B, M in itertools.product((_cfg(32, 8, 128), _cfg(8, 1, 64)), (1, 3, 40), (1, 40, 700, 9000)):   # a longer cache: no less
        sizes = [msa.attend_mass_workspace_bytes(cfg, B, M, L, L) for L in (1, 255, 256, 257, 1000, 9000, 70000, 700000)]
        assert sizes == sorted(sizes)
    with pytest.raises(ValueError):
        msa.attend_mass_workspace_bytes(_cfg(), 1, 2 ** 32 + 1, 8, 8)
    assert msa.attend_mass_workspace_bytes(_cfg(), 1, 1, 0, 8) == 0


def _make(B, M, Hq, Hkv, d, L, seed=0):
    g = torch.Generator().manual_seed(seed)
    q, K, V = (torch.randn(s, generator=g).to(torch.bfloat16) for s in ((B, M, Hq, d), (B, Hkv, L, d), (B, Hkv, L, d)))
    return q, K, V, torch.rand((B, Hkv, L), generator=g) * 3


def _lse(Hq, Hkv, d, q, K, V, q_pos, W, S, pos0):
    return msa.msa_window_attend(_cfg(Hq, Hkv, d), q.cuda(), K.cuda(), V.cuda(), q_pos.cuda(), W, sinks=S, local_pos0=pos0)[1]


def _check(Hq, Hkv, d, q, K, V, mass, q_pos, W, S, pos0, decay=1.0, in_place=False):
    B, M = q.shape[:2]
    L = K.shape[2]
    cfg = _cfg(Hq, Hkv, d)
    lse = _lse(Hq, Hkv, d, q, K, V, q_pos, W, S, pos0)
    ws = torch.full((msa.attend_mass_workspace_bytes(cfg, B, M, L, W, S),), 0xA5, dtype=torch.uint8, device="cuda")
    Kd = K.clone()
    for b in range(B):          # what lies behind every token of a sequence has no effect
        Kd[b, :, max(0, int(q_pos[b].max()) - pos0 + 1):] = float("nan")
    old = None if mass is None else mass.cuda()
    out = msa.msa_attend_mass(cfg, q.cuda(), Kd.cuda(), lse, q_pos.cuda(), W, sinks=S, local_pos0=pos0, mass=old, decay=decay,
                              out=old if in_place else torch.full((B, Hkv, L), 7.0, device="cuda"), workspace=ws)
    torch.cuda.synchronize()
    want, tol = C.attend_mass(q.double(), K.double(), lse.double().cpu(), q_pos, W, S, pos0, mass, decay)
    err = (out.double().cpu() - want).abs()
    assert bool((err <= tol).all()), float((err - tol).max())
    return out


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 3, 8, 45, 130])
@pytest.mark.parametrize("Hq, Hkv, d", [(4, 4, 64), (4, 2, 128), (6, 2, 64), (8, 1, 128), (5, 1, 128)])
@pytest.mark.parametrize("L, W, S", [(1, 1, 0), (50, 1, 0), (50, 7, 3), (97, 32, 33), (130, 200, 4), (161, 33, 0)])
def test_against_64_bits(M, Hq, Hkv, d, L, W, S):
    q, K, V, mass = _make(2, M, Hq, Hkv, d, L, M + L)
    pos0 = 5
    last = torch.tensor([[L - 1], [max(L // 2, 0)]]) + pos0
    q_pos = (last - M + 1 + torch.arange(M)).to(torch.int32)      # the first tokens may lie in front of the cache: they see nothing
    _check(Hq, Hkv, d, q, K, V, mass, q_pos, W, S, pos0, decay=(0.9, 1.0)[M % 2])


@pytest.mark.gpu
@pytest.mark.parametrize("M", [2, 70])
def test_positions_in_any_order(M):
    """Padding, positions past the cache's end, the same position twice, tokens far apart in one tile."""
    g = torch.Generator().manual_seed(2)
    q, K, V, mass = _make(3, M, 4, 2, 64, 300, 1)
    q_pos = torch.randint(-3, 340, (3, M), generator=g, dtype=torch.int32)
    q_pos[0, 0], q_pos[1, 1], q_pos[2] = -2 ** 31, 2 ** 31 - 1, -1
    for W, S in ((16, 4), (400, 0), (1, 0), (2 ** 31 - 1, 2 ** 31 - 1), (60, 100)):
        out = _check(4, 2, 64, q, K, V, mass, q_pos, W, S, 0)
        assert torch.equal(out[2].cpu(), mass[2])


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 70])
def test_old_weights(M):
    """Added to, faded, dropped (whatever they hold), in place; all weights of a token's rows add up to one per head."""
    q, K, V, mass = _make(2, M, 4, 2, 128, 200, 3)
    q_pos = (199 - M + 1 + torch.arange(M)).expand(2, M).contiguous().to(torch.int32)
    q_pos[1] -= 20
    args = (4, 2, 128, q, K, V)
    for decay in (1.0, 0.25):
        a = _check(*args, mass, q_pos, 400, 0, 0, decay=decay)
        b = _check(*args, mass, q_pos, 400, 0, 0, decay=decay, in_place=True)
        assert torch.equal(a, b)
    bad = torch.full_like(mass, float("nan"))
    a, b = _check(*args, None, q_pos, 400, 0, 0), _check(*args, bad, q_pos, 400, 0, 0, decay=0.0)
    assert torch.equal(a, b) and float(a[1, :, 180:].abs().max()) == 0.0
    assert float((a.double().sum(-1) - 2 * M).abs().max()) <= 2 * M * 1e-3      # the sum of 2 heads' M softmaxes, bound as above


@pytest.mark.gpu
@pytest.mark.parametrize("B, M, L, W", [(1, 600, 600, 600), (1, 300, 3000, 100), (3, 257, 401, 128), (1, 1, 5000, 5000), (2, 7, 2500, 2500)])
def test_long(B, M, L, W):
    q, K, V, mass = _make(B, M, 2, 1, 128, L, 4)
    q_pos = (L - M + torch.arange(M)).expand(B, M).contiguous().to(torch.int32)
    _check(2, 1, 128, q, K, V, mass, q_pos, W, 3, 0)


@pytest.mark.gpu
def test_of_a_joint_softmax():
    """With the log-sum over a prefix and a cache, the cache's rows get their share of it."""
    B, M, Hq, Hkv, d, n_pre, L = 2, 3, 4, 2, 64, 90, 40
    q, K, V, _ = _make(B, M, Hq, Hkv, d, L, 9)
    g = torch.Generator().manual_seed(1)
    Kp, Vp = (torch.randn((Hkv, n_pre, d), generator=g).to(torch.bfloat16) for _ in range(2))
    q_pos = (n_pre + L - M + torch.arange(M)).expand(B, M).contiguous().to(torch.int32)
    cfg = _cfg(Hq, Hkv, d)
    lse = msa.msa_prefix_attend(cfg, q.cuda(), Kp.cuda(), Vp.cuda(), K.cuda(), V.cuda(), q_pos.cuda(), local_pos0=n_pre)[1]
    out = msa.msa_attend_mass(cfg, q.cuda(), K.cuda(), lse, q_pos.cuda(), L, local_pos0=n_pre)
    want, tol = C.attend_mass(q.double(), K.double(), lse.double().cpu(), q_pos, L, 0, n_pre, None, 1.0)
    assert bool(((out.double().cpu() - want).abs() <= tol).all())


@pytest.mark.gpu
@pytest.mark.parametrize("M", [3, 70])
def test_queries_of_padding_may_be_anything(M):
    q, K, V, mass = _make(2, M, 4, 2, 64, 90, 9)
    q_pos = (90 - M + torch.arange(M)).expand(2, M).contiguous().to(torch.int32)
    q_pos[:, ::2] = -1
    lse = _lse(4, 2, 64, q, K, V, q_pos, 30, 2, 0)
    bad, bad_lse = q.clone(), lse.clone()
    bad[:, ::2], bad_lse[:, ::2] = float("nan"), float("nan")
    a, b = (msa.msa_attend_mass(_cfg(4, 2, 64), x.cuda(), K.cuda(), y, q_pos.cuda(), 30, sinks=2, mass=mass.cuda())
            for x, y in ((q, lse), (bad, bad_lse)))
    assert torch.equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("B, M, L", [(4, 1, 900), (1, 70, 700), (1, 500, 500)])
def test_graph_replays_and_streams(B, M, L):
    cfg = _cfg(8, 2, 128)
    q, K, V, mass = (t.cuda() for t in _make(B, M, 8, 2, 128, L, 7))
    q_pos = (L - M + torch.arange(M)).expand(B, M).contiguous().to(torch.int32).cuda()
    lse = torch.full((B, M, 8), 6.0, device="cuda")
    ws = torch.full((msa.attend_mass_workspace_bytes(cfg, B, M, L, L, 0),), 0xFF, dtype=torch.uint8, device="cuda")
    out, side = torch.empty_like(mass), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        msa.msa_attend_mass(cfg, q, K, lse, q_pos, L, mass=mass, out=out, workspace=ws)
    for i in range(4):
        q.copy_(torch.randn_like(q.float()).to(torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        want = msa.msa_attend_mass(cfg, q, K, lse, q_pos, L, mass=mass)
        torch.cuda.synchronize()
        assert torch.equal(want, out), i
    got = msa.msa_attend_mass(cfg, q, K, lse, q_pos, L, mass=mass, stream=side)
    side.synchronize()
    assert torch.equal(got, out)


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 66])
def test_offsets_past_32_bits(M):
    """A cache of 2.2 billion elements: the last rows of the last head are found."""
    B, Hkv, L, d = 2, 4, 2_150_000, 128
    cfg = _cfg(8, Hkv, d)
    K = torch.zeros((B, Hkv, L, d), dtype=torch.bfloat16, device="cuda")
    q, Ks, _, _ = _make(B, M, 8, Hkv, d, 300, 10)
    K[:, :, L - 300:] = Ks.cuda()
    q_pos = (L - M + torch.arange(M)).expand(B, M).contiguous().to(torch.int32)
    lse = torch.full((B, M, 8), 7.0)
    out = msa.msa_attend_mass(cfg, q.cuda(), K, lse.cuda(), q_pos.cuda(), 200)
    torch.cuda.synchronize()
    want, tol = C.attend_mass(q.double(), Ks.double(), lse.double(), q_pos - (L - 300), 200, 0, 0, None, 1.0)
    assert bool(((out[:, :, L - 300:].double().cpu() - want).abs() <= tol).all())
    assert float(out[:, :, :L - 300].abs().max()) == 0.0
    del K
    torch.cuda.empty_cache()


@pytest.mark.gpu
def test_python_refusals():
    cfg = _cfg()
    q, K, _, mass = (t.cuda() for t in _make(2, 3, 8, 2, 64, 9))
    pos, lse = torch.zeros((2, 3), dtype=torch.int32, device="cuda"), torch.zeros((2, 3, 8), device="cuda")
    good = dict(q=q, Kloc=K, lse=lse, q_pos=pos, window=4, mass=mass)
    msa.msa_attend_mass(cfg, **good)
    for bad in (dict(q=q[:1]), dict(q=q.transpose(1, 2)), dict(Kloc=K[:, :, ::2]), dict(lse=lse.half()), dict(lse=lse[:, :1]),
                dict(q_pos=pos.long()), dict(mass=mass[:1]), dict(mass=mass.double()), dict(out=mass[0])):
        with pytest.raises(ValueError):
            msa.msa_attend_mass(cfg, **{**good, **bad})
    for bad in (dict(window=0), dict(decay=2.0)):
        with pytest.raises(msa.MsaError):
            msa.msa_attend_mass(cfg, **{**good, **bad})
