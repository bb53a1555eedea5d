"""msa_evict against sorting: which rows stay, their order, ties, odd weights, in place and to other buffers."""
import ctypes

import pytest
import torch

import paper_2603_23516_amd as msa
import plain64_cache as C


def _cfg(Hkv=2, d=64):
    return msa.MsaConfig(1, 1, 1, Hkv, Hkv, d, 1e4)


@pytest.fixture(scope="module")
def lib():
    return msa.load_library()


def _call(lib, cfg, **kw):
    p, o = ctypes.c_void_p(0x10000), ctypes.c_void_p(0x20000)
    a = dict(K=p, V=p, mass=p, lens=p, B=1, L=64, keep=16, S=2, R=4, Ko=o, Vo=o, mo=o, Lo=16, rows=o)
    a.update(kw)
    return lib.msa_evict(ctypes.byref(cfg), a["K"], a["V"], a["mass"], a["lens"], a["B"], a["L"], a["keep"], a["S"], a["R"], a["Ko"],
                         a["Vo"], a["mo"], a["Lo"], a["rows"], None)


_P = ctypes.c_void_p(0x10000)


@pytest.mark.parametrize("kw, status", [
    (dict(K=None), -1), (dict(V=None), -1), (dict(mass=None), -1), (dict(lens=None), -1), (dict(Ko=None), -1), (dict(Vo=None), -1),
    (dict(mo=None), -1), (dict(rows=None), -1), (dict(B=0), -1), (dict(L=0), -1), (dict(keep=0), -1), (dict(keep=17), -1),
    (dict(S=-1), -1), (dict(R=-1), -1), (dict(S=13), -1), (dict(S=2 ** 31 - 1, R=2 ** 31 - 1), -1),
    (dict(Ko=_P), -1), (dict(Vo=_P), -1), (dict(mo=_P), -1), (dict(Ko=_P, Vo=_P, mo=_P), -1),
    (dict(B=65536), -2), (dict(L=(1 << 28) + 1), -2), (dict(Lo=(1 << 28) + 1), -2), (dict(B=16384, keep=16385, Lo=16385), -2),
    (dict(K=ctypes.c_void_p(0x10008)), -4), (dict(mass=ctypes.c_void_p(0x10002)), -4), (dict(lens=ctypes.c_void_p(0x10002)), -4),
    (dict(Vo=ctypes.c_void_p(0x20008)), -4), (dict(rows=ctypes.c_void_p(0x20002)), -4),
])
def test_refusals(lib, kw, status):
    assert _call(lib, _cfg(), **kw) == status


def _weights(B, Hkv, L, kind, g):
    if kind == "spread":
        return torch.exp(1.5 * torch.randn((B, Hkv, L), generator=g))
    if kind == "ties":           # few values, zeros of both signs
        return torch.randint(-1, 3, (B, Hkv, L), generator=g).float() * torch.where(torch.rand((B, Hkv, L), generator=g) < 0.5, 0.0, 1.0)
    if kind == "equal":
        return torch.full((B, Hkv, L), 0.25)
    m = torch.randn((B, Hkv, L), generator=g) * 1e-38      # subnormals among them
    x = torch.rand((B, Hkv, L), generator=g)
    m[x < 0.1], m[x > 0.9] = float("nan"), float("-inf")
    m[(x > 0.5) & (x < 0.55)] = float("inf")
    m[(x > 0.6) & (x < 0.65)] = -float("nan")
    return m


def _check(K, V, mass, lens, keep, S, R, in_place, Lo=None, **kw):
    B, Hkv, L, d = K.shape
    Lo = L if in_place else (keep if Lo is None else Lo)
    if in_place:
        Ko, Vo, mo = K.clone(), V.clone(), mass.clone()
    else:
        Ko, Vo = (torch.full((B, Hkv, Lo, d), 3.0, dtype=torch.bfloat16) for _ in range(2))
        mo = torch.full((B, Hkv, Lo), -9.0)
    want = [Ko.clone(), Vo.clone(), mo.clone(), torch.full((B, Hkv, keep), -1, dtype=torch.int32)]
    for b in range(B):
        n = min(max(int(lens[b]), 0), L)
        for g in range(Hkv):
            rows = C.evict_rows(mass[b, g], n, keep, S, R)
            at = torch.tensor(rows, dtype=torch.long)
            want[2][b, g] = 0.0
            for x, y in zip(want[:3], (K, V, mass)):
                x[b, g, :len(rows)] = y[b, g, at]
            want[3][b, g, :len(rows)] = at.to(torch.int32)
    dev = [t.cuda() for t in (Ko, Vo, mo)]
    if in_place:
        got = msa.msa_evict(_cfg(Hkv, d), *dev, lens.cuda(), keep, sinks=S, recent=R, **kw)
        assert all(a is b for a, b in zip(got, dev))
    else:
        src = [t.cuda() for t in (K, V, mass)]
        got = msa.msa_evict(_cfg(Hkv, d), *src, lens.cuda(), keep, sinks=S, recent=R, Kout=dev[0], Vout=dev[1], mass_out=dev[2], **kw)
    torch.cuda.synchronize()
    for x, y, name in zip(got, want, ("Kout", "Vout", "mass_out", "rows")):
        x = x.cpu()
        same = torch.equal(x.view(torch.int32), y.view(torch.int32)) if x.dtype == torch.float32 else torch.equal(x, y)
        assert same, name
    return got


def _make(B, Hkv, L, d, kind="spread", seed=0):
    g = torch.Generator().manual_seed(seed)
    K, V = (torch.randn((B, Hkv, L, d), generator=g).to(torch.bfloat16) for _ in range(2))
    return K, V, _weights(B, Hkv, L, kind, g)


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("kind", ["spread", "ties", "equal", "odd"])
@pytest.mark.parametrize("Hkv, d, L, keep, S, R", [(1, 64, 1, 1, 0, 0), (2, 64, 2, 1, 0, 1), (3, 128, 65, 64, 0, 0), (2, 64, 130, 33, 4, 7),
                                                   (2, 128, 300, 20, 12, 8), (1, 64, 3000, 1100, 3, 100), (1, 128, 2100, 2099, 0, 0)])
def test_against_sorting(in_place, kind, Hkv, d, L, keep, S, R):
    K, V, mass = _make(3, Hkv, L, d, kind, L + keep)
    lens = torch.tensor([L, max(1, L - 5), max(0, keep - 3)], dtype=torch.int32)
    _check(K, V, mass, lens, keep, S, R, in_place)


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True])
def test_lengths(in_place):
    """Empty sequences, lengths out of range, exactly keep, one more; a buffer longer than what is kept."""
    K, V, mass = _make(7, 2, 90, 64, "ties", 3)
    lens = torch.tensor([0, -4, 1000, 40, 41, 90, 39], dtype=torch.int32)
    _check(K, V, mass, lens, 40, 2, 5, in_place, Lo=57)
    _check(K, V, mass, lens, 90, 2, 5, in_place, Lo=120)


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("L, keep", [(32769, 9000), (70001, 69990), (140000, 70)])
def test_long_caches(in_place, L, keep):
    for kind in ("spread", "ties", "odd"):
        K, V, mass = _make(1, 1, L, 64, kind, 5)
        _check(K, V, mass, torch.tensor([L - 1], dtype=torch.int32), keep, 4, 33, in_place)


@pytest.mark.gpu
def test_again_and_again():
    """Cut in place, appended to and cut again: as one would do by hand."""
    K, V, mass = _make(2, 2, 64, 64, "spread", 7)
    lens = torch.tensor([64, 50], dtype=torch.int32)
    for i in range(4):
        K, V, mass, _ = (t.cpu() for t in _check(K, V, mass, lens, 40, 1, 3, True))
        lens = lens.clamp(max=40) + torch.tensor([7, 1], dtype=torch.int32)


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True])
def test_graph_replays_and_streams(in_place):
    cfg, keep = _cfg(2, 128), 300
    src = [t.cuda() for t in _make(2, 2, 1000, 128, "spread", 9)]
    bufs = [t.clone() for t in src]
    outs = {} if in_place else dict(Kout=torch.zeros((2, 2, keep, 128), dtype=torch.bfloat16, device="cuda"),
                                    Vout=torch.zeros((2, 2, keep, 128), dtype=torch.bfloat16, device="cuda"),
                                    mass_out=torch.zeros((2, 2, keep), device="cuda"))
    lens, rows = torch.tensor([1000, 777], dtype=torch.int32, device="cuda"), torch.zeros((2, 2, keep), dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        msa.msa_evict(cfg, *bufs, lens, keep, sinks=2, recent=9, rows=rows, **outs)
    for i in range(4):
        src[2].copy_(torch.rand_like(src[2]))
        for x, y in zip(bufs, src):
            x.copy_(y)
        graph.replay()
        torch.cuda.synchronize()
        got = bufs if in_place else list(outs.values())
        fresh = [torch.zeros_like(t) for t in got]
        k, v, m, rw = msa.msa_evict(cfg, *src, lens, keep, sinks=2, recent=9, Kout=fresh[0], Vout=fresh[1], mass_out=fresh[2],
                                    stream=side)
        side.synchronize()
        assert torch.equal(rw, rows)
        for x, y in zip(got, (k, v, m)):
            assert torch.equal(x[:, :, :keep], y[:, :, :keep]), i


@pytest.mark.gpu
def test_offsets_past_32_bits():
    """A cache of 2.2 billion elements: rows of the last head's end."""
    B, Hkv, L, d, keep = 2, 4, 2_150_000, 128, 50
    g = torch.Generator().manual_seed(3)
    K = torch.zeros((B, Hkv, L, d), dtype=torch.bfloat16, device="cuda")
    mass = torch.zeros((B, Hkv, L), device="cuda")
    tail = torch.randn((B, Hkv, 200, d), generator=g).to(torch.bfloat16).cuda()
    K[:, :, L - 200:] = tail
    mass[:, :, L - 200:] = 1 + torch.rand((B, Hkv, 200), generator=g).cuda()
    lens = torch.full((B,), L, dtype=torch.int32, device="cuda")
    Ko, Vo = (torch.zeros((B, Hkv, keep, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    mo = torch.zeros((B, Hkv, keep), device="cuda")
    rows = msa.msa_evict(_cfg(Hkv, d), K, K, mass, lens, keep, Kout=Ko, Vout=Vo, mass_out=mo)[3]
    torch.cuda.synchronize()
    for b in range(B):
        for h in range(Hkv):
            at = torch.tensor(C.evict_rows(mass[b, h, L - 200:].cpu(), 200, keep, 0, 0))
            assert torch.equal(rows[b, h].cpu().long(), at + L - 200)
            assert torch.equal(Ko[b, h], tail[b, h, at.cuda()]) and torch.equal(Vo[b, h], Ko[b, h])
    msa.msa_evict(_cfg(Hkv, d), K, K.clone(), mass, lens, keep, Kout=None)
    torch.cuda.synchronize()
    assert torch.equal(K[:, :, :keep], Ko)
    del K
    torch.cuda.empty_cache()


@pytest.mark.gpu
def test_python_refusals():
    cfg = _cfg()
    K, V, mass = (t.cuda() for t in _make(2, 2, 9, 64))
    lens = torch.full((2,), 9, dtype=torch.int32, device="cuda")
    out = dict(Kout=K[:, :, :5].clone(), Vout=K[:, :, :5].clone(), mass_out=mass[:, :, :5].clone())
    good = dict(Kloc=K, Vloc=V, mass=mass, lens=lens, keep=5)
    msa.msa_evict(cfg, **good, **out)
    for bad in (dict(Vloc=V[:1]), dict(mass=mass.double()), dict(lens=lens.long()), dict(lens=lens[:1]), dict(Kout=None), dict(mass_out=None),
                dict(Vout=out["Vout"][:, :, :4]), dict(keep=2 ** 40), dict(rows=torch.zeros((2, 2, 4), dtype=torch.int32, device="cuda"))):
        with pytest.raises(ValueError):
            msa.msa_evict(cfg, **{**good, **out, **bad})
    for bad in (dict(keep=6), dict(keep=0), dict(sinks=3, recent=3)):
        with pytest.raises(msa.MsaError):
            msa.msa_evict(cfg, **{**good, **out, **bad})
