"""msa_norm_rotate_axes against the plain definition in 64 bits: positions of several axes, rows told apart from positions."""
import ctypes

import pytest
import torch

import paper_2603_23516_amd as msa
import plain64 as P
import plain64_cache as C


def _cfg(Hq=8, Hkv=2, d=64, base=1e4):
    return msa.MsaConfig(1, 1, 1, Hq, Hkv, d, base)


@pytest.fixture(scope="module")
def lib():
    return msa.load_library()


def _call(lib, cfg, **kw):
    p = ctypes.c_void_p(0x10000)
    a = dict(q=p, k=p, v=p, pos=p, A=3, axes=[u % 3 for u in range(cfg.head_dim // 2)], rows=p, B=1, M=1, q_out=p, K=p, V=p,
             L=8, pos0=0, eps=1e-6, rotate=1, w=p, stride=1024)
    a.update(kw)
    axes = None if a["axes"] is None else (ctypes.c_int32 * len(a["axes"]))(*a["axes"])
    return lib.msa_norm_rotate_axes(ctypes.byref(cfg), a["q"], a["stride"], a["k"], a["stride"], a["v"], a["stride"], a["w"],
                                    a["w"], a["eps"], a["rotate"], a["pos"], a["A"], axes, a["rows"], a["B"], a["M"], a["q_out"],
                                    a["K"], a["V"], a["L"], a["pos0"], None)


@pytest.mark.parametrize("kw, status", [
    (dict(pos=None), -1), (dict(q=None), -1), (dict(k=None), -1), (dict(V=None), -1), (dict(B=0), -1), (dict(M=0), -1),
    (dict(L=-1), -1), (dict(pos0=-1), -1), (dict(eps=0.0), -1), (dict(rotate=2), -1), (dict(stride=100), -1),
    (dict(A=0), -1), (dict(axes=None), -1), (dict(axes=[0] * 31 + [3]), -1), (dict(axes=[-1] + [0] * 31), -1),
    (dict(A=5), -2), (dict(B=1 << 13, M=1 << 13), -2),
    (dict(rows=ctypes.c_void_p(0x10002)), -4), (dict(pos=ctypes.c_void_p(0x10002)), -4), (dict(stride=1028), -4),
])
def test_refusals(lib, kw, status):
    assert _call(lib, _cfg(), **kw) == status


def _case(B, M, Hq, Hkv, d, A, L, seed=0, far=1000):
    g = torch.Generator().manual_seed(seed)
    qkv = torch.randn((B, M, (Hq + 2 * Hkv) * d), generator=g).to(torch.bfloat16) * 2
    pos = torch.randint(0, far, (B, M, A), generator=g, dtype=torch.int32)
    rows = torch.stack([torch.randperm(L, generator=g)[:M] for _ in range(B)]).to(torch.int32)
    w = [(1 + 0.2 * torch.randn(d, generator=g)).to(torch.bfloat16) for _ in range(2)]
    return qkv, pos, rows, w


def _split(qkv, Hq, Hkv, d):
    return (qkv[..., :Hq * d].unflatten(-1, (Hq, d)), qkv[..., Hq * d:(Hq + Hkv) * d].unflatten(-1, (Hkv, d)),
            qkv[..., (Hq + Hkv) * d:].unflatten(-1, (Hkv, d)))


def _want(x, w, pos, axes, base, rotate):
    y = P.norm(x.double(), None if w is None else w.double(), 1e-6)
    return C.rotate_axes(y, pos, axes, base) if rotate else y


def _near(got, want, size):
    """Rounded to bf16 once (2^-8); the norm and the rotation in fp32: a few times 2^-23 of the pair's size."""
    err = (got.double().cpu() - want).abs()
    assert bool((err <= 2.0 ** -8 * want.abs() + 2.0 ** -20 * size).all()), float(err.max())


@pytest.mark.gpu
@pytest.mark.parametrize("A, mixed", [(1, False), (2, True), (3, False), (3, True), (4, True)])
@pytest.mark.parametrize("B, M, Hq, Hkv, d, weights, rotate", [
    (1, 1, 8, 2, 64, True, True), (3, 5, 32, 8, 128, True, True), (2, 37, 5, 1, 128, False, True), (2, 9, 6, 3, 64, True, False)])
def test_against_64_bits(A, mixed, B, M, Hq, Hkv, d, weights, rotate):
    L = M + 11
    qkv, pos, rows, w = _case(B, M, Hq, Hkv, d, A, L, A + M)
    axes = [u % A if mixed else u * A // (d // 2) for u in range(d // 2)]
    pos[-1, -1] = -1                                                 # padding
    if A > 1:
        pos[0, 0, 1] = -77                                           # a further axis has any sign
    if M > 4:
        rows[0, 3], rows[0, 4] = -1, L                               # no rows of the cache
    w = w if weights else (None, None)
    q, k, v = _split(qkv.cuda(), Hq, Hkv, d)
    old = [torch.randn((B, Hkv, L, d)).to(torch.bfloat16) for _ in range(2)] + [torch.randn((B, M, Hq, d)).to(torch.bfloat16)]
    K, V, qo = (t.cuda() for t in old)
    dev = [None if x is None else x.cuda() for x in w]
    msa.msa_norm_rotate_axes(_cfg(Hq, Hkv, d), q, k, v, pos.cuda(), axes, K, V, rows=rows.cuda(), q_weight=dev[0], k_weight=dev[1],
                             rotate=rotate, q_out=qo)
    torch.cuda.synchronize()
    q, k, v = _split(qkv, Hq, Hkv, d)
    wq, wk = (_want(x, y, pos, axes, 1e4, rotate) for x, y in ((q, w[0]), (k, w[1])))
    wantK, wantV = old[0].double(), old[1].double()
    here = pos[..., 0] >= 0
    for b in range(B):
        for m in range(M):
            if bool(here[b, m]) and 0 <= int(rows[b, m]) < L:
                wantK[b, :, int(rows[b, m])], wantV[b, :, int(rows[b, m])] = wk[b, m], v[b, m].double()
    size = 8.0 if not weights else 16.0                              # |x| < 12 without a norm, < 2 d^(1/2) with one
    _near(qo, torch.where(here[..., None, None], wq, old[2].double()), size)
    _near(K, wantK, size)
    assert torch.equal(V.cpu().double(), wantV)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
def test_one_axis_is_msa_norm_rotate(d):
    """All pairs on one axis, rows from the positions: the same bits as msa_norm_rotate; and without rows the first axis counts."""
    B, M, Hq, Hkv, L = 2, 50, 8, 2, 70
    qkv, _, _, w = _case(B, M, Hq, Hkv, d, 1, L, 3)
    q, k, v = _split(qkv.cuda(), Hq, Hkv, d)
    pos = (100 + torch.arange(M) + 7 * torch.arange(B)[:, None]).to(torch.int32).cuda()
    pos[1, 3] = -5
    w = [x.cuda() for x in w]
    cfg = _cfg(Hq, Hkv, d)
    a, b, c = ([torch.zeros((B, Hkv, L, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)] +
               [torch.zeros((B, M, Hq, d), dtype=torch.bfloat16, device="cuda")] for _ in range(3))
    msa.msa_norm_rotate(cfg, q, k, v, pos, a[0], a[1], q_weight=w[0], k_weight=w[1], local_pos0=100, q_out=a[2])
    msa.msa_norm_rotate_axes(cfg, q, k, v, pos[..., None].contiguous(), [0] * (d // 2), b[0], b[1], q_weight=w[0], k_weight=w[1],
                             local_pos0=100, q_out=b[2])
    two = torch.stack([pos, pos + 1], -1).contiguous()
    msa.msa_norm_rotate_axes(cfg, q, k, v, two, [0] * (d // 2), c[0], c[1], rows=pos - 100, q_weight=w[0], k_weight=w[1], q_out=c[2])
    torch.cuda.synchronize()
    for x, y, z in zip(a, b, c):
        assert torch.equal(x, y) and torch.equal(x, z)


@pytest.mark.gpu
def test_far_positions_and_parts():
    """Positions of a long video, keys or queries alone, a stream of its own."""
    B, M, Hq, Hkv, d, A, L = 1, 20, 4, 2, 128, 3, 20
    qkv, pos, rows, w = _case(B, M, Hq, Hkv, d, A, L, 8, far=2 ** 31 - 1)
    axes = [u * A // (d // 2) for u in range(d // 2)]
    q, k, v = _split(qkv.cuda(), Hq, Hkv, d)
    K = torch.zeros((B, Hkv, L, d), dtype=torch.bfloat16, device="cuda")
    cfg, side = _cfg(Hq, Hkv, d, 1e6), torch.cuda.Stream()
    p, rw = pos.cuda(), rows.cuda()
    torch.cuda.synchronize()
    qo = msa.msa_norm_rotate_axes(cfg, q, None, None, p, axes, None, None, rows=rw, stream=side)
    assert msa.msa_norm_rotate_axes(cfg, None, k, None, p, axes, K, None, rows=rw, stream=side) is None
    side.synchronize()
    q, k, _ = _split(qkv, Hq, Hkv, d)
    _near(qo, C.rotate_axes(q.double(), pos, axes, 1e6), 8.0)
    want = C.rotate_axes(k.double(), pos, axes, 1e6)[0]
    _near(K[0][:, rows[0].long()].transpose(0, 1), want, 8.0)


@pytest.mark.gpu
def test_python_refusals():
    cfg = _cfg()
    z = dict(dtype=torch.bfloat16, device="cuda")
    q, k, K = torch.zeros((2, 3, 8, 64), **z), torch.zeros((2, 3, 2, 64), **z), torch.zeros((2, 2, 9, 64), **z)
    pos, rows = (torch.zeros(s, dtype=torch.int32, device="cuda") for s in ((2, 3, 2), (2, 3)))
    axes = [0, 1] * 16
    good = dict(q=q, k=k, v=k, pos=pos, axes=axes, Kloc=K, Vloc=K.clone(), rows=rows)
    msa.msa_norm_rotate_axes(cfg, **good)
    for bad in (dict(axes=[0] * 31), dict(axes=[0, 4] * 16), dict(axes=[0.0] * 31 + [0.5]), dict(rows=rows[:1]), dict(rows=rows.long()),
                dict(pos=pos[..., 0]), dict(pos=pos[:, :2]), dict(pos=pos.long()), dict(Kloc=None), dict(q=q.transpose(0, 1))):
        with pytest.raises(ValueError):
            msa.msa_norm_rotate_axes(cfg, **{**good, **bad})
    with pytest.raises(msa.MsaError):
        msa.msa_norm_rotate_axes(cfg, **{**good, "axes": [0, 2] * 16})
