"""msa_norm_rotate against the plain definition in 64 bits, its refusals, and the rows it leaves alone."""
import ctypes

import pytest
import torch

import paper_2603_23516_amd as msa
import plain64 as P

HALF_BF16 = torch.finfo(torch.bfloat16).eps / 2


def _cfg(Hq=8, Hkv=2, d=64, base=1e4):
    return msa.MsaConfig(1, 1, 1, Hq, Hkv, d, base)


@pytest.fixture(scope="module")
def lib():
    return msa.load_library()


def _call(lib, cfg, **kw):
    p = ctypes.c_void_p(0x10000)
    a = dict(q=p, qs=512, k=p, ks=128, v=p, vs=128, qw=p, kw=p, eps=1e-6, rotate=1, pos=p, B=1, M=1, q_out=p, Kloc=p, Vloc=p,
             Lloc=4, pos0=0)
    a.update(kw)
    return lib.msa_norm_rotate(ctypes.byref(cfg), a["q"], a["qs"], a["k"], a["ks"], a["v"], a["vs"], a["qw"], a["kw"], a["eps"],
                               a["rotate"], a["pos"], a["B"], a["M"], a["q_out"], a["Kloc"], a["Vloc"], a["Lloc"], a["pos0"], None)


@pytest.mark.parametrize("kw, status", [
    (dict(pos=None), -1), (dict(q=None), -1), (dict(q_out=None), -1), (dict(Kloc=None), -1), (dict(v=None), -1),
    (dict(q=None, q_out=None, k=None, Kloc=None, v=None, Vloc=None), -1), (dict(B=0), -1), (dict(M=0), -1), (dict(Lloc=-1), -1),
    (dict(pos0=-1), -1), (dict(rotate=2), -1), (dict(eps=0.0), -1), (dict(eps=float("nan")), -1), (dict(eps=float("inf")), -1),
    (dict(qs=504), -1), (dict(ks=120), -1), (dict(vs=120), -1), (dict(B=1 << 20, M=1 << 10), -2),
    (dict(pos0=2 ** 31 - 1, Lloc=1), -2), (dict(qs=516), -4), (dict(ks=132), -4), (dict(q=ctypes.c_void_p(0x10002)), -4),
    (dict(qw=ctypes.c_void_p(0x10008)), -4), (dict(Vloc=ctypes.c_void_p(0x10008)), -4), (dict(pos=ctypes.c_void_p(0x10002)), -4),
])
def test_refusals(lib, kw, status):
    assert _call(lib, _cfg(), **kw) == status


def test_refused_configs(lib):
    assert _call(lib, _cfg(d=96)) == msa.MSA_ERR_UNSUPPORTED
    assert _call(lib, _cfg(Hq=7)) == msa.MSA_ERR_INVALID_ARG
    assert _call(lib, _cfg(base=0.5)) == msa.MSA_ERR_INVALID_ARG


def _run(B, M, Hq, Hkv, d, base, weights, rotate, pos, pos0, L, fused=True, seed=0):
    g = torch.Generator().manual_seed(seed)
    qkv = (torch.randn((B, M, (Hq + 2 * Hkv) * d), generator=g) * 3).to(torch.bfloat16)
    qw, kw = [(1 + 0.3 * torch.randn(d, generator=g)).to(torch.bfloat16) if weights else None for _ in range(2)]
    old = [torch.randn(s, generator=g).to(torch.bfloat16) for s in ((B, M, Hq, d), (B, Hkv, L, d), (B, Hkv, L, d))]
    dev = [t.cuda() for t in old]
    x = qkv.cuda()
    parts = [x[..., a * d:b * d].unflatten(-1, (b - a, d)) for a, b in ((0, Hq), (Hq, Hq + Hkv), (Hq + Hkv, Hq + 2 * Hkv))]
    if not fused:
        parts = [t.contiguous() for t in parts]
    out = msa.msa_norm_rotate(_cfg(Hq, Hkv, d, base), *parts, pos.cuda(), dev[1], dev[2], None if qw is None else qw.cuda(),
                              None if kw is None else kw.cuda(), eps=1e-6, rotate=rotate, local_pos0=pos0, q_out=dev[0])
    torch.cuda.synchronize()
    assert out.data_ptr() == dev[0].data_ptr()
    want, size = [t.double() for t in old], [torch.zeros(t.shape, dtype=torch.float64) for t in old]
    y = qkv.double().unflatten(-1, (-1, d))
    yq = P.norm(y[:, :, :Hq], None if qw is None else qw.double(), 1e-6)
    yk = P.norm(y[:, :, Hq:Hq + Hkv], None if kw is None else kw.double(), 1e-6)
    for b in range(B):
        for m in range(M):
            p = int(pos[b, m])
            if p < 0:
                continue
            at = torch.tensor(p if rotate else 0)
            pair = [z[b, m].abs() + z[b, m].abs().roll(d // 2, -1) for z in (yq, yk)]
            want[0][b, m], size[0][b, m] = P.rotate(yq[b, m], at, base), pair[0]
            if 0 <= p - pos0 < L:
                want[1][b, :, p - pos0], size[1][b, :, p - pos0] = P.rotate(yk[b, m], at, base), pair[1]
                want[2][b, :, p - pos0] = y[b, m, Hq + Hkv:]
    for i, (got, w, s) in enumerate(zip(dev, want, size)):
        got = got.double().cpu()
        # one rounding to bf16, and in fp32 at most 32 roundings of the pair's magnitude (squares, root, angles, turn); what
        # was not written and the values (size 0) are equal to the bit
        tol = torch.where(s > 0, HALF_BF16 * w.abs() + 32 * 2.0 ** -24 * s, torch.zeros_like(s))
        assert bool(((got - w).abs() <= tol).all()), (i, float(((got - w).abs() - tol).max()))


@pytest.mark.gpu
@pytest.mark.parametrize("B, M, Hq, Hkv, d, weights, rotate, pos0", [
    (1, 1, 32, 8, 128, True, True, 0), (1, 1, 1, 1, 64, True, True, 0), (3, 5, 8, 2, 64, True, True, 7),
    (2, 33, 24, 8, 64, False, True, 0), (1, 3, 9, 3, 128, True, True, 100), (5, 1, 17, 17, 64, True, False, 0),
    (2, 7, 40, 5, 128, True, True, 3), (1, 65, 8, 8, 128, False, True, 1000000),
])
@pytest.mark.parametrize("fused", [True, False])
def test_against_64_bits(B, M, Hq, Hkv, d, weights, rotate, pos0, fused):
    L = M + 3
    pos = pos0 - 1 + torch.arange(M).expand(B, M) + torch.arange(B)[:, None]   # the first in front of the cache, some padding
    pos = torch.where((torch.arange(B * M).reshape(B, M) % 5) == 3, -1 - pos, pos).to(torch.int32)
    _run(B, M, Hq, Hkv, d, 1e4, weights, rotate, pos, pos0, L, fused)


@pytest.mark.gpu
def test_far_positions():
    """Angles of positions up to the largest: the range is reduced in double."""
    pos = torch.tensor([[0, 1, 2 ** 20 + 1, 2 ** 24 - 1, 2 ** 30 + 7, 2 ** 31 - 2]], dtype=torch.int32)
    for d in (64, 128):
        _run(1, 6, 4, 2, d, 1e6, True, True, pos, 2 ** 31 - 4, 3)


@pytest.mark.gpu
def test_many_tokens_take_one_wave_each():
    B, M = 2, 2500
    pos = torch.arange(M, dtype=torch.int32).expand(B, M).contiguous()
    g = torch.Generator().manual_seed(3)
    x = torch.randn((B, M, 12, 64), generator=g).to(torch.bfloat16).cuda()
    cfg = _cfg()
    K, V = (torch.zeros((B, 2, M, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = msa.msa_norm_rotate(cfg, x[:, :, :8], x[:, :, 8:10], x[:, :, 10:], pos.cuda(), K, V)
    for m0 in (0, 1, 1234, 2499):      # the same tokens one at a time: the same bits
        K1, V1 = (torch.zeros((B, 2, 1, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        xm = x[:, m0:m0 + 1].contiguous()
        q1 = msa.msa_norm_rotate(cfg, xm[:, :, :8], xm[:, :, 8:10], xm[:, :, 10:], pos[:, m0:m0 + 1].cuda().contiguous(), K1, V1,
                                 local_pos0=m0)
        assert torch.equal(q[:, m0:m0 + 1], q1) and torch.equal(K[:, :, m0:m0 + 1], K1) and torch.equal(V[:, :, m0:m0 + 1], V1)


@pytest.mark.gpu
def test_parts_alone_and_zero_rows():
    """Queries alone, keys alone, values alone; a head of zeros stays zero."""
    cfg = _cfg()
    g = torch.Generator().manual_seed(1)
    q = torch.randn((2, 3, 8, 64), generator=g).to(torch.bfloat16).cuda()
    q[0, 0, 0] = 0
    k = torch.randn((2, 3, 2, 64), generator=g).to(torch.bfloat16).cuda()
    pos = torch.arange(3, dtype=torch.int32).expand(2, 3).contiguous().cuda()
    w = torch.ones(64, dtype=torch.bfloat16, device="cuda")
    K, V = (torch.zeros((2, 2, 3, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    both = msa.msa_norm_rotate(cfg, q, k, k, pos, K, V, w, w)
    alone = msa.msa_norm_rotate(cfg, q, None, None, pos, None, None, w, w)
    assert torch.equal(both, alone) and float(both[0, 0, 0].abs().max()) == 0.0
    K1, V1 = torch.zeros_like(K), torch.zeros_like(V)
    assert msa.msa_norm_rotate(cfg, None, k, None, pos, K1, None, None, w) is None
    assert msa.msa_norm_rotate(cfg, None, None, k, pos, None, V1) is None
    assert torch.equal(K, K1) and torch.equal(V, V1)


@pytest.mark.gpu
def test_python_refusals():
    cfg = _cfg()
    q = torch.zeros((2, 3, 8, 64), dtype=torch.bfloat16, device="cuda")
    pos = torch.zeros((2, 3), dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        msa.msa_norm_rotate(cfg, q.transpose(0, 1), None, None, pos, None, None)     # tokens not the same distance apart
    with pytest.raises(ValueError):
        msa.msa_norm_rotate(cfg, q, None, None, pos.cpu(), None, None)
    with pytest.raises(ValueError):
        msa.msa_norm_rotate(cfg, q, None, None, pos[:1], None, None)
    with pytest.raises(ValueError):
        msa.msa_norm_rotate(cfg, q[..., ::2], None, None, pos, None, None)
    with pytest.raises(ValueError):
        msa.msa_norm_rotate(cfg, q, q[:, :, :2], None, pos, None, None)              # keys without their cache


@pytest.mark.gpu
def test_a_long_prompt_is_read_with_streaming_loads():
    """A projection of more than 128 MiB takes other loads: the bits are those of its tokens alone."""
    M, Hq, Hkv, d = 20000, 16, 8, 128
    cfg = _cfg(Hq, Hkv, d)
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn((1, M, Hq + 2 * Hkv, d), generator=g, device="cuda", dtype=torch.bfloat16)
    w = torch.randn(d, generator=g, device="cuda", dtype=torch.bfloat16)
    pos = torch.arange(M, dtype=torch.int32, device="cuda").reshape(1, M)
    K, V = (torch.zeros((1, Hkv, M, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = msa.msa_norm_rotate(cfg, x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:], pos, K, V, w, w)
    for m0 in (0, 7777, M - 5):
        K1, V1 = (torch.zeros((1, Hkv, 5, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        y = x[:, m0:m0 + 5]
        q1 = msa.msa_norm_rotate(cfg, y[:, :, :Hq], y[:, :, Hq:Hq + Hkv], y[:, :, Hq + Hkv:], pos[:, m0:m0 + 5].contiguous(), K1, V1, w, w,
                                 local_pos0=m0)
        assert torch.equal(q[:, m0:m0 + 5], q1) and torch.equal(K[:, :, m0:m0 + 5], K1) and torch.equal(V[:, :, m0:m0 + 5], V1)


@pytest.mark.parametrize("Kloc, Vloc", [((2, 64), (1, 2, 4, 64)), ((1, 2, 4, 64), (4, 64)), ((64,), None), (None, (8, 64)), ((1, 1, 2, 4, 64), None)])
def test_caches_of_other_ranks(Kloc, Vloc):
    """Refused like a cache of another shape, before anything else is read of them."""
    cfg = _cfg()
    kv = torch.zeros((1, 1, 2, 64), dtype=torch.bfloat16)
    K, V = (None if s is None else torch.zeros(s, dtype=torch.bfloat16) for s in (Kloc, Vloc))
    with pytest.raises(ValueError, match="Kloc and Vloc"):
        msa.msa_norm_rotate(cfg, None, None if K is None else kv, None if V is None else kv, torch.zeros((1, 1), dtype=torch.int32), K, V)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("top", [2.0 ** 58, 2.0 ** 61, 1e30, 3.38e38])
@pytest.mark.parametrize("eps", [1e-6, 1e38])
def test_squares_past_fp32(d, top, eps):
    """Finite elements whose squares fp32 does not hold, all of a head or one of it, beside heads of ordinary size.  The bound: one
    rounding to bf16, and in fp32 at most 32 roundings of the pair's magnitude; nothing here underflows (2^-80 at least)."""
    B, M, Hq, Hkv = 1, 5, 8, 2
    g = torch.Generator().manual_seed(d)
    x = torch.randn((B, M, Hq + 2 * Hkv, d), generator=g).clamp(-4, 4)
    x = torch.where(x.abs() < 0.01, 0.01, x)
    x[:, ::2, :, :] *= top / 4
    x[:, 1] *= top * 2.0 ** -40
    x[:, 1, :, d // 3] = -top
    x[:, 3, ::2] *= top / 4
    x = x.to(torch.bfloat16)
    assert bool(x.isfinite().all())
    w = [(1 + 0.2 * torch.randn(d, generator=g)).to(torch.bfloat16) for _ in range(2)]
    pos = torch.arange(M, dtype=torch.int32).reshape(B, M)
    K, V = (torch.zeros((B, Hkv, M, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    xd = x.cuda()
    q = msa.msa_norm_rotate(_cfg(Hq, Hkv, d), xd[:, :, :Hq], xd[:, :, Hq:Hq + Hkv], xd[:, :, Hq + Hkv:], pos.cuda(), K, V,
                            w[0].cuda(), w[1].cuda(), eps=eps)
    eps = float(torch.tensor(eps, dtype=torch.float32))
    for got, src, wt in ((q, x[:, :, :Hq], w[0]), (K.transpose(1, 2), x[:, :, Hq:Hq + Hkv], w[1])):
        y = P.norm(src.double(), wt.double(), eps)
        want, size = P.rotate(y, pos[:, :, None].expand(y.shape[:-1]), 1e4), y.abs() + y.abs().roll(d // 2, -1)
        err = (got.double().cpu() - want).abs() - (HALF_BF16 * want.abs() + 32 * 2.0 ** -24 * size)
        assert float(err.max()) <= 0, float(err.max())
