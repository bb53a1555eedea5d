"""msa_pack_kv4 and msa_unpack_kv4: exact against the plain definition in 64 bits."""
import ctypes

import pytest
import torch

import paper_2603_23516_amd as msa
import plain64 as P


@pytest.fixture(scope="module")
def lib():
    return msa.load_library()


def _cfg(N=3, G=5, Hkv=2, d=64, rotated=1, lens=None):
    return msa.MsaConfig(N, G, 1, Hkv, Hkv, d, 1e4, bank_keys_rotated=rotated, doc_lens=lens)


@pytest.mark.parametrize("ptrs, begin, count, status", [
    ((0, 0, 0, 0, 0, 0), 0, 3, -1), ((1, 1, 0, 1, 1, 1), 0, 3, -1), ((0, 1, 1, 1, 1, 1), 0, 3, -1), ((1, 0, 1, 1, 0, 1), 0, 3, -1),
    ((1, 1, 1, 1, 1, 1), -1, 1, -1), ((1, 1, 1, 1, 1, 1), 0, -1, -1), ((1, 1, 1, 1, 1, 1), 2, 2, -1),
    ((2, 1, 1, 1, 1, 1), 0, 3, -4), ((1, 1, 2, 1, 1, 1), 0, 3, -4), ((1, 1, 1, 2, 1, 1), 0, 3, -4),
])
def test_refusals(lib, ptrs, begin, count, status):
    K, V, K4, K4s, V4, V4s = (ctypes.c_void_p({0: None, 1: 0x10000, 2: 0x10004}[p]) for p in ptrs)
    assert lib.msa_pack_kv4(ctypes.byref(_cfg()), K, V, begin, count, K4, K4s, V4, V4s, None) == status
    if ptrs not in ((0, 1, 1, 1, 1, 1), (1, 0, 1, 1, 0, 1)):       # unpacking one half beside codes that are not asked for is fine
        assert lib.msa_unpack_kv4(ctypes.byref(_cfg()), K4, K4s, V4, V4s, begin, count, K, V, None) == status
    assert lib.msa_pack_kv4(None, K, V, 0, 1, K4, K4s, V4, V4s, None) == -1


def _edges():
    """A block for every border: each code's value, the middle between two, and their neighbours in bf16, at several scales."""
    v = []
    for c in (0.25, 0.5, 0.75, 1.0, 1.25, 1.5, 1.75, 2.0, 2.5, 3.0, 3.5, 4.0, 5.0, 6.0):
        step = 2.0 ** -7 * 2.0 ** torch.log2(torch.tensor(c)).floor().item()
        v += [c - step, c, c + step]
    v = torch.tensor(v, dtype=torch.float64)
    rows = []
    for top in (6.0, 7.0, 7.03125, 3.515625, 4.0):          # the largest value decides the scale
        for e in (-126, -120, -3, 0, 5, 120):
            for part in v.split(15):
                b = torch.zeros(32, dtype=torch.float64)
                b[:len(part)], b[15:15 + len(part)], b[31] = part, -part, top
                rows.append(b * 2.0 ** e)
    rows.append(torch.zeros(32, dtype=torch.float64))
    rows.append(torch.full((32,), 3.3895313892515355e38, dtype=torch.float64))      # the largest bf16: saturates
    rows.append(torch.full((32,), 2.0 ** -133, dtype=torch.float64))                # the smallest
    rows.append(torch.full((32,), 2.0 ** -126, dtype=torch.float64))
    return torch.stack(rows).to(torch.bfloat16)


def _check(cfg, K, V, lens):
    bank = msa.msa_pack_kv4(cfg, K.cuda(), V.cuda())
    back = msa.msa_unpack_kv4(cfg, bank)
    torch.cuda.synchronize()
    for x, codes, scales, y in ((K, bank[0], bank[1], back[0]), (V, bank[2], bank[3], back[1])):
        x = x.double().clone()
        if lens is not None:
            for n in range(x.shape[0]):
                x[n, :, min(max(int(lens[n]), 1), x.shape[2]):] = 0
        want, e = P.pack4(x)
        assert torch.equal(scales.cpu(), e)
        assert torch.equal(y.double().cpu(), want)
        assert torch.equal(P.unpack4(codes.cpu(), scales.cpu()), want)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
def test_borders(d):
    rows = _edges()
    n = (rows.shape[0] * 32 + d - 1) // d
    flat = torch.zeros(n * d, dtype=torch.bfloat16)
    flat[:rows.numel()] = rows.flatten()
    K = flat.reshape(n, 1, 1, d)
    _check(_cfg(n, 1, 1, d), K, -K.flip(0), None)


@pytest.mark.gpu
@pytest.mark.parametrize("N, Hkv, G, d, ragged", [(1, 1, 1, 64, False), (3, 2, 5, 64, True), (7, 3, 33, 128, True),
                                                  (2, 8, 512, 128, False), (50, 2, 8, 64, True)])
def test_random(N, Hkv, G, d, ragged):
    g = torch.Generator().manual_seed(N)
    K = (torch.randn((N, Hkv, G, d), generator=g) * torch.exp(2 * torch.randn((1, 1, 1, d), generator=g))).to(torch.bfloat16)
    V = torch.randn((N, Hkv, G, d), generator=g).to(torch.bfloat16)
    lens = torch.randint(0, G + 2, (N,), generator=g, dtype=torch.int32) if ragged else None
    if ragged:                                       # what lies behind a document's end is not read
        for n in range(N):
            K[n, :, min(max(int(lens[n]), 1), G):] = float("nan")
            V[n, :, min(max(int(lens[n]), 1), G):] = float("inf")
    _check(_cfg(N, G, Hkv, d, lens=None if lens is None else lens.cuda()), K, V, lens)


@pytest.mark.gpu
def test_pieces_and_halves():
    """A bank packed in pieces, keys and values apart, equals the bank packed at once; other documents stay as they were."""
    g = torch.Generator().manual_seed(9)
    K, V = (torch.randn((5, 2, 7, 64), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    cfg = _cfg(5, 7)
    whole = msa.msa_pack_kv4(cfg, K, V)
    bank = tuple(torch.full_like(t, 0xA5) for t in whole)
    msa.msa_pack_kv4(cfg, K, None, 1, 2, bank)
    assert all(torch.equal(bank[i][1:3], whole[i][1:3]) for i in (0, 1))
    assert all(bool((bank[i][j] == 0xA5).all()) for i in (0, 1) for j in (0, 3, 4))
    assert all(bool((bank[i] == 0xA5).all()) for i in (2, 3))
    msa.msa_pack_kv4(cfg, None, V, 0, 5, bank)
    msa.msa_pack_kv4(cfg, K, None, 0, 1, bank)
    msa.msa_pack_kv4(cfg, K, None, 3, 2, bank)
    msa.msa_pack_kv4(cfg, K, V, 5, 0, bank)          # no documents
    for begin, count in ((2 ** 32, None), (0, 2 ** 32), (2 ** 32, 0)):
        with pytest.raises(ValueError):
            msa.msa_pack_kv4(cfg, K, V, begin, count, bank)
        with pytest.raises(ValueError):
            msa.msa_unpack_kv4(cfg, bank, begin, count)
    assert all(torch.equal(a, b) for a, b in zip(bank, whole))
    out = torch.full_like(K, 5.0)
    got, none = msa.msa_unpack_kv4(cfg, (whole[0], whole[1], None, None), 4, 1, K=out)
    assert none is None and bool((out[:4] == 5.0).all()) and torch.equal(out[4], msa.msa_unpack_kv4(cfg, whole)[0][4])


@pytest.mark.gpu
@pytest.mark.parametrize("d, G", [(64, 37), (128, 64)])
def test_keys_turned_by_their_positions(d, G):
    """Without bank_keys_rotated the keys go in turned: at most a step from the exact one where a rounding is close."""
    g = torch.Generator().manual_seed(d)
    K = torch.randn((3, 2, G, d), generator=g).to(torch.bfloat16)
    cfg = _cfg(3, G, 2, d, rotated=0)
    K4, K4s, _, _ = msa.msa_pack_kv4(cfg, K.cuda(), None)
    turned = P.rotate(K.double(), torch.arange(G), 1e4)
    want, e = P.pack4(turned)
    got = P.unpack4(K4.cpu(), K4s.cpu())
    assert torch.equal(K4s.cpu(), e)                 # (no block's maximum of these lies within 2^-20 of a border)
    s = torch.exp2(e.double() - 127).repeat_interleave(32, -1)
    y = (turned / s).abs().clamp(max=6.0)
    mid = (P.CODES[1:] + P.CODES[:-1]) / 2
    close = ((y[..., None] - mid).abs() < 2.0 ** -18).any(-1)     # fp32 rotation: under 2^-20 of the pair's size, 14 at most
    assert torch.equal(got[~close], want[~close])
    assert float(close.double().mean()) < 1e-3
    y0 = y * s
    assert bool(((got.abs() - y0).abs()[close] <= s[close] * (1 + 2.0 ** -10)).all())


@pytest.mark.gpu
@pytest.mark.parametrize("N, G, d, lens", [(130000, 1, 64, False), (131200, 1, 64, True), (2100, 63, 64, False), (2200, 512, 128, True)])
def test_many_rows_are_packed_as_few(N, G, d, lens):
    """Large banks take other loads: a document anywhere in them has the bits it gets alone."""
    g = torch.Generator(device="cuda").manual_seed(N)
    K = torch.randn((N, 1, G, d), generator=g, device="cuda", dtype=torch.bfloat16)
    V = torch.randn((N, 1, G, d), generator=g, device="cuda", dtype=torch.bfloat16)
    n = torch.randint(1, G + 1, (N,), generator=g, device="cuda", dtype=torch.int32) if lens else None
    cfg = _cfg(N, G, 1, d, lens=n)
    bank = msa.msa_pack_kv4(cfg, K, V)
    back = msa.msa_unpack_kv4(cfg, bank)
    for i in (0, 1, N // 3, N - 2, N - 1):
        one = _cfg(1, G, 1, d, lens=None if n is None else n[i:i + 1].contiguous())
        alone = msa.msa_pack_kv4(one, K[i:i + 1], V[i:i + 1])
        assert all(torch.equal(a[i:i + 1], b) for a, b in zip(bank, alone)), i
        assert all(torch.equal(a[i:i + 1], b) for a, b in zip(back, msa.msa_unpack_kv4(one, alone))), i


@pytest.mark.gpu
@pytest.mark.parametrize("N, Hkv, G, d", [(70, 3, 700, 64), (131, 1, 1001, 128), (2, 1, 66000, 64), (23000, 3, 2, 128), (140001, 1, 1, 64)])
def test_many_turned_keys_are_packed_as_few(N, Hkv, G, d):
    """The angles of a position are shared by several documents and heads: each has the bits it gets alone, the last ones too."""
    g = torch.Generator(device="cuda").manual_seed(N)
    K = torch.randn((N, Hkv, G, d), generator=g, device="cuda", dtype=torch.bfloat16)
    n = torch.randint(1, G + 1, (N,), generator=g, device="cuda", dtype=torch.int32)
    K4, K4s, _, _ = msa.msa_pack_kv4(_cfg(N, G, Hkv, d, rotated=0, lens=n), K, None)
    for i in (0, 1, N // 2, N - 2, N - 1):
        a4, a4s, _, _ = msa.msa_pack_kv4(_cfg(1, G, Hkv, d, rotated=0, lens=n[i:i + 1].contiguous()), K[i:i + 1], None)
        assert torch.equal(K4[i:i + 1], a4) and torch.equal(K4s[i:i + 1], a4s), i


@pytest.mark.gpu
@pytest.mark.parametrize("rotated, d, N, lens", [(1, 128, 4001, False), (0, 128, 3900, True), (1, 64, 7999, True), (0, 64, 7801, False)])
def test_codes_past_the_caches_are_packed_as_few(rotated, d, N, lens):
    """More than 256 MiB of codes are stored in another way: a document has the bits it gets alone, the last one too."""
    G = 512
    assert 2 * N * G * (d // 2 + d // 32) >= 256 << 20
    g = torch.Generator(device="cuda").manual_seed(N)
    K, V = (torch.randn((N, 1, G, d), generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    n = torch.randint(1, G + 1, (N,), generator=g, device="cuda", dtype=torch.int32) if lens else None
    bank = msa.msa_pack_kv4(_cfg(N, G, 1, d, rotated, n), K, V)
    for i in (0, 1, 2, 3, N // 3, N // 2, N - 2, N - 1):
        alone = msa.msa_pack_kv4(_cfg(1, G, 1, d, rotated, None if n is None else n[i:i + 1].contiguous()), K[i:i + 1], V[i:i + 1])
        assert all(torch.equal(a[i:i + 1], b) for a, b in zip(bank, alone)), i
    del bank, K, V
    torch.cuda.empty_cache()
