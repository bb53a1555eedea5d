"""msa_sparse_attend4 against the plain definition in 64 bits over what the packed bank stands for, alone and at the end of the
chain that leads to it."""
import ctypes
import itertools

import pytest
import torch

import paper_2603_23516_amd as msa
import plain64 as P

FEW, MANY = 2.0 ** -16, 2.0 ** -8


def _cfg(N=4, G=8, Hq=8, Hkv=2, d=64, **kw):
    return msa.MsaConfig(N, G, 1, Hq, Hkv, d, 1e4, bank_keys_rotated=1, **kw)


@pytest.fixture(scope="module")
def lib():
    return msa.load_library()


def _call(lib, cfg, **kw):
    p = ctypes.c_void_p(0x10000)
    a = dict(q=p, B=1, M=1, K4=p, K4s=p, V4=p, V4s=p, idx=p, k=2, Kl=p, Vl=p, L=64, pos0=0, q_pos=p, out=p, lse=p, ws=p,
             bytes=1 << 40)
    a.update(kw)
    return lib.msa_sparse_attend4(ctypes.byref(cfg), a["q"], a["B"], a["M"], a["K4"], a["K4s"], a["V4"], a["V4s"], a["idx"],
                                  a["k"], a["Kl"], a["Vl"], a["L"], a["pos0"], a["q_pos"], a["out"], a["lse"], a["ws"],
                                  a["bytes"], None)


@pytest.mark.parametrize("kw, status", [
    (dict(q=None), -1), (dict(K4=None), -1), (dict(K4s=None), -1), (dict(V4=None), -1), (dict(V4s=None), -1), (dict(idx=None), -1),
    (dict(Kl=None), -1), (dict(Vl=None), -1), (dict(q_pos=None), -1), (dict(out=None), -1), (dict(ws=None), -1), (dict(B=0), -1),
    (dict(M=0), -1), (dict(k=0), -1), (dict(L=-1), -1), (dict(pos0=-1), -1), (dict(k=65), -2), (dict(B=256, M=256), -2),
    (dict(L=(1 << 28) + 1), -2), (dict(bytes=255), -3), (dict(K4=ctypes.c_void_p(0x10008)), -4),
    (dict(V4s=ctypes.c_void_p(0x10008)), -4), (dict(idx=ctypes.c_void_p(0x10002)), -4), (dict(ws=ctypes.c_void_p(0x10008)), -4),
])
def test_refusals(lib, kw, status):
    assert _call(lib, _cfg(), **kw) == status


def test_refused_sizes(lib):
    assert _call(lib, msa.MsaConfig(4, 1 << 27, 1, 8, 2, 64, 1e4), k=4) == msa.MSA_ERR_UNSUPPORTED      # k G rows
    c = _cfg(2048, 512, 32, 8, 128)
    for B, M, k, L in ((1, 1, 1, 0), (8, 1, 32, 2048), (1, 64, 8, 64)):
        n = msa.sparse_attend4_workspace_bytes(c, B, M, k, L)
        assert n >= 256 and n % 256 == 0
        assert _call(lib, c, B=B, M=M, k=k, L=L, bytes=n - 1) == msa.MSA_ERR_WORKSPACE
    pooled = _cfg(2048, 512, 32, 8, 128, token_pool=1)
    assert msa.sparse_attend4_workspace_bytes(pooled, 1, 100, 16, 100) >= 8 * 16 * 512 * 128 * 4
    assert msa.sparse_attend4_workspace_bytes(c, 1, 1, 65, 0) == 0
    for cfg in (c, pooled, _cfg(2048, 1, 32, 8, 128, token_pool=1), _cfg(2048, 8, 8, 1, 64, token_pool=1)):
        for B, M in ((1, 1), (3, 5), (8, 31), (1, 32), (2, 500), (40, 16), (1, 9)):
            for k0, k1 in ((1, 64), (3, 3), (64, 64)):      # more documents, a longer local context: never less
                sizes = [msa.sparse_attend4_workspace_bytes(cfg, B, M, k, L)
                         for k, L in ((k0, 0), (k0, 10), (min(k0 + 1, k1), 600), (k1, 600), (k1, 4000), (k1, 50000))]
                assert sizes == sorted(sizes), (B, M, k0)


@pytest.mark.parametrize("G", [1, 3, 8, 20, 33, 512])
@pytest.mark.parametrize("Hq, Hkv, d", [(32, 8, 128), (8, 1, 64), (8, 8, 64)])
def test_more_documents_never_ask_for_less(G, Hq, Hkv, d):
    """Every k at a fixed local context, and lengths around the border between the two kernels at a fixed k: what serves the
    largest call serves the smaller ones."""
    cfg = _cfg(2048, G, Hq, Hkv, d, token_pool=1)
    for B, M in itertools.product((1, 3, 8, 64, 400), (1, 7, 8, 9, 16, 31, 32, 40)):
        for L in (0, 1, 100, 1111, 3328, 9000):
            sizes = [msa.sparse_attend4_workspace_bytes(cfg, B, M, k, L) for k in range(1, 65)]
            assert sizes == sorted(sizes), (B, M, L)
        for k in (1, 2, 31, 64):
            sizes = [msa.sparse_attend4_workspace_bytes(cfg, B, M, k, L) for L in range(0, 3600, 16)]
            assert sizes == sorted(sizes), (B, M, k)


def _make(N, G, Hq, Hkv, d, B, M, L, seed):
    g = torch.Generator().manual_seed(seed)
    shapes = ((N, Hkv, G, d), (N, Hkv, G, d), (B, M, Hq, d), (B, Hkv, L, d), (B, Hkv, L, d))
    return [torch.randn(s, generator=g).to(torch.bfloat16) for s in shapes], g


def _check(N, G, Hq, Hkv, d, B, M, k, L, scope, pool, lens, idx, q_pos, pos0, seed=0):
    (K, V, q, Kl, Vl), _ = _make(N, G, Hq, Hkv, d, B, M, L, seed)
    cfg = _cfg(N, G, Hq, Hkv, d, select_scope=scope, token_pool=pool, doc_lens=None if lens is None else lens.cuda())
    bank = msa.msa_pack_kv4(cfg.replace(doc_lens=None), K.cuda(), V.cuda())
    kept = [P.unpack4(bank[i].cpu(), bank[i + 1].cpu()) for i in (0, 2)]
    Kd, Vd = Kl.clone(), Vl.clone()
    for b in range(B):
        behind = max(0, int(q_pos[b].max()) - pos0 + 1)
        Kd[b, :, behind:] = float("nan")
        Vd[b, :, behind:] = float("inf")
    ws = torch.full((msa.sparse_attend4_workspace_bytes(cfg, B, M, k, L),), 0xA5, dtype=torch.uint8, device="cuda")
    out, lse = msa.msa_sparse_attend4(cfg, q.cuda(), bank, idx.cuda(), Kd.cuda() if L else None, Vd.cuda() if L else None, pos0,
                                      q_pos.cuda(), workspace=ws)
    torch.cuda.synchronize()
    ref = P.sparse_attend4(q.double(), *kept, idx, lens, Kl.double(), Vl.double(), q_pos, pos0)
    ref.check(out, lse, MANY if pool and M >= 8 else FEW)
    return out


@pytest.mark.gpu
@pytest.mark.parametrize("Hq, Hkv, d", [(4, 4, 64), (6, 2, 128), (8, 1, 64), (8, 2, 128)])
@pytest.mark.parametrize("G, k, L", [(1, 64, 0), (3, 5, 40), (8, 4, 33), (33, 7, 1), (64, 3, 100), (512, 2, 0)])
@pytest.mark.parametrize("M, scope, pool", [(1, 0, 0), (2, 1, 0), (3, 0, 1), (9, 0, 1), (40, 1, 1), (9, 0, 0)])
def test_against_64_bits(Hq, Hkv, d, G, k, L, M, scope, pool):
    if M == 40 and G * k > 250:
        G = 30
    B, N = 2, 70
    g = torch.Generator().manual_seed(G + M)
    shape = (B, 1 if pool else M, 1 if scope else Hkv, k)
    idx = torch.randint(-1, N, shape, generator=g, dtype=torch.int32)          # pads, documents twice
    idx[0, 0, 0, 0] = N                                                       # outside the bank
    idx[1, :, -1] = -1                                                        # no document at all
    lens = torch.randint(0, G + 3, (N,), generator=g, dtype=torch.int32) if G != 64 else None
    pos0 = G
    q_pos = (pos0 + L - M + torch.arange(M).expand(B, M) - torch.tensor([[0], [L // 3]])).to(torch.int32)
    q_pos[1, 0] = pos0 - 1                                                    # sees no local row: with no document nothing
    _check(N, G, Hq, Hkv, d, B, M, k, L, scope, pool, lens, idx, q_pos, pos0)


@pytest.mark.gpu
@pytest.mark.parametrize("M, pool", [(1, 0), (10, 1)])
def test_split_rows(M, pool):
    """Enough rows for several workgroups per head."""
    idx = torch.arange(12, dtype=torch.int32).flip(0).reshape(1, 1, 1, 12).contiguous()
    q_pos = (512 + 300 - M + torch.arange(M)).reshape(1, M).to(torch.int32)
    _check(12, 256, 4, 1, 128, 1, M, 12, 300, 0, pool, None, idx, q_pos, 512)


@pytest.mark.gpu
def test_same_as_the_bank_in_16_bits():
    """Where four bits hold the bank exactly, msa_sparse_attend over it in bf16 says the same (its tolerances: its weights are
    pairs too, the local context is left out since it would be turned)."""
    N, G, Hq, Hkv, d, k = 16, 32, 8, 2, 64, 4
    (K, V, q, _, _), g = _make(N, G, Hq, Hkv, d, 2, 1, 1, 3)
    cfg = _cfg(N, G, Hq, Hkv, d)
    bank = msa.msa_pack_kv4(cfg, K.cuda(), V.cuda())
    Kx, Vx = msa.msa_unpack_kv4(cfg, bank)
    idx = torch.randint(0, N, (2, 1, Hkv, k), generator=g, dtype=torch.int32).cuda()
    zero = torch.zeros((2, 1), dtype=torch.int32, device="cuda")           # position 0: msa_sparse_attend turns queries by nothing
    a, la = msa.msa_sparse_attend4(cfg, q.cuda(), bank, idx, None, None, 0, zero)
    b, lb = msa.msa_sparse_attend(cfg, q.cuda(), Kx, Vx, idx, None, None, 0, zero)
    assert float((a.float() - b.float()).abs().max()) <= 2.0 ** -6 and float((la - lb).abs().max()) <= 1e-3


@pytest.mark.gpu
def test_from_projections_to_both_attentions():
    """As a program runs it: documents and tokens from fused projections through msa_norm_rotate, the bank packed, then a local
    layer's window attention and a routed layer's attention, token by token; the plain chain rounds where the tensors do."""
    Hq, Hkv, d, N, G, base, T, k = 8, 2, 64, 10, 24, 1e4, 40, 3
    g = torch.Generator().manual_seed(12)
    w = [(1 + 0.2 * torch.randn(d, generator=g)).to(torch.bfloat16) for _ in range(2)]
    cfg = msa.MsaConfig(N, G, 1, Hq, Hkv, d, base, bank_keys_rotated=1)
    pdoc = torch.randn((N, G, (Hq + 2 * Hkv) * d), generator=g).to(torch.bfloat16)
    ptok = torch.randn((1, T, (Hq + 2 * Hkv) * d), generator=g).to(torch.bfloat16)

    def cut(x):
        x = x.unflatten(-1, (-1, d))
        return x[:, :, :Hq], x[:, :, Hq:Hq + Hkv], x[:, :, Hq + Hkv:]

    wd = [t.cuda() for t in w]
    K, V = (torch.zeros((N, Hkv, G, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    _, kd, vd = cut(pdoc.cuda())
    msa.msa_norm_rotate(cfg, None, kd, vd, torch.arange(G, dtype=torch.int32).expand(N, G).contiguous().cuda(), K, V, None, wd[1])
    bank = msa.msa_pack_kv4(cfg, K, V)
    Kl, Vl = (torch.full((1, Hkv, T, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    idx = torch.randint(0, N, (1, 1, Hkv, k), generator=g, dtype=torch.int32)
    got = []
    for t0, t1 in ((0, 30), (30, 31), (31, 32), (32, 40)):        # a prompt, single tokens, a chunk
        q, kk, vv = cut(ptok[:, t0:t1].cuda())
        pos = torch.arange(G + t0, G + t1, dtype=torch.int32).reshape(1, -1).cuda()
        qr = msa.msa_norm_rotate(cfg, q, kk, vv, pos, Kl, Vl, *wd, local_pos0=G)
        win, wl = msa.msa_window_attend(cfg, qr, Kl, Vl, pos, 16, sinks=2, local_pos0=G)
        c1 = cfg.replace(token_pool=1)
        mem, ml = msa.msa_sparse_attend4(c1, qr, bank, idx.cuda(), Kl, Vl, G, pos)
        got.append((qr, win, wl, mem, ml))
    torch.cuda.synchronize()
    qr, win, wl, mem, ml = (torch.cat(x, 1) for x in zip(*got))
    y = P.norm(ptok.double().unflatten(-1, (-1, d))[:, :, Hq:Hq + Hkv], w[1].double(), 1e-6)
    want = P.rotate(y, torch.arange(G, G + T)[None, :, None].expand(1, T, Hkv), base).transpose(1, 2)
    assert float((Kl.double().cpu() - want).abs().max()) <= 2.0 ** -7 * float(want.abs().max())
    kept = [P.unpack4(bank[i].cpu(), bank[i + 1].cpu()) for i in (0, 2)]
    pos = torch.arange(G, G + T).reshape(1, T)
    cache = [t.double().cpu() for t in (qr, Kl, Vl)]
    P.window_attend(*cache, pos, 16, 2, G).check(win, wl, MANY)
    P.sparse_attend4(cache[0], *kept, idx, None, cache[1], cache[2], pos, G).check(mem, ml, MANY)


@pytest.mark.gpu
@pytest.mark.parametrize("M, pool", [(1, 0), (9, 1)])
def test_graph_replays(M, pool):
    N, G, Hq, Hkv, d, k, L = 20, 128, 8, 1, 128, 8, 200
    (K, V, q, Kl, Vl), g = _make(N, G, Hq, Hkv, d, 1, M, L, 8)
    cfg = _cfg(N, G, Hq, Hkv, d, token_pool=pool)
    bank = msa.msa_pack_kv4(cfg, K.cuda(), V.cuda())
    q, Kl, Vl = q.cuda(), Kl.cuda(), Vl.cuda()
    idx = torch.randint(0, N, (1, 1, Hkv, k), generator=g, dtype=torch.int32).cuda()
    q_pos = torch.full((1, M), G + L - 1, dtype=torch.int32, device="cuda")
    ws = torch.full((msa.sparse_attend4_workspace_bytes(cfg, 1, M, k, L),), 0xFF, dtype=torch.uint8, device="cuda")
    out, lse = torch.empty_like(q), torch.empty((1, M, Hq), dtype=torch.float32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        msa.msa_sparse_attend4(cfg, q, bank, idx, Kl, Vl, G, q_pos, out=out, lse=lse, workspace=ws)
    for i in range(4):
        idx.copy_(torch.randint(-1, N, idx.shape, generator=g, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        o, y = msa.msa_sparse_attend4(cfg, q, bank, idx, Kl, Vl, G, q_pos)
        torch.cuda.synchronize()
        assert torch.equal(o, out) and torch.equal(y, lse), i


@pytest.mark.gpu
@pytest.mark.parametrize("M, pool", [(1, 0), (32, 1)])
def test_offsets_past_32_bits(M, pool):
    """A bank whose codes alone are 2.3 GB: its last documents are found."""
    N, G, Hq, Hkv, d, k = 9000, 512, 8, 8, 128, 3
    cfg = _cfg(N, G, Hq, Hkv, d, token_pool=pool)
    bank = tuple(torch.zeros_like(t) for t in msa.alloc_kv4(cfg))
    bank[1].fill_(127), bank[3].fill_(127)
    (K, V, q, Kl, Vl), _ = _make(4, G, Hq, Hkv, d, 1, M, 8, 11)
    small = msa.msa_pack_kv4(_cfg(4, G, Hq, Hkv, d), K.cuda(), V.cuda())
    for t, x in zip(bank, small):
        t[N - 4:] = x
    idx = torch.tensor([N - 1, N - 3, N - 4], dtype=torch.int32).reshape(1, 1, 1, k).expand(1, 1, Hkv, k).contiguous()
    q_pos = torch.full((1, M), G + 7, dtype=torch.int32)
    out, lse = msa.msa_sparse_attend4(cfg, q.cuda(), bank, idx.cuda(), Kl.cuda(), Vl.cuda(), G, q_pos.cuda())
    torch.cuda.synchronize()
    kept = [P.unpack4(small[i].cpu(), small[i + 1].cpu()) for i in (0, 2)]
    P.sparse_attend4(q.double(), *kept, idx - (N - 4), None, Kl.double(), Vl.double(), q_pos, G).check(out, lse, MANY)
    back = msa.msa_unpack_kv4(cfg, bank, N - 1, 1)
    assert torch.equal(back[0][N - 1].double().cpu(), kept[0][3]) and torch.equal(back[1][N - 1].double().cpu(), kept[1][3])


@pytest.mark.gpu
def test_python_refusals():
    N, G, Hq, Hkv, d, k = 4, 8, 8, 2, 64, 2
    (K, V, q, Kl, Vl), _ = _make(N, G, Hq, Hkv, d, 2, 3, 9, 0)
    cfg = _cfg(N, G, Hq, Hkv, d)
    bank = msa.msa_pack_kv4(cfg, K.cuda(), V.cuda())
    pos = torch.zeros((2, 3), dtype=torch.int32, device="cuda")
    idx = torch.zeros((2, 3, Hkv, k), dtype=torch.int32, device="cuda")
    good = dict(q=q.cuda(), bank=bank, idx=idx, Kloc=Kl.cuda(), Vloc=Vl.cuda(), local_pos0=G, q_pos=pos)
    msa.msa_sparse_attend4(cfg, **good)
    for bad in (dict(q=q), dict(idx=idx[:, :1]), dict(idx=idx[:, :, :1]), dict(idx=idx.long()), dict(bank=bank[::-1]),
                dict(bank=(None,) + bank[1:]), dict(Kloc=None), dict(q_pos=pos[:1]), dict(Vloc=Kl.cuda()[:, :, 1:]),
                dict(local_pos0=2 ** 32 + G)):
        with pytest.raises(ValueError):
            msa.msa_sparse_attend4(cfg, **{**good, **bad})


@pytest.mark.gpu
def test_a_question_of_more_than_65535_tokens():
    N, G, d, M = 6, 8, 64, 66001
    (K, V, q, Kl, Vl), _ = _make(N, G, 2, 1, d, 1, M, 20, 0)
    cfg = msa.MsaConfig(N, G, 1, 2, 1, d, 1e4, token_pool=1)
    bank = msa.msa_pack_kv4(cfg.replace(bank_keys_rotated=1), K.cuda(), V.cuda())
    idx = torch.tensor([4, -1, 2], dtype=torch.int32).reshape(1, 1, 1, 3)
    q_pos = (G + torch.arange(M, dtype=torch.int32) % 23).reshape(1, M)
    out, lse = msa.msa_sparse_attend4(cfg, q.cuda(), bank, idx.cuda(), Kl.cuda(), Vl.cuda(), G, q_pos.cuda())
    at = [0, 1, 40000, 65535, 65536, M - 1]
    kept = [P.unpack4(bank[i].cpu(), bank[i + 1].cpu()) for i in (0, 2)]
    P.sparse_attend4(q[:, at].double(), *kept, idx, None, Kl.double(), Vl.double(), q_pos[:, at], G).check(out[:, at], lse[:, at], MANY)


@pytest.mark.gpu
@pytest.mark.parametrize("what", ["norm", "window", "attend4", "pack", "unpack"])
def test_results_on_another_stream_take_no_memory_in_use(what):
    """What the current stream still has to read, though its tensors are gone, is not handed to a call on another stream."""
    N, G, Hq, Hkv, d, B, M = 16, 64, 8, 2, 64, 2, 64
    (K, V, q, Kl, Vl), _ = _make(N, G, Hq, Hkv, d, B, M, M, 21)
    K, V, q, Kl, Vl = (t.cuda() for t in (K, V, q, Kl, Vl))
    cfg = _cfg(N, G, Hq, Hkv, d)
    bank = msa.msa_pack_kv4(cfg, K, V)
    pos = torch.arange(M, dtype=torch.int32, device="cuda").repeat(B, 1)
    idx = torch.zeros((B, M, Hkv, 2), dtype=torch.int32, device="cuda")
    kt, vt = Kl.transpose(1, 2).contiguous(), Vl.transpose(1, 2).contiguous()
    Kn, Vn = torch.zeros_like(Kl), torch.zeros_like(Vl)
    calls = dict(norm=lambda s: msa.msa_norm_rotate(cfg, q, kt, vt, pos, Kn, Vn, stream=s),
                 window=lambda s: msa.msa_window_attend(cfg, q, Kl, Vl, pos, 20, stream=s),
                 attend4=lambda s: msa.msa_sparse_attend4(cfg, q, bank, idx, Kl, Vl, 0, pos, stream=s),
                 pack=lambda s: msa.msa_pack_kv4(cfg, K, V, stream=s), unpack=lambda s: msa.msa_unpack_kv4(cfg, bank, stream=s))
    want = calls[what](None)
    want = [want] if torch.is_tensor(want) else list(want)
    sizes = [t.numel() * t.element_size() for t in want]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        held = [torch.full((n,), 7, dtype=torch.uint8, device="cuda") for n in sizes]
        torch.cuda._sleep(20_000_000)
        kept = [t.clone() for t in held]
        del held
        got = calls[what](side)
        got = [got] if torch.is_tensor(got) else list(got)
        side.synchronize()
        torch.cuda.synchronize()
        assert all(bool((t == 7).all()) for t in kept)
        assert all(torch.equal(a, b) for a, b in zip(want, got))
