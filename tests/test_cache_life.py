"""A local cache as it is served from: a prompt with an image written, attended, weighed and cut, then token after token behind a
shared prefix in a captured step, weighed and cut again.  Against the same steps by the plain definitions in 64 bits."""
import math

import pytest
import torch

import paper_2603_23516_amd as msa
import plain64 as P
import plain64_cache as C

B, Hq, Hkv, d, A = 2, 8, 2, 64, 3
PRE, PROMPT, KEEP, CAP = 60, 40, 24, 48
AXES = [u * A // (d // 2) for u in range(d // 2)]


def _tokens(g, M):
    return torch.randn((B, M, (Hq + 2 * Hkv) * d), generator=g).to(torch.bfloat16)


def _split(x):
    return (x[..., :Hq * d].unflatten(-1, (Hq, d)), x[..., Hq * d:(Hq + Hkv) * d].unflatten(-1, (Hkv, d)),
            x[..., (Hq + Hkv) * d:].unflatten(-1, (Hkv, d)))


def _near_bf16(got, want):
    assert bool(((got.double().cpu() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -18).all())


@pytest.mark.gpu
def test_prompt_then_tokens():
    g = torch.Generator().manual_seed(11)
    cfg = msa.MsaConfig(1, 1, 1, Hq, Hkv, d, 1e4)
    dev = dict(device="cuda")
    Kp, Vp = (torch.randn((Hkv, PRE, d), generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    K, V = (torch.zeros((B, Hkv, CAP, d), dtype=torch.bfloat16, **dev) for _ in range(2))
    mass = torch.zeros((B, Hkv, CAP), **dev)
    lens = torch.tensor([PROMPT, PROMPT - 11], dtype=torch.int32)

    # the prompt: text, then an image of 4 x 4 patches at one time, then text; the second sequence is shorter, its end padding
    t = PRE + torch.arange(PROMPT)
    image = (torch.arange(PROMPT) >= 10) & (torch.arange(PROMPT) < 26)
    i = torch.arange(PROMPT) - 10
    pos = torch.stack([torch.where(image, PRE + 10, t), torch.where(image, PRE + 10 + i // 4, t), torch.where(image, PRE + 10 + i % 4, t)], -1)
    pos = pos.expand(B, PROMPT, A).contiguous().to(torch.int32)
    rows = torch.arange(PROMPT, dtype=torch.int32).expand(B, PROMPT).contiguous()
    there = torch.arange(PROMPT) < lens[:, None]
    pos[~there] = -1
    q_row = torch.where(there, rows, -1).to(torch.int32)
    x = _tokens(g, PROMPT)
    q, k, v = _split(x.cuda())
    q_out = torch.zeros((B, PROMPT, Hq, d), dtype=torch.bfloat16, **dev)
    msa.msa_norm_rotate_axes(cfg, q, k, v, pos.cuda(), AXES, K, V, rows=rows.cuda(), q_out=q_out)
    q64, k64, v64 = (y.double() for y in _split(x))
    qw, kw = C.rotate_axes(q64, pos, AXES, 1e4), C.rotate_axes(k64, pos, AXES, 1e4)
    torch.cuda.synchronize()
    for b in range(B):
        n = int(lens[b])
        _near_bf16(q_out[b, :n], qw[b, :n])
        _near_bf16(K[b, :, :n], kw[b, :n].transpose(0, 1))
        assert torch.equal(V[b, :, :n].cpu().double(), v64[b, :n].transpose(0, 1))
    out, lse = msa.msa_prefix_attend(cfg, q_out, Kp, Vp, K, V, (q_row + PRE).cuda(), local_pos0=PRE)
    lse = torch.where(there[..., None].cuda(), lse, -math.inf)       # the padding sees the prefix: it weighs nothing in the cache
    msa.msa_attend_mass(cfg, q_out, K, lse, (q_row + PRE).cuda(), CAP, local_pos0=PRE, mass=mass, decay=0.0, out=mass)
    torch.cuda.synchronize()
    want = C.prefix_attend(q_out.double().cpu(), Kp.double().cpu(), Vp.double().cpu(), None, K.double().cpu(), V.double().cpu(),
                           q_row + PRE, PRE)
    want.check(out, torch.where(there[..., None].cuda(), lse, want.lse.float().cuda()))
    wm, tol = C.attend_mass(q_out.double().cpu(), K.double().cpu(), lse.double().cpu(), q_row, CAP, 0, 0, None, 1.0)
    assert bool(((mass.double().cpu() - wm).abs() <= tol).all())

    def cut():
        nonlocal lens
        held = [y.clone().cpu() for y in (K, V, mass)]
        kept = msa.msa_evict(cfg, K, V, mass, lens.cuda(), KEEP, sinks=2, recent=6)[3].cpu()
        torch.cuda.synchronize()
        for b in range(B):
            for h in range(Hkv):
                at = C.evict_rows(held[2][b, h], int(lens[b]), KEEP, 2, 6)
                assert kept[b, h, :len(at)].tolist() == at
                for y, z in zip((K, V, mass), held):
                    assert torch.equal(y[b, h, :len(at)].cpu(), z[b, h, at])
        lens = lens.clamp(max=KEEP)

    cut()
    assert lens.tolist() == [KEEP, KEEP]
    lens = torch.tensor([KEEP, KEEP - 3], dtype=torch.int32)         # (the second gave its last rows up: another length)

    # token after token, the step captured once: rows and positions are what changes
    x1 = torch.zeros((B, 1, (Hq + 2 * Hkv) * d), dtype=torch.bfloat16, **dev)
    pos1, row1 = torch.zeros((B, 1, A), dtype=torch.int32, **dev), torch.zeros((B, 1), dtype=torch.int32, **dev)
    q1 = torch.zeros((B, 1, Hq, d), dtype=torch.bfloat16, **dev)
    o1, y1 = torch.zeros_like(q1), torch.zeros((B, 1, Hq), **dev)
    ws = [torch.empty(max(n, 256), dtype=torch.uint8, **dev) for n in (msa.prefix_attend_workspace_bytes(cfg, B, 1, PRE, CAP),
                                                                       msa.attend_mass_workspace_bytes(cfg, B, 1, CAP, CAP))]

    def step():
        q, k, v = _split(x1)
        msa.msa_norm_rotate_axes(cfg, q, k, v, pos1, AXES, K, V, rows=row1, q_out=q1)
        msa.msa_prefix_attend(cfg, q1, Kp, Vp, K, V, row1, out=o1, lse=y1, workspace=ws[0])
        msa.msa_attend_mass(cfg, q1, K, y1, row1, CAP, mass=mass, decay=0.95, out=mass, workspace=ws[1])

    mass[1, :, KEEP - 3:] = 0.0
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for i in range(10):
        x1.copy_(_tokens(g, 1))
        pos1.copy_((PRE + 30 + i + torch.arange(B)[:, None, None] * 100).expand(B, 1, A))
        row1.copy_(lens[:, None])
        held = [y.clone() for y in (K, V, mass)]
        graph.replay()
        torch.cuda.synchronize()
        row = row1.cpu()
        want = C.prefix_attend(q1.double().cpu(), Kp.double().cpu(), Vp.double().cpu(), None, K.double().cpu(), V.double().cpu(), row, 0)
        want.check(o1, y1)
        wm, tol = C.attend_mass(q1.double().cpu(), K.double().cpu(), y1.double().cpu(), row, CAP, 0, 0, held[2].cpu(), 0.95)
        assert bool(((mass.double().cpu() - wm).abs() <= tol).all()), i
        new = C.rotate_axes(_split(x1.cpu())[1].double(), pos1.cpu(), AXES, 1e4)
        for b in range(B):
            n = int(lens[b])
            _near_bf16(K[b, :, n], new[b, 0])
            for y, z in zip((K, V), held):
                assert torch.equal(y[b, :, :n], z[b, :, :n]) and torch.equal(y[b, :, n + 1:], z[b, :, n + 1:])
        lens = lens + 1
        if i == 5:
            cut()
            assert all(float(mass[b, :, int(lens[b]):].abs().sum()) == 0.0 for b in range(B))
    cut()
