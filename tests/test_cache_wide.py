"""The operators around the life of a local cache at the largest batches and numbers of heads: grids are as wide as they may be."""
import pytest
import torch

import paper_2603_23516_amd as msa
import plain64_cache as C

MANY, ENDS = 65535, 40


def _cfg(Hkv, r=1, d=64):
    return msa.MsaConfig(1, 1, 1, Hkv * r, Hkv, d, 1e4)


def _of(shape, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)


def _ends(Hkv):
    """(batch, heads) of the first and of the last ones: those that the definition is worked out for."""
    return [(slice(None), slice(0, ENDS)), (slice(None), slice(Hkv - ENDS, Hkv))] if Hkv > 1 else \
        [(slice(0, ENDS), slice(None)), (slice(MANY - ENDS, MANY), slice(None))]


@pytest.mark.gpu
@pytest.mark.parametrize("B, Hkv, M", [(MANY, 1, 1), (1, MANY, 1), (MANY, 1, 5), (1, MANY, 70)])
def test_prefix_attend_and_mass(B, Hkv, M):
    d, n_pre, L = 64, 5, 3
    cfg = _cfg(Hkv)
    q, Kp, Vp, K, V = (_of(s, i) for i, s in enumerate(((B, M, Hkv, d), (Hkv, n_pre, d), (Hkv, n_pre, d), (B, Hkv, L, d), (B, Hkv, L, d))))
    q_pos = (n_pre + torch.arange(B)[:, None] % 4 - 1 + torch.zeros((1, M))).to(torch.int32)      # none, one, two or all rows
    lens = (torch.arange(B) % 6).to(torch.int32)
    dev = [t.cuda() for t in (q, Kp, Vp, K, V, q_pos)]
    out, lse = msa.msa_prefix_attend(cfg, *dev, local_pos0=n_pre, prefix_lens=lens.cuda())
    mass = msa.msa_attend_mass(cfg, dev[0], dev[3], lse, dev[5], L, local_pos0=n_pre)
    torch.cuda.synchronize()
    for b, g in _ends(Hkv):
        x = q[b][:, :, g].double()
        want = C.prefix_attend(x, Kp[g].double(), Vp[g].double(), lens[b], K[b][:, g].double(), V[b][:, g].double(), q_pos[b], n_pre)
        want.check(out[b][:, :, g].contiguous(), lse[b][:, :, g].contiguous(), 2.0 ** -8)
        y, tol = C.attend_mass(x, K[b][:, g].double(), lse[b][:, :, g].double().cpu(), q_pos[b], L, 0, n_pre, None, 1.0)
        assert bool(((mass[b][:, g].double().cpu() - y).abs() <= tol).all())


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B, Hkv", [(65536, 1), (1, 65535), (16384, 4)])
def test_evict(B, Hkv, in_place):
    d, L, keep = 64, 9, 4
    K, V = _of((B, Hkv, L, d), 1), _of((B, Hkv, L, d), 2)
    mass = torch.rand((B, Hkv, L), generator=torch.Generator().manual_seed(3)).argsort(-1).float() / 8      # no two of a head are equal
    lens = (torch.arange(B) % (L + 1)).to(torch.int32) if B > 1 else torch.tensor([L], dtype=torch.int32)
    into = [t.cuda() for t in (K, V, mass)]
    others = {} if in_place else dict(Kout=torch.zeros_like(into[0][:, :, :keep]), Vout=torch.zeros_like(into[1][:, :, :keep]),
                                      mass_out=torch.zeros_like(into[2][:, :, :keep]))
    others = {n: t.contiguous() for n, t in others.items()}
    Ko, Vo, mo, rows = (t.cpu() for t in msa.msa_evict(_cfg(Hkv), *into, lens.cuda(), keep, sinks=1, recent=1, **others))
    n = lens[:, None].expand(B, Hkv)
    t = torch.arange(L)
    middle = (t >= 1) & (t < n[..., None] - 1)
    order = torch.where(middle, mass, -1.0).argsort(-1, descending=True)[..., :keep - 2]
    last = (n - 1)[..., None].clamp(min=0)
    want = torch.cat([torch.zeros((B, Hkv, 1), dtype=torch.long), order.sort(-1)[0], last.long()], -1)
    short = torch.arange(keep).expand(B, Hkv, keep)
    want = torch.where((n > keep)[..., None], want, torch.where(short < n[..., None], short, -1))
    assert torch.equal(rows.long(), want)
    at, kept = want.clamp(min=0), want >= 0
    for x, y in ((Ko, K), (Vo, V)):
        y = y.gather(2, at[..., None].expand(B, Hkv, keep, d))
        assert torch.equal(torch.where(kept[..., None], x[:, :, :keep], 0), torch.where(kept[..., None], y, 0))
    assert torch.equal(mo[..., :keep], torch.where(kept, mass.gather(2, at), 0.0)) and not bool(((n > keep)[..., None] & (mo[..., keep:] != 0)).any())


@pytest.mark.gpu
@pytest.mark.parametrize("B, Hkv", [(MANY, 1), (1, MANY)])
def test_norm_rotate_axes(B, Hkv):
    d, L = 64, 2
    cfg = _cfg(Hkv)
    q, k, v = (_of((B, 1, Hkv, d), i) for i in range(3))
    pos = torch.randint(0, 3000, (B, 1, 2), generator=torch.Generator().manual_seed(5), dtype=torch.int32)
    rows = (torch.arange(B) % 3)[:, None].to(torch.int32)                                       # a third of them behind the cache
    axes = [u % 2 for u in range(d // 2)]
    K, V = (torch.zeros((B, Hkv, L, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    out = msa.msa_norm_rotate_axes(cfg, q.cuda(), k.cuda(), v.cuda(), pos.cuda(), axes, K, V, rows=rows.cuda())
    torch.cuda.synchronize()
    for b, g in _ends(Hkv):
        for x, got in ((q, out), (k, None)):
            want = C.rotate_axes(x[b][:, :, g].double(), pos[b], axes, 1e4)
            # a rounding, and two products in fp32 with sines and cosines of angles worked out in 64 bits
            tol = want.abs() * 2.0 ** -8 + x[b][:, :, g].double().abs().amax() * 2.0 ** -20
            if got is not None:
                assert bool(((got[b][:, :, g].double().cpu() - want).abs() <= tol).all())
            else:
                for i in range(want.shape[0]):
                    t = int(rows[b][i, 0])
                    for row in range(L):
                        y = K[b][i, g, row].double().cpu()
                        if row == t:
                            assert bool(((y - want[i, 0]).abs() <= tol[i, 0]).all())
                            assert torch.equal(V[b][i, g, row].cpu(), v[b][i, 0, g])
                        else:
                            assert not bool(y.any())
