"""A cache that msa_evict has cut, read by row by the calls that take it: the kept rows of each head, then a token appended behind them."""
import pytest
import torch

import paper_2603_23516_amd as msa
import plain64 as P
import plain64_cache as C

B, Hq, Hkv, d, L, KEEP, N, G, k = 2, 8, 2, 64, 60, 24, 5, 8, 2


@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("pos0", [0, 1000])
def test_read_by_row(in_place, pos0):
    g = torch.Generator().manual_seed(3)
    cfg = msa.MsaConfig(N, G, 1, Hq, Hkv, d, 1e4, bank_keys_rotated=1)
    K, V, new_k, new_v = (torch.randn(s, generator=g).to(torch.bfloat16) for s in ((B, Hkv, L, d),) * 2 + ((B, Hkv, d),) * 2)
    q, Kb, Vb = (torch.randn(s, generator=g).to(torch.bfloat16) for s in ((B, 1, Hq, d), (N, Hkv, G, d), (N, Hkv, G, d)))
    mass, lens = torch.rand((B, Hkv, L), generator=g), torch.tensor([L, 17], dtype=torch.int32)     # the second is short enough
    dev = [t.cuda() for t in (K, V, mass)]
    outs = {} if in_place else dict(Kout=torch.zeros_like(dev[0]), Vout=torch.zeros_like(dev[1]), mass_out=torch.zeros_like(dev[2]))
    Kc, Vc, _, _ = msa.msa_evict(cfg, *dev, lens.cuda(), KEEP, sinks=2, recent=5, **outs)
    # by hand: the rows that stay, then the new token's
    cut = [torch.zeros((B, Hkv, L, d), dtype=torch.bfloat16) for _ in range(2)]
    row = lens.clamp(max=KEEP)
    for b in range(B):
        for h in range(Hkv):
            at = C.evict_rows(mass[b, h], int(lens[b]), KEEP, 2, 5)
            for x, y, z in zip(cut, (K, V), (new_k, new_v)):
                x[b, h, :len(at)], x[b, h, len(at)] = y[b, h, at], z[b, h]
        for x, z in ((Kc, new_k), (Vc, new_v)):
            x[b, :, int(row[b])] = z[b].cuda()
    q_pos = (pos0 + row)[:, None].to(torch.int32)
    cut64 = [t.double() for t in cut]
    for W, S in ((10, 3), (L, 0)):
        out, lse = msa.msa_window_attend(cfg, q.cuda(), Kc, Vc, q_pos.cuda(), W, sinks=S, local_pos0=pos0)
        P.window_attend(q.double(), *cut64, q_pos, W, S, pos0).check(out, lse, 2.0 ** -16)
    out, lse = msa.msa_prefix_attend(cfg, q.cuda(), Kb[0].cuda(), Vb[0].cuda(), Kc, Vc, q_pos.cuda(), local_pos0=pos0)
    C.prefix_attend(q.double(), Kb[0].double(), Vb[0].double(), None, *cut64, q_pos, pos0).check(out, lse, 2.0 ** -16)
    bank = msa.msa_pack_kv4(cfg, Kb.cuda(), Vb.cuda())
    kept = [P.unpack4(bank[i].cpu(), bank[i + 1].cpu()) for i in (0, 2)]
    idx = torch.tensor([[[[3, 0], [1, 4]]], [[[2, -1], [0, 1]]]], dtype=torch.int32)
    out, lse = msa.msa_sparse_attend4(cfg, q.cuda(), bank, idx.cuda(), Kc, Vc, pos0, q_pos.cuda())
    P.sparse_attend4(q.double(), *kept, idx, None, *cut64, q_pos, pos0).check(out, lse, 2.0 ** -16)
    out = msa.msa_attend_mass(cfg, q.cuda(), Kc, lse, q_pos.cuda(), L, local_pos0=pos0)
    want, tol = C.attend_mass(q.double(), cut64[0], lse.double().cpu(), q_pos, L, 0, pos0, None, 1.0)
    assert bool(((out.double().cpu() - want).abs() <= tol).all())
