"""Operators of a served cache at positions at the end of what 32 bits hold, and the bits that attention over a prefix keeps: against the
plain definitions in 64 bits."""
import pytest
import torch

import paper_2603_23516_amd as msa
import plain64 as P
import plain64_cache as C
import test_prefix_attend as prefix_of
import test_sparse_attend4 as sparse4_of

LAST = 2 ** 31 - 1


def _cfg(Hq=8, Hkv=2, d=64):
    return msa.MsaConfig(1, 1, 1, Hq, Hkv, d, 1e4)


# ---- a token at the last position sees every row that there is ---------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("B, M, Hq, Hkv", [(3, 2, 8, 1), (3, 16, 8, 1), (4, 24, 4, 1), (3, 128, 2, 2)])
@pytest.mark.parametrize("d", [64, 128])
def test_prefix_attend_at_the_last_position(B, M, Hq, Hkv, d):
    """Tokens of all sequences in a tile, and a sequence's own (96 columns a sequence and 384 in all); lengths of the prefix below
    zero and past its end."""
    x = prefix_of._make(B, M, Hq, Hkv, d, 130, 70, B + M)
    lens = torch.tensor([-3, 500, 0, 64][:B], dtype=torch.int32)
    q_pos = torch.full((B, M), LAST, dtype=torch.int32)
    prefix_of._check(Hq, Hkv, d, *x, q_pos, 0, lens)
    q_pos[:, ::2] = (torch.arange(M)[::2] % 71 - 1).to(torch.int32)      # beside tokens that see part of the cache, or nothing of it
    prefix_of._check(Hq, Hkv, d, *x, q_pos, 0, lens)


@pytest.mark.gpu
@pytest.mark.parametrize("M, pool", [(2, 0), (3, 1), (40, 1)])
def test_sparse_attend4_at_the_last_position(M, pool):
    B, N, Hkv, k = 2, 9, 2, 2
    g = torch.Generator().manual_seed(M)
    idx = torch.stack([torch.randperm(N, generator=g)[:k] for _ in range(B * (1 if pool else M) * Hkv)])
    idx = idx.reshape(B, 1 if pool else M, Hkv, k).to(torch.int32)
    q_pos = torch.full((B, M), LAST, dtype=torch.int32)
    q_pos[0, 1] = 5
    sparse4_of._check(N, 4, 8, Hkv, 64, B, M, k, 33, 0, pool, None, idx, q_pos, 0)


@pytest.mark.gpu
@pytest.mark.parametrize("M", [2, 40, 130])
def test_windows_past_32_bits_at_the_last_position(M):
    """A window of 2^31 and more holds every row up to a token's own; one of 2^31 - 1 has lost the first row by then."""
    B, Hq, Hkv, d, L = 2, 4, 2, 64, 90
    q, _, _, K, V = prefix_of._make(B, M, Hq, Hkv, d, 1, L, M)
    q_pos = torch.full((B, M), LAST, dtype=torch.int32)
    q_pos[0, 1] = 33
    cfg = _cfg(Hq, Hkv, d)
    for W in (2 ** 31, 2 ** 40, LAST):
        out, lse = msa.msa_window_attend(cfg, q.cuda(), K.cuda(), V.cuda(), q_pos.cuda(), W)
        P.window_attend(q.double(), K.double(), V.double(), q_pos, W, 0, 0).check(out, lse)
        mass = msa.msa_attend_mass(cfg, q.cuda(), K.cuda(), lse, q_pos.cuda(), W)
        want, tol = C.attend_mass(q.double(), K.double(), lse.double().cpu(), q_pos, W, 0, 0, None, 1.0)
        assert bool(((mass.double().cpu() - want).abs() <= tol).all())


# ---- attention over a prefix carries its weights as the other calls for few tokens do ----------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("B, M, Hq, Hkv, n_pre, L", [(1, 1, 8, 1, 200, 65), (5, 1, 4, 1, 900, 300), (40, 1, 4, 4, 300, 97), (3, 3, 6, 2, 130, 400),
                                                     (1, 11, 8, 1, 3000, 30), (2, 95, 2, 2, 64, 120), (1, 40, 2, 1, 33, 41), (9, 1, 5, 1, 0, 700),
                                                     (9, 1, 7, 1, 700, 0)])
@pytest.mark.parametrize("d", [64, 128])
def test_prefix_attend_of_few_tokens_keeps_pairs(B, M, Hq, Hkv, n_pre, L, d):
    """Weights as bf16 (hi, lo) pairs, off by 2^-16 of themselves at most, wherever tokens do not fill tiles of their own."""
    q, Kp, Vp, K, V = prefix_of._make(B, M, Hq, Hkv, d, n_pre, L, B + M)
    q_pos = prefix_of._ends(B, M, L, n_pre)
    dev = [t.cuda() if t.numel() else None for t in (Kp, Vp, K, V)]
    out, lse = msa.msa_prefix_attend(_cfg(Hq, Hkv, d), q.cuda(), *dev, q_pos.cuda(), local_pos0=n_pre)
    C.prefix_attend(q.double(), Kp.double(), Vp.double(), None, K.double(), V.double(), q_pos, n_pre).check(out, lse, 2.0 ** -16)


# ---- weights behind an attention that has no window ----------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("M", [3, 40, 130])
@pytest.mark.parametrize("over", [0, 1, 50, 10 ** 9])
def test_mass_behind_an_attention_without_a_window(M, over):
    """Tokens at the cache's end and past it see all of its rows: with a window greater than their rows, or with all rows among the
    first ones, every head's weights add up to the cache's share of the softmax."""
    B, Hq, Hkv, d, n_pre, L = 2, 4, 2, 64, 30, 97
    r = Hq // Hkv
    q, Kp, Vp, K, V = prefix_of._make(B, M, Hq, Hkv, d, n_pre, L, M)
    q_pos = (n_pre + L - 1 + over - (torch.arange(M) % 7)).expand(B, M).contiguous().to(torch.int32)
    cfg = _cfg(Hq, Hkv, d)
    dev = [t.cuda() for t in (q, Kp, Vp, K, V, q_pos)]
    lse = msa.msa_prefix_attend(cfg, *dev, local_pos0=n_pre)[1]
    most = int(q_pos.max()) - n_pre
    all_rows = dict(q=dev[0], Kloc=dev[3], lse=lse, q_pos=dev[5], local_pos0=n_pre)
    a, b, c = (msa.msa_attend_mass(cfg, **all_rows, **kw) for kw in (dict(window=most + 1), dict(window=1, sinks=L), dict(window=2 ** 40)))
    assert torch.equal(a, b) and torch.equal(a, c)
    want, tol = C.attend_mass(q.double(), K.double(), lse.double().cpu(), q_pos, 2 ** 40, 0, n_pre, None, 1.0)
    assert bool(((a.double().cpu() - want).abs() <= tol).all())
    # the prefix' share, in 64 bits: what is left of each head's 1 is the cache's
    x = torch.matmul(q.double().reshape(B, M, Hkv, r, d).movedim(2, 0).reshape(Hkv, -1, d), Kp.double().transpose(1, 2)) / d ** 0.5
    y = lse.double().cpu().reshape(B, M, Hkv, r).movedim(2, 0).reshape(Hkv, -1, 1)
    left = (1 - torch.exp(x - y).sum(-1)).reshape(Hkv, B, M * r).sum(-1).T
    # lse is off by 2^-16 (S + 1) + 2^-22 |lse| with S < 32 (the bound of plain64's Attended), and with it every share
    assert bool(((a.double().cpu().sum(-1) - left).abs() <= tol.sum(-1) + M * r * 2.0 ** -10).all())
    if over >= L:
        assert float(msa.msa_attend_mass(cfg, **all_rows, window=L).abs().max()) == 0.0      # a window of Lloc rows has slid past all of them


def test_workspace_of_masses_is_the_same_for_every_window():
    for B, M, L in ((1, 1, 1), (4, 509, 5003), (1, 9000, 9000), (40, 1, 8192)):
        sizes = {msa.attend_mass_workspace_bytes(_cfg(32, 8, 128), B, M, L, W, S) for W in (1, 1000, L, 2 ** 40) for S in (0, 16, L, 2 ** 40)}
        assert len(sizes) == 1 and min(sizes) >= 256
