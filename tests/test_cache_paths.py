"""The operators around the life of a local cache by path: the borders between their kernels, many parts, workspaces that calls and
graphs share, several host threads."""
import threading

import pytest
import torch

import paper_2603_23516_amd as msa
import plain64_cache as C
import test_attend_mass as mass_of
import test_evict as evict_of
import test_prefix_attend as prefix_of


def _cfg(Hq=8, Hkv=2, d=64):
    return msa.MsaConfig(1, 1, 1, Hq, Hkv, d, 1e4)


# ---- attention over a prefix ------------------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("B, M, Hq, Hkv", [(3, 24, 4, 1), (4, 24, 4, 1), (4, 23, 4, 1), (1, 95, 4, 1), (1, 96, 4, 1), (2, 95, 2, 2),
                                           (6, 96, 1, 1), (4, 12, 8, 1), (5, 11, 8, 1), (3, 32, 7, 1), (3, 44, 3, 1)])
def test_prefix_where_its_kernels_meet(B, M, Hq, Hkv):
    """Tokens of all sequences in a tile, or a sequence's own: 96 columns a sequence and 384 in all, heads that do not divide a tile."""
    x = prefix_of._make(B, M, Hq, Hkv, 64, 77, M + 20, B + M)
    lens = torch.tensor([77, 0, 40, 33, 77, 64][:B], dtype=torch.int32)
    prefix_of._check(Hq, Hkv, 64, *x, prefix_of._ends(B, M, M + 20, 77), 77, lens)


@pytest.mark.gpu
@pytest.mark.parametrize("B, M, n_pre, L", [(1, 1, 20000, 9000), (1, 3, 20480, 30), (2, 1, 50, 9000), (5, 1, 20000, 64)])
def test_prefix_in_many_parts(B, M, n_pre, L):
    """More parts than a wave takes at a time, than a wave has lanes, and twice as many; some sequences see few of them."""
    x = prefix_of._make(B, M, 2, 1, 64, n_pre, L, 3)
    q_pos = prefix_of._ends(B, M, L, n_pre)
    prefix_of._check(2, 1, 64, *x, q_pos, n_pre)
    lens = torch.tensor([n_pre - 1, 700, 0, 33, 4100][:B], dtype=torch.int32)
    q_pos[0] = n_pre + 40
    prefix_of._check(2, 1, 64, *x, q_pos, n_pre, lens)


@pytest.mark.gpu
@pytest.mark.parametrize("B, M", [(3, 1), (2, 17), (4, 40)])
def test_a_workspace_of_the_longest_call_serves_shorter_ones(B, M):
    cfg = _cfg(8, 2, 128)
    q, Kp, Vp, K, V = (t.cuda() for t in prefix_of._make(B, M, 8, 2, 128, 4000, 900, 5))
    ws = torch.full((msa.prefix_attend_workspace_bytes(cfg, B, M, 4000, 900),), 0x7F, dtype=torch.uint8, device="cuda")
    mw = torch.full((msa.attend_mass_workspace_bytes(cfg, B, M, 900, 900),), 0x7F, dtype=torch.uint8, device="cuda")
    for P, L in ((4000, 900), (31, 900), (4000, 1), (1000, 333), (1, 1)):
        a = [t[:, :P].contiguous() for t in (Kp, Vp)] + [t[:, :, :L].contiguous() for t in (K, V)]
        pos = prefix_of._ends(B, M, L, P).cuda()
        one, two = (msa.msa_prefix_attend(cfg, q, *a, pos, local_pos0=P, workspace=w) for w in (ws, None))
        assert torch.equal(one[0], two[0]) and torch.equal(one[1], two[1]), (P, L)
        lse = torch.where(pos[..., None] >= P, one[1], torch.full_like(one[1], -float("inf")))
        one, two = (msa.msa_attend_mass(cfg, q, a[2], lse, pos, L, local_pos0=P, workspace=w) for w in (mw, None))
        assert torch.equal(one, two), (P, L)


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", [((3, 1, 2000, 300), (5, 2, 700, 900)), ((8, 40, 900, 100), (4, 60, 1500, 100)), ((1, 1, 4000, 5), (6, 96, 600, 200))])
def test_graphs_that_share_a_workspace(sizes):
    """Two captured calls on one workspace, replayed in turn: each leaves what it should, whatever the other left behind.  (What a
    graph reads is kept: inputs, positions, workspace.)"""
    cfg, sets = _cfg(8, 2, 128), []
    need = max(msa.prefix_attend_workspace_bytes(cfg, *s) for s in sizes)
    need = max([need] + [msa.attend_mass_workspace_bytes(cfg, B, M, L, L) for B, M, P, L in sizes])
    ws = torch.full((need,), 0xEE, dtype=torch.uint8, device="cuda")
    for i, (B, M, P, L) in enumerate(sizes):
        x = [t.cuda() for t in prefix_of._make(B, M, 8, 2, 128, P, L, i)]
        pos = prefix_of._ends(B, M, L, P).cuda()
        out, lse, mass = torch.empty_like(x[0]), torch.empty((B, M, 8), device="cuda"), torch.empty((B, 2, L), device="cuda")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            msa.msa_prefix_attend(cfg, *x, pos, local_pos0=P, out=out, lse=lse, workspace=ws)
            msa.msa_attend_mass(cfg, x[0], x[3], lse, pos, L, local_pos0=P, out=mass, workspace=ws)
        want = msa.msa_prefix_attend(cfg, *x, pos, local_pos0=P)
        sets.append((graph, (out, lse, mass), want + (msa.msa_attend_mass(cfg, x[0], x[3], want[1], pos, L, local_pos0=P),), (x, pos)))
    for i in (0, 1, 1, 0, 1, 0, 0):
        graph, got, want, _ = sets[i]
        for t in got:
            t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i


@pytest.mark.gpu
def test_calls_from_several_threads():
    cfg = _cfg(8, 2, 128)
    sets = [[t.cuda() for t in prefix_of._make(4, 1, 8, 2, 128, 1500, 200, i)] for i in range(4)]
    pos = prefix_of._ends(4, 1, 200, 1500).cuda()
    lens = torch.full((4,), 200, dtype=torch.int32, device="cuda")

    def work(x, stream=None):
        out, lse = msa.msa_prefix_attend(cfg, *x, pos, local_pos0=1500, stream=stream)
        mass = msa.msa_attend_mass(cfg, x[0], x[3], lse, pos, 200, local_pos0=1500, stream=stream)
        outs = [torch.zeros((4, 2, 50, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)] + [torch.zeros((4, 2, 50), device="cuda")]
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        return [out, lse, mass] + list(msa.msa_evict(cfg, x[3], x[4], mass, lens, 50, sinks=1, recent=3, Kout=outs[0], Vout=outs[1],
                                                     mass_out=outs[2], stream=stream))

    want = [work(x) for x in sets]
    torch.cuda.synchronize()
    bad = []

    def run(i):
        stream = torch.cuda.Stream()
        for _ in range(10):
            got = work(sets[i], stream)
            stream.synchronize()
            if not all(torch.equal(a, b) for a, b in zip(got, want[i])):
                bad.append(i)

    threads = [threading.Thread(target=run, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad


# ---- weights of the cache's rows -----------------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("M, Hq, Hkv", [(64, 1, 1), (65, 1, 1), (16, 4, 1), (17, 4, 1), (12, 5, 1), (13, 5, 1), (9, 7, 1), (10, 7, 1), (300, 3, 1),
                                        (200, 8, 1), (513, 2, 2)])
@pytest.mark.parametrize("d", [64, 128])
def test_mass_where_its_kernels_meet(M, Hq, Hkv, d):
    """Up to 64 columns in registers, more through LDS; heads that do not divide a step; several parts."""
    L = M + 130
    q, K, V, mass = mass_of._make(2, M, Hq, Hkv, d, L, M)
    q_pos = (L - M + torch.arange(M)).expand(2, M).contiguous().to(torch.int32)
    q_pos[1] -= 60
    mass_of._check(Hq, Hkv, d, q, K, V, mass, q_pos, 100, 2, 0, decay=0.5)
    mass_of._check(Hq, Hkv, d, q, K, V, mass, q_pos, L, 0, 0, in_place=True)


@pytest.mark.gpu
def test_mass_of_tokens_out_of_order():
    """Positions at random: hardly any tile is seen whole, and the tokens of a tile's first and last row lie anywhere."""
    g = torch.Generator().manual_seed(4)
    q, K, V, mass = mass_of._make(1, 400, 4, 2, 128, 700, 6)
    q_pos = torch.randint(-50, 720, (1, 400), generator=g, dtype=torch.int32)
    for W, S in ((700, 0), (64, 0), (200, 150), (1, 700)):
        mass_of._check(4, 2, 128, q, K, V, mass, q_pos, W, S, 0)


# ---- eviction --------------------------------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("L", [1024, 1025, 8192, 8193, 16384, 16385, 32768, 32769])
def test_evict_where_its_kernels_meet(in_place, L):
    for kind, keep in (("spread", L // 3), ("ties", L // 2), ("odd", 65)):
        K, V, mass = evict_of._make(1, 2, L, 64, kind, L)
        evict_of._check(K, V, mass, torch.tensor([L], dtype=torch.int32), keep, 3, 30, in_place)


@pytest.mark.gpu
@pytest.mark.parametrize("L", [700, 40000])
def test_evict_by_the_last_bit(L):
    """Weights one step apart, weights from the smallest to the largest, few and many rows that weigh the same at the border, all
    that is wanted or nothing of the middle."""
    g = torch.Generator().manual_seed(L)
    step = (0x3F800000 + torch.randperm(L, generator=g).to(torch.int32)).view(torch.float32)
    wide = (torch.randint(0, 0x7F800000, (L,), generator=g).to(torch.int32)).view(torch.float32) * torch.where(torch.rand(L, generator=g) < 0.5, -1.0, 1.0)
    few, many = step.clone(), step.clone()
    few[torch.randperm(L, generator=g)[:40]] = 1.00001
    many[torch.randperm(L, generator=g)[:L // 2]] = 1.00001
    none = torch.full((L,), float("-inf"))
    mass = torch.stack([step, wide, few, many, none, -step])[:, None]
    B = mass.shape[0]
    K, V = (torch.randn((B, 1, L, 64), generator=g).to(torch.bfloat16) for _ in range(2))
    lens = torch.full((B,), L, dtype=torch.int32)
    for keep, S, R in ((L // 2, 0, 0), (L // 2 + 17, 5, 9), (40, 30, 10), (L - 1, 0, 0), (1, 0, 0)):
        evict_of._check(K, V, mass.contiguous(), lens, keep, S, R, False)


@pytest.mark.gpu
def test_evict_of_many_sequences():
    K, V, mass = evict_of._make(300, 8, 40, 64, "ties", 2)
    lens = torch.randint(0, 41, (300,), generator=torch.Generator().manual_seed(1), dtype=torch.int32)
    for in_place in (False, True):
        evict_of._check(K, V, mass, lens, 24, 2, 6, in_place)
