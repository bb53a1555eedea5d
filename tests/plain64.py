"""Plain definitions, in 64 bits on the CPU, of the operators around the local cache and the bank in four bits."""
import math

import torch

CODES = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def rotate(x, pos, base):
    """x [..., d] at pos [...]: element u pairs with u + d/2, angle pos * base^(-2u/d)."""
    h = x.shape[-1] // 2
    ang = pos.double()[..., None] * base ** (-torch.arange(h, dtype=torch.float64) / h)
    a, b, c, s = x[..., :h], x[..., h:], torch.cos(ang), torch.sin(ang)
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def norm(x, w, eps):
    return x if w is None else x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * w


def scale_byte(amax):
    """The smallest e with amax <= 7 * 2^(e - 127), between 2 and 252, by trying them."""
    for e in range(2, 253):
        if amax <= 7 * 2.0 ** (e - 127):
            return e
    return 252


def pack4(x):
    """x [..., d] float64 -> (values it is kept as, scale bytes [..., d/32])."""
    b = x.reshape(-1, 32)
    e = torch.tensor([scale_byte(float(m)) for m in b.abs().amax(1)], dtype=torch.float64)
    y = (b / (2.0 ** (e - 127))[:, None]).abs().clamp(max=6.0)
    dist = (y[..., None] - CODES).abs()
    near = dist == dist.amin(-1, keepdim=True)
    even = near & (torch.arange(8) % 2 == 0)                                   # of two equally near ones the even code
    pick = torch.where(even.any(-1, keepdim=True), even, near).double().argmax(-1)
    v = torch.sign(b) * CODES[pick] * (2.0 ** (e - 127))[:, None]
    return v.reshape(x.shape), e.reshape(x.shape[:-1] + (x.shape[-1] // 32,)).to(torch.uint8)


def unpack4(codes, scales):
    n = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()
    v = CODES[n & 7] * torch.where(n >= 8, -1.0, 1.0)
    return v * torch.exp2(scales.double() - 127).repeat_interleave(32, -1)


def attend(q, K, V, seen):
    """q [d], K, V [t][d], seen [t] -> (output [d], log of the sum); nothing seen: zeros, -inf."""
    if not bool(seen.any()):
        return torch.zeros(V.shape[1], dtype=torch.float64), -math.inf
    x = (K[seen] @ q) / math.sqrt(q.shape[0])
    lse = torch.logsumexp(x, 0)
    return torch.exp(x - lse) @ V[seen], float(lse)


def window_attend(q, Kloc, Vloc, q_pos, window, sinks, pos0):
    """q [B][M][Hq][d], caches [B][Hkv][L][d], all float64."""
    B, M, Hq, d = q.shape
    r = Hq // Kloc.shape[1]
    out, lse = torch.zeros_like(q), torch.full((B, M, Hq), -math.inf, dtype=torch.float64)
    t = torch.arange(Kloc.shape[2])
    for b in range(B):
        for m in range(M):
            p = int(q_pos[b, m]) - pos0
            seen = (t <= p) & ((p - t < window) | (t < sinks))
            for h in range(Hq):
                out[b, m, h], lse[b, m, h] = attend(q[b, m, h], Kloc[b, h // r], Vloc[b, h // r], seen)
    return out, lse


def sparse_attend4(q, K, V, idx, lens, Kloc, Vloc, q_pos, pos0):
    """K, V [N][Hkv][G][d]: what the bank stands for; idx [B][M'][S][k]."""
    B, M, Hq, d = q.shape
    N, Hkv, G, _ = K.shape
    r, Mp, S = Hq // Hkv, idx.shape[1], idx.shape[2]
    out, lse = torch.zeros_like(q), torch.full((B, M, Hq), -math.inf, dtype=torch.float64)
    for b in range(B):
        for m in range(M):
            near = torch.arange(Kloc.shape[2]) + pos0 <= int(q_pos[b, m])
            for g in range(Hkv):
                docs = [int(i) for i in idx[b, m if Mp > 1 else 0, g if S > 1 else 0] if 0 <= int(i) < N]
                n = [G if lens is None else min(max(int(lens[i]), 1), G) for i in docs]
                Kx = torch.cat([K[i, g, :x] for i, x in zip(docs, n)] + [Kloc[b, g][near]])
                Vx = torch.cat([V[i, g, :x] for i, x in zip(docs, n)] + [Vloc[b, g][near]])
                seen = torch.ones(Kx.shape[0], dtype=torch.bool)
                for h in range(g * r, g * r + r):
                    out[b, m, h], lse[b, m, h] = attend(q[b, m, h], Kx, Vx, seen)
    return out, lse
