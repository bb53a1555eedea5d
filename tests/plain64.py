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
    """q [d], K, V [t][d], seen [t] -> output [d], log of the sum (nothing seen: zeros, -inf), and for error bounds the same mean
    of |V|, the largest sum of |q_i k_i| / sqrt(d) and the number of rows."""
    if not bool(seen.any()):
        return torch.zeros(V.shape[1], dtype=torch.float64), -math.inf, torch.zeros(V.shape[1], dtype=torch.float64), 0.0, 0
    x = (K[seen] @ q) / math.sqrt(q.shape[0])
    lse = torch.logsumexp(x, 0)
    w = torch.exp(x - lse)
    size = float((K[seen].abs() @ q.abs()).max()) / math.sqrt(q.shape[0])
    return w @ V[seen], float(lse), w @ V[seen].abs(), size, int(seen.sum())


class Attended:
    """Outputs and log-sums of many heads with their error bounds.

    Scores: fp32 sums of d <= 128 exact products, off by d 2^-24 sum|q_i k_i| at most, scaled and rounded a few times: a weight
    is off by delta = 2^-16 (S + 1) relative, S the largest sum|q_i k_i| / sqrt(d).  The sum of n weights adds n 2^-23.  Weights
    rounded to bf16 are off by 2^-8 at most, those carried as (hi, lo) pairs by 2^-16.  The output is rounded to bf16: 2^-8."""

    def __init__(self, shape, d):
        z = dict(dtype=torch.float64)
        self.out, self.mass = torch.zeros(shape + (d,), **z), torch.zeros(shape + (d,), **z)
        self.lse, self.size, self.n = torch.full(shape, -math.inf, **z), torch.zeros(shape, **z), torch.zeros(shape, **z)

    def put(self, at, got):
        self.out[at], self.lse[at], self.mass[at], self.size[at], self.n[at] = got

    def check(self, out, lse, weights=2.0 ** -8):
        out, lse = out.double().cpu(), lse.double().cpu()
        delta = 2.0 ** -16 * (self.size + 1) + self.n * 2.0 ** -23
        tol = 2.0 ** -8 * self.out.abs() + (weights + 2 * delta)[..., None] * self.mass
        err = (out - self.out).abs()
        assert bool((err <= tol).all()), f"output: off by {float((err - tol).max())} more than the bound"
        empty = torch.isinf(self.lse)
        assert torch.equal(torch.isinf(lse) & (lse < 0), empty)
        off = (lse - self.lse).abs()[~empty] - (delta + 2.0 ** -22 * self.lse.abs())[~empty]
        assert bool((off <= 0).all()), f"log-sum: off by {float(off.max())} more than the bound"


def window_attend(q, Kloc, Vloc, q_pos, window, sinks, pos0):
    """q [B][M][Hq][d], caches [B][Hkv][L][d], all float64."""
    B, M, Hq, d = q.shape
    r = Hq // Kloc.shape[1]
    res = Attended((B, M, Hq), d)
    t = torch.arange(Kloc.shape[2])
    for b in range(B):
        for m in range(M):
            p = int(q_pos[b, m]) - pos0
            seen = (t <= p) & ((p - t < window) | (t < sinks))
            for h in range(Hq):
                res.put((b, m, h), attend(q[b, m, h], Kloc[b, h // r], Vloc[b, h // r], seen))
    return res


def sparse_attend4(q, K, V, idx, lens, Kloc, Vloc, q_pos, pos0):
    """K, V [N][Hkv][G][d]: what the bank stands for; idx [B][M'][S][k]."""
    B, M, Hq, d = q.shape
    N, Hkv, G, _ = K.shape
    r, Mp, S = Hq // Hkv, idx.shape[1], idx.shape[2]
    res = Attended((B, M, Hq), d)
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
                    res.put((b, m, h), attend(q[b, m, h], Kx, Vx, seen))
    return res
