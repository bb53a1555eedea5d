"""Plain definitions, in 64 bits on the CPU, of the operators around the life of a local cache."""
import math

import torch

import plain64 as P


def rotate_axes(x, pos, axes, base):
    """x [B][M][H][d], pos [B][M][A]: pair u by the position of axis axes[u]."""
    h = x.shape[-1] // 2
    ang = pos.double()[..., list(axes)][:, :, None] * base ** (-torch.arange(h, dtype=torch.float64) / h)
    a, b, c, s = x[..., :h], x[..., h:], torch.cos(ang), torch.sin(ang)
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def prefix_attend(q, Kpre, Vpre, lens, Kloc, Vloc, q_pos, pos0):
    """q [B][M][Hq][d], Kpre, Vpre [Hkv][P][d], lens [B] or None, Kloc, Vloc [B][Hkv][L][d], all float64."""
    B, M, Hq, d = q.shape
    Hkv, n_pre = Kpre.shape[:2]
    r = Hq // Hkv
    res = P.Attended((B, M, Hq), d)
    t = torch.arange(Kloc.shape[2])
    for b in range(B):
        n = n_pre if lens is None else min(max(int(lens[b]), 0), n_pre)
        for m in range(M):
            seen = torch.cat([torch.ones(n, dtype=torch.bool), t <= int(q_pos[b, m]) - pos0])
            for g in range(Hkv):
                K, V = torch.cat([Kpre[g, :n], Kloc[b, g]]), torch.cat([Vpre[g, :n], Vloc[b, g]])
                for h in range(g * r, g * r + r):
                    res.put((b, m, h), P.attend(q[b, m, h], K, V, seen))
    return res


def attend_mass(q, Kloc, lse, q_pos, window, sinks, pos0, mass, decay):
    """-> (out [B][Hkv][L], its error bound).

    A score is an fp32 sum of d <= 128 exact products, off by d 2^-24 S with S the sum of their magnitudes, scaled and rounded a few
    times; lse is scaled and rounded: a weight is off by 2^-16 (S / sqrt(d) + 1) + 2^-21 |lse| of itself.  n weights are added with
    n 2^-23 at most, the old one scaled and added with 2^-23."""
    B, M, Hq, d = q.shape
    Hkv, L = Kloc.shape[1:3]
    old = torch.zeros((B, Hkv, L), dtype=torch.float64) if mass is None or decay == 0 else mass.double() * decay
    out, tol = old.clone(), old.abs() * 2.0 ** -22
    t = torch.arange(L)
    for b in range(B):
        for m in range(M):
            p = int(q_pos[b, m]) - pos0
            seen = (t <= p) & ((p - t < window) | (t < sinks))
            if not bool(seen.any()):
                continue
            for h in range(Hq):
                g, y = h // (Hq // Hkv), float(lse[b, m, h])
                if y == -math.inf:
                    continue
                K = Kloc[b, g][seen]
                w = torch.exp(K @ q[b, m, h] / math.sqrt(d) - y)
                size = K.abs() @ q[b, m, h].abs() / math.sqrt(d)
                out[b, g, seen] += w
                tol[b, g, seen] += w * (2.0 ** -16 * (size + 1) + 2.0 ** -21 * abs(y) + M * (Hq // Hkv) * 2.0 ** -23)
    return out, tol


def evict_rows(mass, n, keep, sinks, recent):
    """Rows of one (sequence, KV head) that stay, by sorting tuples."""
    if n <= keep:
        return list(range(n))
    middle = range(sinks, n - recent)

    def weight(t):
        x = float(mass[t])
        return (0, 0.0) if math.isnan(x) else (1, x)

    best = sorted(middle, key=lambda t: (tuple(-w for w in weight(t)), t))[:keep - sinks - recent]
    return sorted(list(range(sinks)) + best + list(range(n - recent, n)))
