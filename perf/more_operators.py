"""Operators around the life of a local cache while serving, as measured cases.

  axes     msa_norm_rotate_axes: norm of every query and key head, rotation to a position of several axes (time, height, width),
           and the append of keys and values to rows of the local cache that are told apart from the positions
  prefix   msa_prefix_attend: attention of a batch over a prefix that its sequences share and over their own local caches
  mass     msa_attend_mass: the attention weight that every row of the local cache receives, added up over tokens and heads
  evict    msa_evict: the rows of a cache that weigh most, the first ones and the last ones kept, the others dropped

Sizes follow the package's own configurations (32 query and 8 KV heads of 128 dimensions, the small 8 and 2 heads of 64) and the
ranges around them.
"""
import math

import numpy as np
import torch

DEV = "cuda"
own = False


# ---- cases --------------------------------------------------------------------------------------------------
def _axes(name, **kw):
    c = dict(op="axes", B=1, M=1, Hq=32, Hkv=8, d=128, T=2048, A=3, weights=True, mixed=False, base=1e6)
    c.update(kw)
    return dict(name=name, **c)


def _prefix(name, **kw):
    c = dict(op="prefix", B=1, M=1, Hq=32, Hkv=8, d=128, P=4096, T=1024, ragged=False, part=False)
    c.update(kw)
    return dict(name=name, **c)


def _mass(name, **kw):
    c = dict(op="mass", B=1, M=1, Hq=32, Hkv=8, d=128, T=2048, W=2048, S=0, ragged=False, decay=1.0)
    c.update(kw)
    return dict(name=name, **c)


def _evict(name, **kw):
    c = dict(op="evict", B=1, Hkv=8, d=128, T=4096, keep=1024, S=4, R=64, ragged=False)
    c.update(kw)
    return dict(name=name, **c)


def listed():
    return [
        # eight streams decoding behind prompts with images, one layer's projection: latency
        _axes("axes_decode", B=8, T=2048),
        # a prompt of 16384 tokens, text and images in turn: bandwidth
        _axes("axes_prompt", M=16384, T=16384),
        # three images in chunks of odd length, height and width alone, axes in turn, a small model without norms
        _axes("axes_chunk_64", B=3, M=1025, Hq=8, Hkv=2, d=64, T=1100, A=2, weights=False, mixed=True, base=1e4),
        # four streams behind a short instruction, a small model: the shortest call
        _prefix("prefix_tiny", B=4, Hq=8, Hkv=2, d=64, P=700, T=256, ragged=True),
        # sixty-four streams decoding behind one long instruction, each at its own length
        _prefix("prefix_decode", B=64, P=32768, T=1024, ragged=True),
        # five drafted tokens of each of 24 streams, odd sizes, streams that share a part of the prefix or none of it
        _prefix("prefix_draft", B=24, M=5, Hq=16, Hkv=8, d=64, P=4999, T=777, ragged=True, part=True),
        # eight questions of 128 tokens each about one document
        _prefix("prefix_question", B=8, M=128, P=16384, T=640),
        # forty streams decoding, each at its own length
        _mass("mass_decode", B=40, T=8192, W=8192, ragged=True),
        # the weights of a prompt of 8192 tokens, before its cache is cut
        _mass("mass_prompt", M=8192, T=8192, W=8192, decay=0.0),
        # chunks of prompts of different lengths, odd sizes, 64 dims, a window and first tokens, older weights fading
        _mass("mass_chunk_64", B=4, M=509, Hq=16, Hkv=8, d=64, T=5003, W=1000, S=16, ragged=True, decay=0.9),
        # a quarter of a prompt's rows kept
        _evict("evict_prompt", T=16384, keep=4096, S=4, R=512),
        # every 128 tokens of decoding a batch of streams is cut back to 4096 rows; shorter streams keep theirs
        _evict("evict_batch", B=32, T=4224, keep=4096, S=4, R=256, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_once(rng):
    op = rng.choice(["axes", "prefix", "prefix", "mass", "mass", "evict"])
    Hq, Hkv, d = rng.choice([(32, 8, 128)] * 4 + [(8, 2, 64), (16, 8, 64), (32, 4, 128), (8, 8, 64), (24, 8, 64)])
    if op == "axes":
        B = _log_int(rng, 1, 64)
        M = _log_int(rng, 1, max(1, 16384 // B))
        return dict(op=op, B=B, M=M, Hq=Hq, Hkv=Hkv, d=d, T=M + _log_int(rng, 1, 2048), A=rng.choice([1, 2, 3, 3, 4]),
                    weights=rng.random() < 0.75, mixed=rng.random() < 0.5, base=rng.choice([1e4, 1e6]))
    if op == "prefix":
        many = rng.random() < 0.4
        B, M = (rng.randint(1, 8), _log_int(rng, 2, 256)) if many else (_log_int(rng, 1, 96), 1)
        return dict(op=op, B=B, M=M, Hq=Hq, Hkv=Hkv, d=d, P=_log_int(rng, 1, 32768), T=M + _log_int(rng, 1, 2048),
                    ragged=rng.random() < 0.6, part=rng.random() < 0.3)
    if op == "mass":
        many = rng.random() < 0.5
        B, M = (rng.randint(1, 4), _log_int(rng, 2, 4096)) if many else (_log_int(rng, 1, 64), 1)
        T = M + _log_int(rng, 16, 8192 if not many else 2048)
        return dict(op=op, B=B, M=M, Hq=Hq, Hkv=Hkv, d=d, T=T, W=T if rng.random() < 0.5 else _log_int(rng, 1, 8192),
                    S=rng.choice([0, 1, 4, 16, 129]), ragged=rng.random() < 0.5, decay=rng.choice([0.0, 0.5, 0.98, 1.0, 1.0]))
    T = _log_int(rng, 16, 32768)
    keep = _log_int(rng, max(1, T // 32), T)
    S = rng.randint(0, min(16, keep))
    return dict(op=op, B=_log_int(rng, 1, 64), Hkv=Hkv, d=d, T=T, keep=keep, S=S, R=rng.randint(0, min(512, keep - S)),
                ragged=rng.random() < 0.5)


def _cost(c):
    w = work(c)
    return max(w["bytes"], w["flops"] / 50)


def draw(rng):
    most = max(_cost(c) for c in listed()) * 0.9
    while True:
        c = _draw_once(rng)
        rows = c.get("B", 1) * c.get("M", 1) * c.get("Hq", 1) * (c["T"] + c.get("P", 0)) if c["op"] in ("prefix", "mass") else 0
        cache = c["B"] * c["Hkv"] * c["T"] * c["d"]
        if _cost(c) <= most and rows <= 2 ** 31 and cache <= 2 ** 30:
            return c


# ---- inputs -------------------------------------------------------------------------------------------------
def _gen(seed, salt):
    g = torch.Generator(device=DEV)
    g.manual_seed(1_000_003 * int(seed) + salt)
    return g


def _normal(gen, shape):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.bfloat16)


def _axis_of_pair(c):
    """Which axis turns pair u of a head: one run of pairs after another, or the axes in turn."""
    half = c["d"] // 2
    return [u % c["A"] if c["mixed"] else u * c["A"] // half for u in range(half)]


def _last_rows(c, gen):
    """Row of every sequence's last token: the cache's end, or anywhere past the tokens of the pass."""
    if not c["ragged"]:
        return torch.full((c["B"],), c["T"] - 1, device=DEV)
    return torch.randint(c["M"] - 1, c["T"], (c["B"],), generator=gen, device=DEV)


def prepare(case, seed):
    c = dict(case)
    g = _gen(seed, 1)
    if c["op"] == "axes":
        B, M, Hq, Hkv, d, T, A = (c[n] for n in ("B", "M", "Hq", "Hkv", "d", "T", "A"))
        qkv = _normal(g, (B, M, (Hq + 2 * Hkv) * d)) * 2                 # what the layer's fused projection gives
        rows = (torch.randint(0, T - M + 1, (B, 1), generator=g, device=DEV) + torch.arange(M, device=DEV)).to(torch.int32)
        # text moves all axes together; in an image of 16 x 16 patches the first stands still and the others walk over it
        far = torch.randint(0, 100000, (B, 1), generator=g, device=DEV)
        t = torch.arange(M, device=DEV) + far
        image = (t // 256) % 2 == 1
        axes = [torch.where(image, t // 256 * 256, t), torch.where(image, t // 256 * 256 + t // 16 % 16, t),
                torch.where(image, t // 256 * 256 + t % 16, t), t // 256]
        pos = torch.stack(axes[:A], -1).to(torch.int32).contiguous()
        pos[torch.rand((B, M), generator=g, device=DEV) < 0.02] = -1     # padding of a batch
        w = [1 + 0.2 * _normal(g, (d,)) if c["weights"] else None for _ in range(2)]
        return dict(c=c, q=qkv[..., :Hq * d].unflatten(-1, (Hq, d)), k=qkv[..., Hq * d:(Hq + Hkv) * d].unflatten(-1, (Hkv, d)),
                    v=qkv[..., (Hq + Hkv) * d:].unflatten(-1, (Hkv, d)), pos=pos, rows=rows, axes=_axis_of_pair(c), qw=w[0],
                    kw=w[1], q_out=_normal(g, (B, M, Hq, d)), Kloc=_normal(g, (B, Hkv, T, d)), Vloc=_normal(g, (B, Hkv, T, d)))
    if c["op"] == "prefix":
        B, M, Hq, Hkv, d, P, T = (c[n] for n in ("B", "M", "Hq", "Hkv", "d", "P", "T"))
        q_pos = (P + _last_rows(c, g)[:, None] - M + 1 + torch.arange(M, device=DEV)).to(torch.int32)
        lens = None
        if c["part"]:
            lens = torch.randint(P // 2, P + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
            lens[torch.rand((B,), generator=g, device=DEV) < 0.1] = 0
        return dict(c=c, q=_normal(g, (B, M, Hq, d)), Kpre=_normal(g, (Hkv, P, d)), Vpre=_normal(g, (Hkv, P, d)),
                    Kloc=_normal(g, (B, Hkv, T, d)), Vloc=_normal(g, (B, Hkv, T, d)), q_pos=q_pos, lens=lens)
    if c["op"] == "mass":
        B, M, Hq, Hkv, d, T = (c[n] for n in ("B", "M", "Hq", "Hkv", "d", "T"))
        q_pos = (_last_rows(c, g)[:, None] - M + 1 + torch.arange(M, device=DEV)).to(torch.int32)
        s = dict(c=c, q=_normal(g, (B, M, Hq, d)), Kloc=_normal(g, (B, Hkv, T, d)), q_pos=q_pos)
        # rows that later tokens use have no weight yet
        mass = torch.rand((B, Hkv, T), generator=g, device=DEV).pow(4) * 8
        s["mass"] = torch.where(torch.arange(T, device=DEV) <= q_pos[:, -1, None, None], mass, 0.0)
        s["lse"] = torch.stack([torch.logsumexp(_scores(s, b, _seen(s, b)), -1).permute(2, 0, 1).flatten(1)
                                for b in range(B)])                     # as the attention of these tokens gives it
        s["out"] = torch.empty_like(s["mass"])
        return s
    B, Hkv, d, T, keep = (c[n] for n in ("B", "Hkv", "d", "T", "keep"))
    lens = torch.full((B,), T, device=DEV, dtype=torch.int32)
    if c["ragged"]:
        lens = torch.randint(max(1, T // 2), T + 1, (B,), generator=g, device=DEV, dtype=torch.int32)
    mass = torch.exp(1.5 * torch.randn((B, Hkv, T), generator=g, device=DEV))
    mass[torch.rand((B, Hkv, T), generator=g, device=DEV) < 0.03] = 0.0  # rows that nothing has looked at
    return dict(c=c, Kloc=_normal(g, (B, Hkv, T, d)), Vloc=_normal(g, (B, Hkv, T, d)), mass=mass, lens=lens,
                Kout=torch.zeros((B, Hkv, keep, d), device=DEV, dtype=torch.bfloat16),
                Vout=torch.zeros((B, Hkv, keep, d), device=DEV, dtype=torch.bfloat16),
                mass_out=torch.zeros((B, Hkv, keep), device=DEV),
                rows=torch.zeros((B, Hkv, keep), device=DEV, dtype=torch.int32))


# ---- the plain forms ----------------------------------------------------------------------------------------
def _plain_axes(s):
    c, pos = s["c"], s["pos"].long()
    d = c["d"]
    theta = torch.pow(torch.tensor(c["base"], dtype=torch.float64, device=DEV),
                      torch.arange(d // 2, device=DEV, dtype=torch.float64) * (-2.0 / d))
    angle = pos[..., torch.tensor(s["axes"], device=DEV)].double()[:, :, None] * theta
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()

    def turned(x, w):
        x = x.float()
        if w is not None:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w.float()
        a, b = x[..., :d // 2], x[..., d // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin], -1).to(torch.bfloat16)

    here = pos[..., 0] >= 0
    q_out = torch.where(here[..., None, None], turned(s["q"], s["qw"]), s["q_out"])
    row = s["rows"].long()
    at = here & (row >= 0) & (row < c["T"])
    b = torch.arange(c["B"], device=DEV)[:, None].expand_as(row)[at]
    s["Kloc"][b, :, row[at]] = turned(s["k"], s["kw"])[at]
    s["Vloc"][b, :, row[at]] = s["v"][at]
    return q_out, s["Kloc"], s["Vloc"]


def _rows(q, Hkv):
    """[B][M][Hq][d] -> fp32 [B][Hkv][r M][d]."""
    B, M, Hq, d = q.shape
    return q.float().reshape(B, M, Hkv, Hq // Hkv, d).permute(0, 2, 3, 1, 4).reshape(B, Hkv, Hq // Hkv * M, d)


def _back(x, M, r):
    """[B][Hkv][r M][...] -> [B][M][Hq][...]."""
    x = x.unflatten(2, (r, M)).movedim(3, 1)
    return x.flatten(2, 3).contiguous()


def _plain_prefix(s):
    c = s["c"]
    B, M, Hkv, P = c["B"], c["M"], c["Hkv"], c["P"]
    r, scale = c["Hq"] // Hkv, 1 / math.sqrt(c["d"])
    q = _rows(s["q"], Hkv)
    every = q.transpose(0, 1).reshape(Hkv, -1, c["d"])                   # the queries of all sequences, by KV head
    far = torch.matmul(every, s["Kpre"].float().transpose(-1, -2)).unflatten(1, (B, -1)).transpose(0, 1)
    near = torch.matmul(q, s["Kloc"].float().transpose(-1, -2))          # [B][Hkv][r M][T]
    x = torch.cat([far, near], -1) * scale
    del far, near
    t = torch.arange(P, device=DEV)
    seen = torch.cat([(t < (P if s["lens"] is None else s["lens"].long()[:, None, None])).expand(B, M, P),
                      torch.arange(c["T"], device=DEV) + P <= s["q_pos"].long()[:, :, None]], -1)
    x.masked_fill_(~seen.repeat(1, r, 1)[:, None], -math.inf)
    top = x.amax(-1, keepdim=True).clamp_min(-3e38)
    x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    out = torch.matmul(x[..., :P].transpose(0, 1).reshape(Hkv, -1, P), s["Vpre"].float()).unflatten(1, (B, -1)).transpose(0, 1)
    out = (out + torch.matmul(x[..., P:], s["Vloc"].float())) / total.clamp_min(1e-30)
    lse = (top + torch.log(total)).squeeze(-1)
    return _back(out, M, r).to(torch.bfloat16), _back(lse, M, r)


def _seen(s, b):
    """Which rows of the cache the tokens of sequence b see, [M][T]."""
    c = s["c"]
    t, p = torch.arange(c["T"], device=DEV), s["q_pos"][b].long()[:, None]
    return (t <= p) & ((p - t < c["W"]) | (t < c["S"]))


def _scores(s, b, seen):
    """Scores of sequence b, fp32 [Hkv][r][M][T], minus infinity where a row is not seen."""
    c = s["c"]
    q = s["q"][b].float().unflatten(1, (c["Hkv"], -1)).permute(1, 2, 0, 3)
    x = torch.matmul(q.flatten(1, 2), s["Kloc"][b].float().transpose(-1, -2)).unflatten(1, (-1, c["M"]))
    return x.mul_(1 / math.sqrt(c["d"])).masked_fill_(~seen, -math.inf)


def _plain_mass(s):
    c = s["c"]
    for b in range(c["B"]):
        lse = s["lse"][b].unflatten(1, (c["Hkv"], -1)).permute(1, 2, 0)[..., None]
        weight = _scores(s, b, _seen(s, b)).sub_(lse).exp_()
        s["out"][b] = s["mass"][b] * c["decay"] + weight.sum((1, 2))
    return s["out"]


def _plain_evict(s):
    c = s["c"]
    T, keep = c["T"], c["keep"]
    t, n = torch.arange(T, device=DEV), s["lens"].long()[:, None, None]
    always = (t < c["S"]) | (t >= n - c["R"])
    # by weight, the lowest row first where weights are equal; then those that stay anyway in front, rows not in use last
    order = torch.sort(s["mass"], dim=-1, descending=True, stable=True).indices
    rank = torch.where(t >= n, 2, torch.where(always, 0, 1)).expand_as(order)
    order = order.gather(-1, torch.sort(rank.gather(-1, order), dim=-1, stable=True).indices)
    kept = torch.where(order[..., :keep] < n, order[..., :keep], T).sort(dim=-1).values
    there = kept < T
    at = kept.clamp_max(T - 1)
    for x, y in (("Kloc", "Kout"), ("Vloc", "Vout")):
        moved = s[x].gather(2, at[..., None].expand(*at.shape, c["d"]))
        s[y].copy_(torch.where(there[..., None], moved, s[y]))
    s["mass_out"].copy_(torch.where(there, s["mass"].gather(2, at), s["mass_out"]))
    s["rows"].copy_(torch.where(there, kept, -1))
    return s["Kout"], s["Vout"], s["mass_out"], s["rows"]


# ---- the framework's calls --------------------------------------------------------------------------------------
def _plan(s):
    """What a program keeps from call to call: the config, the workspace and the output buffers."""
    import paper_2603_23516_amd as msa
    c = s["c"]
    cfg = msa.MsaConfig(1, 1, 1, c.get("Hq", c["Hkv"]), c["Hkv"], c["d"], c.get("base", 1e6))
    plan = dict(msa=msa, cfg=cfg)
    size = None
    if c["op"] == "prefix":
        size = msa.prefix_attend_workspace_bytes(cfg, c["B"], c["M"], c["P"], c["T"])
        plan.update(out=torch.empty_like(s["q"]), lse=torch.empty(s["q"].shape[:3], dtype=torch.float32, device=DEV))
    if c["op"] == "mass":
        size = msa.attend_mass_workspace_bytes(cfg, c["B"], c["M"], c["T"], c["W"], c["S"])
    if size is not None:
        plan.update(workspace=torch.empty(max(size, 256), dtype=torch.uint8, device=DEV))
    return plan


def run(state):
    s, c = state, state["c"]
    if own:
        if "plan" not in s:
            s["plan"] = _plan(s)
        p = s["plan"]
        msa, cfg = p["msa"], p["cfg"]
        if c["op"] == "axes":
            msa.msa_norm_rotate_axes(cfg, s["q"], s["k"], s["v"], s["pos"], s["axes"], s["Kloc"], s["Vloc"], rows=s["rows"],
                                     q_weight=s["qw"], k_weight=s["kw"], eps=1e-6, q_out=s["q_out"])
            return s["q_out"], s["Kloc"], s["Vloc"]
        if c["op"] == "prefix":
            return msa.msa_prefix_attend(cfg, s["q"], s["Kpre"], s["Vpre"], s["Kloc"], s["Vloc"], s["q_pos"], local_pos0=c["P"],
                                         prefix_lens=s["lens"], out=p["out"], lse=p["lse"], workspace=p["workspace"])
        if c["op"] == "mass":
            return msa.msa_attend_mass(cfg, s["q"], s["Kloc"], s["lse"], s["q_pos"], c["W"], sinks=c["S"], mass=s["mass"],
                                       decay=c["decay"], out=s["out"], workspace=p["workspace"])
        return msa.msa_evict(cfg, s["Kloc"], s["Vloc"], s["mass"], s["lens"], c["keep"], sinks=c["S"], recent=c["R"],
                             Kout=s["Kout"], Vout=s["Vout"], mass_out=s["mass_out"], rows=s["rows"])
    return {"axes": _plain_axes, "prefix": _plain_prefix, "mass": _plain_mass, "evict": _plain_evict}[c["op"]](s)


# ---- what a pass cannot do without -----------------------------------------------------------------------------------
def _pairs(c, window, sinks):
    """Rows that the tokens of one sequence see, and the rows that any of them sees, with the sequence at the cache's end
    (at half of it where lengths differ)."""
    last = c["T"] - 1 if not c["ragged"] else max(c["M"] - 1, (c["T"] + c["M"]) // 2 - 1)
    first = last - c["M"] + 1
    pairs = 0
    for p in range(first, last + 1):
        lo = max(0, p - window + 1)
        pairs += p + 1 - lo + min(sinks, lo)
    lo = max(0, first - window + 1)
    return pairs, last + 1 - lo + min(sinks, lo)


def work(case):
    c = case
    d = c["d"]
    if c["op"] == "axes":
        n = c["B"] * c["M"] * (c["Hq"] + 2 * c["Hkv"]) * d
        return {"bytes": 4 * n + 4 * c["B"] * c["M"] * (c["A"] + 1), "flops": 8 * n}
    if c["op"] == "prefix":
        pairs, rows = _pairs(c, c["T"], 0)
        q, shared = c["B"] * c["M"] * c["Hq"], c["P"] * (0.675 if c["part"] else 1)
        return {"bytes": 4 * q * d + 4 * q + 4 * c["Hkv"] * c["P"] * d + 4 * c["B"] * c["Hkv"] * rows * d,
                "flops": 4 * d * (q * shared + c["B"] * c["Hq"] * pairs)}
    if c["op"] == "mass":
        pairs, rows = _pairs(c, c["W"], c["S"])
        q = c["B"] * c["M"] * c["Hq"]
        return {"bytes": 2 * q * d + 4 * q + 2 * c["B"] * c["Hkv"] * rows * d + (8 if c["decay"] else 4) * c["B"] * c["Hkv"] * c["T"],
                "flops": 2 * c["B"] * c["Hq"] * pairs * d}
    length = 0.75 * c["T"] if c["ragged"] else c["T"]
    heads, kept = c["B"] * c["Hkv"], min(c["keep"], length)
    return {"bytes": heads * (4 * length + kept * (8 * d + 8)), "flops": heads * length}


# ---- the definition in 64 bits -----------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    B, Hkv, d, T = c["B"], c["Hkv"], c["d"], c["T"]
    if c["op"] == "axes":
        half = d // 2
        which = torch.tensor(s["axes"], device=DEV)
        turn = s["pos"].double().index_select(2, which) * c["base"] ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half)
        turn = torch.polar(torch.ones_like(turn), turn)[:, :, None]

        def turned(x, w):
            x = x.double()
            if w is not None:
                x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / d + 1e-6) * w.double()
            z = torch.complex(x[..., :half], x[..., half:]) * turn
            return torch.cat([z.real, z.imag], -1)

        q, k = turned(s["q"], s["qw"]), turned(s["k"], s["kw"])
        padding = s["pos"][..., 0] < 0
        q[padding] = s["q_out"].double()[padding]
        Kloc, Vloc = s["Kloc"].double(), s["Vloc"].double()
        for b in range(B):
            m = torch.nonzero(~padding[b]).flatten()
            Kloc[b][:, s["rows"][b][m].long()] = k[b][m].transpose(0, 1)
            Vloc[b][:, s["rows"][b][m].long()] = s["v"][b][m].double().transpose(0, 1)
        return q, Kloc, Vloc
    if c["op"] == "evict":
        mass, lens = s["mass"].cpu().numpy(), s["lens"].tolist()
        Kout, Vout, mass_out = s["Kout"].double(), s["Vout"].double(), s["mass_out"].double()
        rows = np.full(s["rows"].shape, -1, dtype=np.int64)
        for b in range(B):
            n = lens[b]
            for g in range(Hkv):
                stay = np.arange(n)
                if n > c["keep"]:
                    middle = np.arange(c["S"], n - c["R"])
                    best = middle[np.lexsort((middle, -mass[b, g, middle].astype(np.float64)))][:c["keep"] - c["S"] - c["R"]]
                    stay = np.sort(np.concatenate([np.arange(c["S"]), best, np.arange(n - c["R"], n)]))
                rows[b, g, :len(stay)] = stay
                at = torch.from_numpy(stay).to(DEV)
                Kout[b, g, :len(stay)] = s["Kloc"][b, g, at].double()
                Vout[b, g, :len(stay)] = s["Vloc"][b, g, at].double()
                mass_out[b, g, :len(stay)] = s["mass"][b, g, at].double()
        return Kout, Vout, mass_out, torch.from_numpy(rows).to(DEV)
    M, Hq = c["M"], c["Hq"]
    if c["op"] == "mass":
        out = s["mass"].double() * c["decay"]
        for b in range(B):
            last, row = s["q_pos"][b].long()[:, None], torch.arange(T, device=DEV)[None]
            seen = (row <= last) & ((row > last - c["W"]) | (row < c["S"]))
            for h in range(Hq):
                x = s["q"][b, :, h].double() @ s["Kloc"][b, h * Hkv // Hq].double().T / math.sqrt(d)
                w = torch.exp(x - s["lse"][b, :, h, None].double())
                out[b, h * Hkv // Hq] += torch.where(seen, w, 0.0).sum(0)
        return out
    out = torch.zeros((B, M, Hq, d), dtype=torch.float64, device=DEV)
    lse = torch.full((B, M, Hq), -math.inf, dtype=torch.float64, device=DEV)
    for b in range(B):
        n = c["P"] if s["lens"] is None else int(s["lens"][b])
        row = torch.cat([torch.full((n,), -1, device=DEV), c["P"] + torch.arange(T, device=DEV)])
        seen = row[None] <= s["q_pos"][b].long()[:, None]
        for g in range(Hkv):
            K = torch.cat([s["Kpre"][g, :n], s["Kloc"][b, g]]).double()
            V = torch.cat([s["Vpre"][g, :n], s["Vloc"][b, g]]).double()
            heads = slice(g * Hq // Hkv, (g + 1) * Hq // Hkv)
            q = s["q"][b, :, heads].double().transpose(0, 1)
            x = (q.reshape(-1, d) @ K.T / math.sqrt(d)).masked_fill(~seen.repeat(q.shape[0], 1), -math.inf)
            y = torch.logsumexp(x, 1)
            o = torch.exp(x - torch.where(torch.isinf(y), 0.0, y)[:, None]) @ V
            out[b, :, heads] = o.reshape(q.shape).transpose(0, 1)
            lse[b, :, heads] = y.reshape(q.shape[:2]).T
    return out, lse
