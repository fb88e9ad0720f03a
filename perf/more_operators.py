"""What the normed rotation and the cache that keeps its rows' attention weight are
timed on: norms and rotation of queries and keys and their gradient, attention
that appends and adds up what every row was given, and eviction by that sum.

norm_rope: of each head's row x of d channels, r = (mean x^2 + eps)^-1/2, y = w x r,
then the pairs of y turn by their positions (time, height, width), as in the
rotation without a norm.  Its gradient, with g the output's gradient turned back
and n = x r: dx = r (w g - n mean(w g n)), dw = sum over tokens and heads of g n.

Attention with mass: a cache of bf16 rows in pools, unit u = (l*B + b)*Hkv + g at
rows row_off[u] + t, t < len[u].  c = count[b] new rows of k and v are appended,
query i sees the rows before them and the first i + 1 of them, and
  out = softmax(scale q K^T) V,  mass[t] <- decay mass[t] + sum of the weights that
row t got from the queries and heads of its group (new rows start at 0).

Eviction: unit u keeps keep[u] rows: the first `sinks`, the last `recent` and of the
others those of the largest mass, ties to the lower index; they stay in order and
move together, in place or into another cache.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
THETA = 1e6
EPS = 1e-6
# Model shapes of the seeded workloads: layers, query heads, kv heads, head dim.
MODELS = {"tiny": (4, 8, 2, 64), "7b": (28, 28, 4, 128), "72b": (80, 64, 8, 128)}


# ---- the cases ---------------------------------------------------------------

def _norm(name, kind, model, L, B, n, **kw):
    _, Hq, Hkv, d = MODELS[model]
    c = {"name": name, "kind": kind, "L": L, "B": B, "Hq": Hq, "Hkv": Hkv, "d": d, "n": n, "rot": d,
         "s0": d // 8, "s1": 3 * d // 16, "s2": 3 * d // 16, "interleaved": False, "adjacent": False,
         "fp32": False, "w_fp32": False, "far": 1 << 15}
    c.update(kw)
    return c


def _attend(name, model, L, B, lo, hi, n, **kw):
    _, Hq, Hkv, d = MODELS[model]
    c = {"name": name, "kind": "attend", "L": L, "B": B, "Hq": Hq, "Hkv": Hkv, "d": d, "lo": lo, "hi": hi,
         "n": n, "fp32": False, "ragged": False, "append": True, "decay": 1.0}
    c.update(kw)
    return c


def _evict(name, model, L, B, lo, hi, share, **kw):
    _, Hq, Hkv, d = MODELS[model]
    c = {"name": name, "kind": "evict", "L": L, "B": B, "Hq": Hq, "Hkv": Hkv, "d": d, "lo": lo, "hi": hi,
         "share": share, "sinks": 4, "recent": 32, "inplace": True}
    c.update(kw)
    return c


def listed():
    return [
        # One token of eight sequences, queries and keys of all layers: latency.
        _norm("norm_step", "norm", "7b", 28, 8, 1),
        # A long video's prompt (64 frames of 196 tokens and the question) in one layer.
        _norm("norm_prompt", "norm", "7b", 1, 1, 12608, w_fp32=True),
        # The gradient over a training batch of two sequences of an odd length in one layer of a large model.
        _norm("grad_train", "grad", "72b", 1, 2, 8191),
        # The gradient of short fp32 sequences in all layers of a small model, axes interleaved.
        _norm("grad_tiny", "grad", "tiny", 4, 3, 77, fp32=True, w_fp32=True, interleaved=True, s0=12, s1=10, s2=10),
        # One token over a small model's pruned cache: launches and latency.
        _attend("token_tiny", "tiny", 4, 1, 90, 170, 1, fp32=True),
        # One token over a short video's pruned cache, all layers, old weights fading.
        _attend("token_7b", "7b", 28, 1, 620, 1490, 1, fp32=True, decay=0.98),
        # Serving: one token of each of eight sequences over their pruned caches, all layers.
        _attend("token_batched", "7b", 28, 8, 2300, 5800, 1),
        # A follow-up question of up to 65 tokens to each of three long videos, one layer.
        _attend("question", "7b", 1, 3, 9001, 12801, 65, ragged=True),
        # A long second prompt over a long video in one layer of a large model.
        _attend("prompt_long", "72b", 1, 1, 23040, 23040, 2048),
        # A small model's cache that went over its budget is cut back, in place: latency.
        _evict("evict_tiny", "tiny", 4, 1, 150, 250, 0.7),
        # A short video's caches in all layers, cut back in place to their layers' budgets.
        _evict("evict_7b", "7b", 28, 1, 2400, 3136, 0.6),
        # The caches of a batch of eight videos compacted into pools of their own.
        _evict("evict_batched", "7b", 28, 8, 2300, 5800, 0.5, inplace=False),
    ]


def _log(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.99))))


def draw(rng):
    most = [work(c) for c in listed()]
    top_bytes, top_flops = max(w["bytes"] for w in most), max(w["flops"] for w in most)
    while True:
        kind = rng.choice(("norm", "grad", "attend", "attend", "attend", "evict", "evict"))
        model = rng.choice(("tiny", "7b", "7b", "72b"))
        Lm, _, _, d = MODELS[model]
        L, B = rng.choice((1, 1, 2, Lm)), rng.choice((1, 1, 2, 3, 8))
        if kind in ("norm", "grad"):
            rot = rng.choice((d, d, d // 2))
            a = rng.randint(0, rot // 4)
            c = _norm(None, kind, model, L, B, _log(rng, 1, 16000), rot=rot, s0=rot // 2 - 2 * a, s1=a, s2=a,
                      interleaved=rng.random() < 0.4, adjacent=rng.random() < 0.3, fp32=rng.random() < 0.4,
                      far=rng.choice((1 << 12, 1 << 17, 1 << 22)))
            c["w_fp32"] = c["fp32"] or rng.random() < 0.5
        elif kind == "attend":
            hi = _log(rng, 3, 32000)
            lo = max(0, int(hi * rng.uniform(0.3, 1.0)))
            n = rng.choice((1, 1, 2, _log(rng, 2, 3000)))
            c = _attend(None, model, L, B, lo, hi, n, fp32=rng.random() < (0.6 if n == 1 else 0.2),
                        ragged=rng.random() < 0.5, append=rng.random() < 0.7, decay=rng.choice((1.0, 0.97, 0.0)))
        else:
            hi = _log(rng, 1, 32000)
            lo = max(0, int(hi * rng.uniform(0.2, 1.0)))
            c = _evict(None, model, L, B, lo, hi, rng.uniform(0.02, 1.0), sinks=rng.choice((0, 4, 128)),
                       recent=rng.choice((0, 32, 1000)), inplace=rng.random() < 0.6)
        del c["name"]
        w = work(c)
        if w["bytes"] <= top_bytes and w["flops"] <= top_flops and _scores(c) <= 3.5e9:
            return c


# ---- sizes -------------------------------------------------------------------

def _spread(i, lo, hi):
    """A size in [lo, hi] for item i, the same in every run."""
    return lo + ((i * 2654435761 + 97) % (1 << 32) * (hi - lo + 1) >> 32)


def _lens(c):
    return [_spread(u, c["lo"], c["hi"]) for u in range(c["L"] * c["B"] * c["Hkv"])]


def _counts(c):
    """Queries of each sequence."""
    if not c["ragged"]:
        return [c["n"]] * c["B"]
    return [c["n"] if b == 0 else _spread(b, 0, c["n"]) for b in range(c["B"])]


def _keeps(c):
    """Rows that each unit keeps, fewer in deep layers, on average the case's share of the longest."""
    per = c["B"] * c["Hkv"]
    f = lambda l: c["share"] * (1.25 - 0.5 * l / max(c["L"] - 1, 1))  # noqa: E731
    return [int(c["hi"] * min(f(u // per), 1.0)) for u in range(c["L"] * per)]


def _scores(c):
    return c["L"] * c["B"] * c["Hq"] * c["n"] * (c["hi"] + c["n"]) if c["kind"] == "attend" else 0


def _seen(c, n, k):
    """(rows held, first query's rows) of a unit of n rows with k queries."""
    return (n + k, n + 1) if c["append"] else (n, n - k + 1)


def work(c):
    L, B, Hq, Hkv, d = c["L"], c["B"], c["Hq"], c["Hkv"], c["d"]
    G = Hq // Hkv
    if c["kind"] in ("norm", "grad"):
        values, e = L * B * c["n"] * (Hq + Hkv) * d, 4 if c["fp32"] else 2
        passes, flops = (2, 8) if c["kind"] == "norm" else (3, 16)
        return {"bytes": passes * e * values + 12 * B * c["n"], "flops": flops * values}
    lens, byts, flops = _lens(c), 0, 0
    if c["kind"] == "attend":
        counts = _counts(c)
        for u, n in enumerate(lens):
            k = counts[u // Hkv % B]
            if k == 0:
                continue
            rows, first = _seen(c, n, k)
            byts += 4 * d * rows + 8 * n + 4 * (rows - n)  # keys and values, the mass
            if c["append"]:
                byts += 4 * d * k  # into the pools
            j = max(0, min(k, k + first - 1))  # queries that see a row
            flops += 4 * d * G * (j * max(first, 1) + j * (j - 1) // 2)
        byts += L * sum(counts) * Hq * d * (6 if c["fp32"] else 4)
        return {"bytes": byts, "flops": flops}
    for n, k in zip(lens, _keeps(c)):
        m = min(n, k)
        byts += 4 * n + 4 * m  # the mass, the indices
        byts += 2 * m * (4 * d + 4) if m < n or not c["inplace"] else 0
        flops += n
    return {"bytes": byts, "flops": flops}


# ---- inputs ------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(0xCAC4E + 7919 * seed)
    return g


def _rows(g, shape, d):
    """Rows as a model leaves them: a few loud channels, a few loud tokens."""
    x = torch.randn(shape + (d,), generator=g, device=DEV)
    x *= torch.exp(0.5 * torch.randn((d,), generator=g, device=DEV))
    loud = torch.rand(shape, generator=g, device=DEV) < 0.01
    return torch.where(loud[..., None], 6 * x, x)


def _positions(g, c):
    """Time, height and width of visual tokens, then text with three equal positions."""
    B, n = c["B"], c["n"]
    start = torch.randint(0, c["far"], (B, 1), generator=g, device=DEV, dtype=torch.int32)
    i = torch.arange(n, device=DEV, dtype=torch.int32)[None]
    text = i >= n - n // 8
    axes = (torch.where(text, i, i // 196), torch.where(text, i, i % 196 // 14), torch.where(text, i, i % 14))
    return torch.stack([start + x for x in axes]).contiguous()


def _pool(c, g, caps):
    """Pools with room for these rows a unit, one unit behind the other."""
    first = [0] * len(caps)
    for u in range(1, len(caps)):
        first[u] = first[u - 1] + caps[u - 1]
    total = max(1, sum(caps))
    s = {"row_off": torch.tensor(first, dtype=torch.int64, device=DEV), "caps": caps, "max_rows": max(caps),
         "cap": torch.tensor(caps, dtype=torch.int32, device=DEV)}
    if g is None:
        s["k_pool"] = torch.zeros((total, c["d"]), dtype=torch.bfloat16, device=DEV)
        s["v_pool"], s["mass"] = torch.zeros_like(s["k_pool"]), torch.zeros((total,), device=DEV)
    else:
        s["k_pool"], s["v_pool"] = (_rows(g, (total,), c["d"]).to(torch.bfloat16) for _ in "kv")
        # Heavy tails; some rows were never looked at, some alike.
        m = torch.exp(2 * torch.randn((total,), generator=g, device=DEV))
        r = torch.rand((total,), generator=g, device=DEV)
        s["mass"] = torch.where(r < 0.05, 0.0, torch.where(r < 0.15, torch.round(4 * m) / 4, m))
    return s


def prepare(case, seed):
    g, c = _gen(seed), case
    L, B, Hq, Hkv, d = c["L"], c["B"], c["Hq"], c["Hkv"], c["d"]
    s = {"case": c}
    if c["kind"] in ("norm", "grad"):
        s["pos"] = _positions(g, c)
        typ, wtyp = (torch.float32 if f else torch.bfloat16 for f in (c["fp32"], c["w_fp32"]))
        for side, H in (("q", Hq), ("k", Hkv)):
            s[side] = _rows(g, (L, B, c["n"], H), d).to(typ)
            s[side + "_weight"] = (1 + 0.2 * torch.randn((L, d), generator=g, device=DEV)).to(wtyp)
            s[side + "_out"] = torch.empty_like(s[side])
            if c["kind"] == "grad":
                s[side + "_dout"] = (0.01 * torch.randn(s[side].shape, generator=g, device=DEV)).to(typ)
        return s
    lens = _lens(c)
    if c["kind"] == "attend":
        s |= _pool(c, g, [n + c["n"] for n in lens])
        s["q"] = torch.randn((L, B, c["n"], Hq, d), generator=g, device=DEV).to(torch.bfloat16)
        s["k"], s["v"] = (_rows(g, (L, B, c["n"], Hkv), d).to(torch.bfloat16) for _ in "kv")
        s["count"] = torch.tensor(_counts(c), dtype=torch.int32, device=DEV) if c["ragged"] else None
        s["out"] = torch.zeros(s["q"].shape, dtype=torch.float32 if c["fp32"] else torch.bfloat16, device=DEV)
    else:
        s |= _pool(c, g, [n + 1 for n in lens])
        keeps = _keeps(c)
        s["keep"] = torch.tensor(keeps, dtype=torch.int32, device=DEV)
        s["index"] = torch.full((len(lens), max(max(min(n, k) for n, k in zip(lens, keeps)), 1)), -1, dtype=torch.int32,
                                device=DEV)
        s["mass_before"] = s["mass"].clone()
        if not c["inplace"]:
            s["to"] = _pool(c, None, [min(n, k) + 1 for n, k in zip(lens, keeps)])
            s["to"]["len"] = torch.zeros((len(lens),), dtype=torch.int32, device=DEV)
    s["before"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    s["len"] = s["before"].clone()
    return s


# ---- the plain forms -----------------------------------------------------------

def _axis(c):
    """The axis of each frequency."""
    i = torch.arange(c["rot"] // 2, device=DEV)
    if c["interleaved"]:
        return torch.where((i % 3 == 1) & (i < 3 * c["s1"]), 1, torch.where((i % 3 == 2) & (i < 3 * c["s2"]), 2, 0))
    return (i >= c["s0"]).long() + (i >= c["s0"] + c["s1"]).long()


def _turn(y, c, pos, back=False):
    """fp32 y [L, B, n, H, d] turned (back); angles in 64 bits."""
    rot = c["rot"]
    f = THETA ** (-2.0 * torch.arange(rot // 2, device=DEV, dtype=torch.float64) / rot)
    a = pos[_axis(c)].permute(1, 2, 0).double() * f  # [B, n, rot/2]
    cos, sin = torch.cos(a).float()[None, :, :, None], torch.sin(a).float()[None, :, :, None]
    sin = -sin if back else sin
    if c["adjacent"]:
        y1, y2 = y[..., 0:rot:2], y[..., 1:rot:2]
        r = torch.stack((y1 * cos - y2 * sin, y2 * cos + y1 * sin), dim=-1).flatten(-2)
    else:
        y1, y2 = y[..., :rot // 2], y[..., rot // 2:rot]
        r = torch.cat((y1 * cos - y2 * sin, y2 * cos + y1 * sin), dim=-1)
    return torch.cat((r, y[..., rot:]), dim=-1)


def _plain_norm(s, c, side):
    x, w = s[side].float(), s[side + "_weight"].float()[:, None, None, None]
    r = torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS)
    if c["kind"] == "norm":
        s[side + "_out"].copy_(_turn(x * r * w, c, s["pos"]))
        return
    g = _turn(s[side + "_dout"].float(), c, s["pos"], back=True)
    n = x * r
    dn = g * w
    s[side + "_out"].copy_(r * (dn - n * (dn * n).mean(dim=-1, keepdim=True)))
    s[side + "_dw"] = (g * n).sum(dim=(1, 2, 3), dtype=torch.float64).float()


def _unit_rows(s, rows):
    """Pool rows [units, rows] of the first `rows` rows of every unit (clamped to the pool)."""
    at = s["row_off"][:, None] + torch.arange(rows, device=DEV)[None]
    return at.clamp(max=s["k_pool"].shape[0] - 1)


def _plain_attend(s, c):
    L, B, Hq, Hkv, d, n = c["L"], c["B"], c["Hq"], c["Hkv"], c["d"], c["n"]
    G, units, rows = Hq // Hkv, L * B * Hkv, max(s["max_rows"], 1)
    held = s["len"].long()[:, None]  # [units, 1]
    count = s["count"].long() if c["ragged"] else torch.full((B,), n, device=DEV)
    count = count[None, :, None].expand(L, B, Hkv).reshape(units, 1)
    i = torch.arange(n, device=DEV)[None]
    if c["append"]:
        ok = i < count
        at = (s["row_off"][:, None] + held + i)[ok]
        for side in "kv":
            s[side + "_pool"][at] = s[side].permute(0, 1, 3, 2, 4).reshape(units, n, d)[ok]
        s["mass"][at] = 0.0
        base, held = held, held + count
        s["len"].copy_(held[:, 0])
    else:
        base = held - count
    at = _unit_rows(s, rows)
    t = torch.arange(rows, device=DEV)[None]
    x = s["q"].float().reshape(L, B, n, Hkv, G, d).permute(0, 1, 3, 2, 4, 5).reshape(units, n * G, d)
    S = torch.matmul(x, s["k_pool"][at].float().transpose(1, 2)) * d ** -0.5
    ends = torch.where(i < count, torch.minimum(base + i + 1, held), 0).repeat_interleave(G, dim=1)
    S.masked_fill_(t[:, None] >= ends[..., None], -math.inf)
    top = S.amax(dim=-1, keepdim=True)
    S = torch.exp(S - torch.where(top > -math.inf, top, 0.0))
    total = S.sum(dim=-1, keepdim=True)
    S /= torch.where(total > 0, total, 1.0)
    V = torch.where((t < held)[..., None], s["v_pool"][at].float(), 0.0)
    o = torch.matmul(S, V).reshape(L, B, Hkv, n, G, d).permute(0, 1, 3, 2, 4, 5).reshape(L, B, n, Hq, d)
    live = (i < count.reshape(L, B, Hkv)[0, :, :1])[None, :, :, None, None]
    s["out"].copy_(torch.where(live, o.to(s["out"].dtype), s["out"]))
    got = S.sum(dim=1, dtype=torch.float64)
    ok = (t < held) & (count > 0)
    s["mass"][at[ok]] = (c["decay"] * s["mass"][at].double() + got).float()[ok]


def _plain_evict(s, c):
    units, rows = len(s["caps"]), s["max_rows"]
    to = s if c["inplace"] else s["to"]
    n, t = s["len"].long()[:, None], torch.arange(rows, device=DEV)[None]
    keep = torch.minimum(s["keep"].long()[:, None], n)
    first = keep.clamp(max=c["sinks"])
    last = (keep - first).clamp(max=c["recent"])
    at = _unit_rows(s, rows)
    m = s["mass"][at]
    held = (t < first) | ((t >= n - last) & (t < n))
    m = torch.where(held, math.inf, torch.where(t < n, m, -math.inf))
    rank = torch.sort(m, dim=1, descending=True, stable=True).indices  # ties to the lower index
    stays = torch.zeros((units, rows), dtype=torch.bool, device=DEV)
    stays.scatter_(1, rank, t.expand(units, rows) < keep)
    src, u = at[stays], torch.arange(units, device=DEV)[:, None].expand(units, rows)[stays]
    j = (stays.long().cumsum(dim=1) - 1)[stays]
    dst = to["row_off"][u] + j
    for name in ("k_pool", "v_pool", "mass"):
        to[name][dst] = s[name][src]
    s["index"][u, j] = t.expand(units, rows)[stays].int()
    to["len"].copy_(keep[:, 0])


def _plain(s, c):
    if c["kind"] == "attend":
        _plain_attend(s, c)
    elif c["kind"] == "evict":
        _plain_evict(s, c)
    else:
        _plain_norm(s, c, "q")
        _plain_norm(s, c, "k")


# ---- the framework's calls -----------------------------------------------------

_BUFFERS = ("k_pool", "v_pool", "mass", "row_off", "cap", "len")


def _handles(s, c):
    """What a program keeps beside its buffers: the caches' handles and the rotation's parameters."""
    import paper_2608_24063_amd as vc
    from paper_2608_24063_amd.tensors import MassCache, NormRope, Rope
    if c["kind"] in ("norm", "grad"):
        s["rope"] = NormRope(Rope(c["d"], rot=c["rot"], theta=THETA, sections=(c["s0"], c["s1"], c["s2"]),
                                  layout=vc.VC_ROPE_INTERLEAVED if c["interleaved"] else vc.VC_ROPE_SECTIONED,
                                  pairing=vc.VC_ROPE_ADJACENT if c["adjacent"] else vc.VC_ROPE_HALVES), eps=EPS)
        return
    make = lambda x: MassCache(c["L"], c["B"], c["Hq"], c["Hkv"], c["d"], x["caps"], DEV,  # noqa: E731
                               buffers={k: x[k] for k in _BUFFERS})
    s["cache"] = make(s)
    s["to_cache"] = make(s["to"]) if "to" in s else None


def _own(s, c):
    if "rope" not in s and "cache" not in s:
        _handles(s, c)
    if c["kind"] == "norm":
        s["rope"].apply(s["pos"], s["q"], s["k"], s["q_weight"], s["k_weight"], q_out=s["q_out"], k_out=s["k_out"])
    elif c["kind"] == "grad":
        _, _, s["q_dw"], s["k_dw"] = s["rope"].grad(s["pos"], s["q"], s["k"], s["q_weight"], s["k_weight"], s["q_dout"],
                                                    s["k_dout"], q_din=s["q_out"], k_din=s["k_out"])
    elif c["kind"] == "attend":
        k, v = (s["k"], s["v"]) if c["append"] else (None, None)
        s["cache"].attend(s["q"], s["out"], c["d"] ** -0.5, k=k, v=v, count=s["count"], decay=c["decay"])
    else:
        s["cache"].evict(s["keep"], sinks=c["sinks"], recent=c["recent"], to=s["to_cache"], index=s["index"])


def run(s):
    c = s["case"]
    if c["kind"] in ("attend", "evict"):
        s["len"].copy_(s["before"])
    if c["kind"] == "evict" and c["inplace"]:
        s["mass"].copy_(s["mass_before"])
    (_own if own else _plain)(s, c)
    if c["kind"] == "norm":
        return {"q": s["q_out"], "k": s["k_out"]}
    if c["kind"] == "grad":
        return {"q_din": s["q_out"], "k_din": s["k_out"], "q_dw": s["q_dw"], "k_dw": s["k_dw"]}
    if c["kind"] == "attend":
        return {"out": s["out"], "mass": s["mass"], "len": s["len"], "k_pool": s["k_pool"], "v_pool": s["v_pool"]}
    to = s if c["inplace"] else s["to"]
    return {"k_pool": to["k_pool"], "v_pool": to["v_pool"], "mass": to["mass"], "index": s["index"], "len": to["len"]}


# ---- the definition in 64 bits -------------------------------------------------

def _exact_turn(x, c, pos, sign):
    rot, out = c["rot"], x.clone()
    for i in range(rot // 2):
        if c["interleaved"]:
            ax = 1 if i % 3 == 1 and i < 3 * c["s1"] else 2 if i % 3 == 2 and i < 3 * c["s2"] else 0
        else:
            ax = 0 if i < c["s0"] else 1 if i < c["s0"] + c["s1"] else 2
        a = pos[ax].double() * math.exp(-2.0 * i / rot * math.log(THETA))
        co, si = torch.cos(a)[None, :, :, None], sign * torch.sin(a)[None, :, :, None]
        p, q = (2 * i, 2 * i + 1) if c["adjacent"] else (i, i + rot // 2)
        out[..., p] = x[..., p] * co - x[..., q] * si
        out[..., q] = x[..., q] * co + x[..., p] * si
    return out


def _exact_norm(s, c):
    got = {}
    for side in "qk":
        x, w = s[side].double(), s[side + "_weight"].double()[:, None, None, None]
        var = x.square().mean(dim=-1, keepdim=True) + EPS
        if c["kind"] == "norm":
            got[side] = _exact_turn(x / var.sqrt() * w, c, s["pos"], 1.0)
            continue
        # By the quotient rule, with h = w g: dx_c = h_c / sqrt(var) - x_c sum(h x) / (d var^1.5).
        g = _exact_turn(s[side + "_dout"].double(), c, s["pos"], -1.0)
        h = w * g
        got[side + "_din"] = h / var.sqrt() - x * (h * x).sum(dim=-1, keepdim=True) / (c["d"] * var ** 1.5)
        got[side + "_dw"] = torch.stack([(g[l] * x[l] / var[l].sqrt()).reshape(-1, c["d"]).sum(dim=0)
                                         for l in range(c["L"])])
    return got


def _exact_attend(s, c):
    B, Hq, Hkv, d = c["B"], c["Hq"], c["Hkv"], c["d"]
    G, counts, lens = Hq // Hkv, _counts(c), _lens(c)
    out, mass, held = s["out"].double(), s["mass"].double(), list(lens)
    pools = {side: s[side + "_pool"].clone() for side in "kv"}
    first = s["row_off"].tolist()
    for u, n in enumerate(lens):
        l, b, g = u // (B * Hkv), u // Hkv % B, u % Hkv
        k, o = counts[b], first[u]
        if k == 0:
            continue
        if c["append"]:
            pools["k"][o + n:o + n + k] = s["k"][l, b, :k, g]
            pools["v"][o + n:o + n + k] = s["v"][l, b, :k, g]
            mass[o + n:o + n + k] = 0
            held[u] = n = n + k
        K, V = pools["k"][o:o + n].double(), pools["v"][o:o + n].double()
        got = torch.zeros((n,), dtype=torch.float64, device=DEV)
        for i0 in range(0, k, 256):
            i1 = min(k, i0 + 256)
            q = s["q"][l, b, i0:i1, g * G:(g + 1) * G].reshape(-1, d).double()
            sees = n - k + 1 + torch.arange(i0, i1, device=DEV).repeat_interleave(G)
            S = (q @ K.t() * d ** -0.5).masked_fill(torch.arange(n, device=DEV)[None] >= sees[:, None], -math.inf)
            P = torch.softmax(S, dim=-1).nan_to_num(0.0) if n else S
            out[l, b, i0:i1, g * G:(g + 1) * G] = (P @ V).reshape(i1 - i0, G, d)
            got += P.sum(dim=0)
        mass[o:o + n] = c["decay"] * mass[o:o + n] + got
    return {"out": out, "mass": mass, "len": torch.tensor(held, dtype=torch.int32), "k_pool": pools["k"],
            "v_pool": pools["v"]}


def _exact_evict(s, c):
    to = s if c["inplace"] else s["to"]
    got = {name: to[name].clone() for name in ("k_pool", "v_pool", "mass")}
    index, lens = s["index"].clone(), []
    first, dst = s["row_off"].tolist(), to["row_off"].tolist()
    for u, (n, k) in enumerate(zip(_lens(c), _keeps(c))):
        k = min(n, k)
        a = min(c["sinks"], k)
        z = min(c["recent"], k - a)
        m, t = s["mass"][first[u]:first[u] + n].cpu().numpy().astype(np.float64), np.arange(a, n - z)
        mid = t[np.lexsort((t, -m[a:n - z]))][:k - a - z]
        rows = np.sort(np.concatenate((mid, np.arange(a), np.arange(n - z, n))))
        rows = torch.from_numpy(rows).to(DEV)
        for name in got:
            got[name][dst[u]:dst[u] + k] = s[name][first[u] + rows]
        index[u, :k] = rows.int()
        lens.append(k)
    return got | {"index": index, "len": torch.tensor(lens, dtype=torch.int32)}


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    return (_exact_attend if kind == "attend" else _exact_evict if kind == "evict" else _exact_norm)(s, case)
