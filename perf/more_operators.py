"""The operators between the qkv linear and attn_proj, as their speed is watched: rotary positions of queries and
keys, and attention over packed sequences, forward and backward.

`listed()` names the cases, `draw()` gives further ones of the same ranges, `prepare()` makes what a program
holds before a pass, `run()` is one pass, `exact()` the same results in 64 bits, `work()` the bytes and flops
that a pass cannot do without. `own` says whether `run()` computes with elementary operations in 32 bits (angles
in 64) or calls this repository's kernels.

A case's rows are `n` sequences one after the other and `pad` rows behind the last one, which belong to nothing and
hold NaN, as memory may that nobody wrote; outputs keep what they held there. The sequences' lengths are equal, or
follow from the number `cut`.
"""
from __future__ import annotations

import math
import random

import torch

own = False
DEV = "cuda"
F32, F64, BF16 = torch.float32, torch.float64, torch.bfloat16
BASE = 1.0e6                                   # of the rotary frequencies
SCALED = dict(factor=4.0, low=1.0, high=32.0, original=8192)   # frequencies for a context four times as long
MOST_PAIRS = 16 * 128 * 16384 * 16385 // 2     # of queries and keys, times heads and their width, in a forward pass
MOST_BACK = 16 * 128 * 8192 * 8193 // 2        # the same in a backward pass
MOST_ROTARY = 16384 * 24 * 128                 # elements of queries and keys


def listed():
    return [
        # Eight sequences continued by one token each, at positions of a long context: the smallest call.
        {"name": "rotary_generate_8", "kind": "rotary", "rows": 8, "n": 8, "pad": 0, "cut": 0, "far": 32768, "heads": 16, "kv": 8, "D": 128,
         "R": 128, "pairs": "half", "scaled": False, "inverse": False, "fused": True},
        # Packed sequences of different lengths, part of a head of no round width, neighbours as pairs, a scaled context; the gradient's way back.
        {"name": "rotary_odd_1003", "kind": "rotary", "rows": 1003, "n": 7, "pad": 21, "cut": 5, "far": 0, "heads": 9, "kv": 3, "D": 80,
         "R": 32, "pairs": "neighbours", "scaled": True, "inverse": True, "fused": False},
        # Queries and keys of the adapter stage's batch: eight sequences of 2048, 16 heads on 8.
        {"name": "rotary_16384", "kind": "rotary", "rows": 16384, "n": 8, "pad": 0, "cut": 0, "far": 0, "heads": 16, "kv": 8, "D": 128,
         "R": 128, "pairs": "half", "scaled": False, "inverse": False, "fused": False},
        # A short prompt alone, no statistics kept: a chain of latencies.
        {"name": "attn_prompt_37", "kind": "attn", "rows": 37, "n": 1, "pad": 0, "cut": 0, "heads": 12, "kv": 12, "D": 64, "causal": True,
         "fused": True, "train": False},
        # The 124M model's training batch, B=16, T=1024: twelve heads of 64 out of the fused qkv activation.
        {"name": "attn_16x1024", "kind": "attn", "rows": 16384, "n": 16, "pad": 0, "cut": 0, "heads": 12, "kv": 12, "D": 64, "causal": True,
         "fused": True, "train": True},
        # Documents of different lengths packed into one batch, two queries' heads to a key's, rows left over.
        {"name": "attn_packed_8000", "kind": "attn", "rows": 8000, "n": 23, "pad": 192, "cut": 3, "heads": 16, "kv": 8, "D": 128,
         "causal": True, "fused": False, "train": True},
        # Sequences that see themselves whole (a scorer or an encoder), heads of no round width.
        {"name": "attn_whole_80", "kind": "attn", "rows": 4593, "n": 3, "pad": 0, "cut": 0, "heads": 7, "kv": 7, "D": 80, "causal": False,
         "fused": True, "train": True},
        # One long sequence of the adapter model's heads: the largest.
        {"name": "attn_long_16384", "kind": "attn", "rows": 16384, "n": 1, "pad": 0, "cut": 0, "heads": 16, "kv": 8, "D": 128, "causal": True,
         "fused": False, "train": True},
        # The way back through a short sequence.
        {"name": "attn_bwd_200", "kind": "attn_bwd", "rows": 200, "n": 1, "pad": 0, "cut": 0, "heads": 12, "kv": 12, "D": 64, "causal": True,
         "fused": True},
        # Through the training batch, gradients into one fused buffer, as the qkv linear's backward takes it.
        {"name": "attn_bwd_16x1024", "kind": "attn_bwd", "rows": 16384, "n": 16, "pad": 0, "cut": 0, "heads": 12, "kv": 12, "D": 64,
         "causal": True, "fused": True},
        # Through packed documents: a key's gradients are sums over the queries' heads that share it.
        {"name": "attn_bwd_packed_8000", "kind": "attn_bwd", "rows": 8000, "n": 23, "pad": 192, "cut": 3, "heads": 16, "kv": 8, "D": 128,
         "causal": True, "fused": False},
        # Through one long sequence.
        {"name": "attn_bwd_long_8192", "kind": "attn_bwd", "rows": 8192, "n": 1, "pad": 0, "cut": 0, "heads": 16, "kv": 8, "D": 128,
         "causal": True, "fused": False},
    ]


def _log(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / step)) * step))


def draw(rng):
    kind = rng.choice(["rotary", "attn", "attn", "attn_bwd", "attn_bwd"])
    kv = rng.choice([1, 2, 3, 4, 8, 12])
    heads = kv * rng.choice([g for g in (1, 1, 2, 4, 8) if kv * g <= 16])
    D = rng.choice([64, 64, 128, 128, rng.randrange(16, 129, 8)])
    rows = _log(rng, 1, 16384)
    case = {"kind": kind, "rows": rows, "n": _log(rng, 1, max(1, min(64, rows // 2))), "pad": rng.choice([0, 0, rng.randint(1, 300)]),
            "cut": rng.randint(1, 10 ** 6), "heads": heads, "kv": kv, "D": D, "fused": rng.random() < 0.5}
    if kind == "rotary":
        pairs = rng.choice(["half", "half", "neighbours"])
        whole = D // 16 * 16 if pairs == "half" else D
        case.update(R=rng.choice([whole, whole, rng.randrange(16, whole + 1, 16)]), pairs=pairs, scaled=rng.random() < 0.4,
                    inverse=rng.random() < 0.4, far=rng.choice([0, 0, 32768]))
        return case
    case["causal"] = rng.random() < 0.8
    if kind == "attn":
        case["train"] = rng.random() < 0.8
    while _products(case) > (MOST_BACK if kind == "attn_bwd" else MOST_PAIRS):
        case["rows"] = case["rows"] * 3 // 4
    case["n"] = min(case["n"], case["rows"])
    return case


# ---------------------------------------------------------------------------------------- sequences
def lengths(case):
    """The sequences' lengths: equal ones, or cut at random places (with short and empty ones among them)."""
    rows, n = case["rows"], case["n"]
    if not case["cut"]:
        return [rows // n] * n
    rng = random.Random(case["cut"])
    share = [rng.expovariate(1.0) ** 1.5 for _ in range(n)]
    at = [round(rows * sum(share[:i]) / sum(share)) for i in range(n)] + [rows]
    return [b - a for a, b in zip(at, at[1:])]


def _spans(case):
    at = 0
    for m in lengths(case):
        if m:
            yield at, at + m
        at += m


def _products(case):
    """Pairs of a query and a key that it sees, times heads and their width."""
    seen = sum(m * (m + 1) // 2 if case["causal"] else m * m for m in lengths(case))
    return seen * case["heads"] * case["D"]


# ---------------------------------------------------------------------------------------- states
class _State:
    pass


def _normal(g, shape, std, dtype=F32):
    return torch.randn(shape, generator=g, device=DEV, dtype=F32).mul_(std).to(dtype)


def _rows(case):
    return case["rows"] + case["pad"]


def _columns(case, names, fill=0.0):
    """Tensors [rows, heads, D] by name (q: all heads, else the keys' heads): slices of one buffer where the case is fused."""
    T, D = _rows(case), case["D"]
    count = [case["heads"] if n == "q" else case["kv"] for n in names]
    if case["fused"]:
        whole = torch.full((T, sum(count) * D), fill, dtype=BF16, device=DEV)
        parts = whole.split([c * D for c in count], 1)
    else:
        parts = [torch.full((T, c * D), fill, dtype=BF16, device=DEV) for c in count]
    return [p.unflatten(1, (c, D)) for p, c in zip(parts, count)]


def _queries_keys(g, case):
    """Queries and keys as models have them: heads differ in how sharp they are, and keys share a direction."""
    rows, H, K, D = case["rows"], case["heads"], case["kv"], case["D"]
    q = _normal(g, (rows, H, D), 1.0) * torch.rand((1, H, 1), generator=g, device=DEV).mul_(2.0).add_(0.5) + _normal(g, (1, H, D), 0.3)
    k = _normal(g, (rows, K, D), 1.0) + _normal(g, (1, K, D), 0.5)
    return q, k


def prepare(case, seed):
    s = _State()
    s.case = case
    s.workspace = None
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    rows, T, H, D = case["rows"], _rows(case), case["heads"], case["D"]
    bounds = [0]
    for m in lengths(case):
        bounds.append(bounds[-1] + m)
    s.bounds = torch.tensor(bounds, dtype=torch.int32, device=DEV)
    if case["kind"] == "rotary":
        s.q, s.k = _columns(case, "qk", math.nan)
        for t, x in zip((s.q, s.k), _queries_keys(g, case)):
            t[:rows] = x.to(BF16)
        s.q_out, s.k_out = _columns(case, "qk")
        s.scale = 0.1 * math.log(SCALED["factor"]) + 1.0 if case["scaled"] else 1.0
        s.positions = torch.randint(0, case["far"], (T,), generator=g, device=DEV, dtype=torch.int32) if case["far"] else None
        s.freq = frequencies(case).to(DEV)
        return s
    s.scale = 1.0 / math.sqrt(D)
    s.q, s.k, s.v = _columns(case, "qkv", math.nan)
    q, k = _queries_keys(g, case)
    s.q[:rows], s.k[:rows] = q.to(BF16), k.to(BF16)
    s.v[:rows] = _normal(g, (rows, case["kv"], D), 1.0, BF16)
    s.out = torch.zeros((T, H, D), dtype=BF16, device=DEV)
    s.lse = torch.zeros((H, T), dtype=F32, device=DEV)
    if case["kind"] == "attn_bwd":
        s.out, s.lse = _attend(s)
        s.out[rows:] = math.nan
        s.dout = torch.full((T, H, D), math.nan, dtype=BF16, device=DEV)
        s.dout[:rows] = _normal(g, (rows, H, D), 1e-3, BF16)
        s.dq, s.dk, s.dv = _columns(case, "qkv")
    elif not case["train"]:
        s.lse = None
    return s


def frequencies(case):
    """Radians per position of each pair, in 64 bits. Scaled: pairs that turn fewer than `low` times over the original context are
    slowed by `factor`, those that turn more than `high` times stay, with a straight line between."""
    R = case["R"]
    f = BASE ** (-torch.arange(0, R, 2, dtype=F64) / R)
    if case["scaled"]:
        turns = SCALED["original"] * f / (2.0 * math.pi)
        keep = ((turns - SCALED["low"]) / (SCALED["high"] - SCALED["low"])).clamp(0.0, 1.0)
        f = f * (keep + (1.0 - keep) / SCALED["factor"])
    return f


# ---------------------------------------------------------------------------------------- a pass
_nb = None


def _binding():
    global _nb
    if _nb is None:
        from paper_2609_28568_b200 import binding
        _nb = binding
    return _nb


def _rotary(s):
    c = s.case
    T, rows, R = _rows(c), c["rows"], c["R"]
    if own:
        nb = _binding()
        nb.nb_rotary(s.q_out, s.k_out, s.q, s.k, s.freq, s.positions, s.bounds, T, c["n"], c["heads"], c["kv"], c["D"], R,
                     s.q_out.stride(0), s.k_out.stride(0), s.q.stride(0), s.k.stride(0), s.scale,
                     nb.ROTARY_HALF if c["pairs"] == "half" else nb.ROTARY_NEIGHBOURS, c["inverse"])
        return {"q": s.q_out, "k": s.k_out}
    if s.positions is None:
        at = torch.arange(rows, device=DEV, dtype=torch.int32)
        at = at - s.bounds[torch.searchsorted(s.bounds, at, right=True) - 1]
    else:
        at = s.positions[:rows]
    angle = at.double()[:, None] * s.freq
    cos, sin = ((s.scale * f(angle)).float()[:, None] for f in (torch.cos, torch.sin))
    if c["inverse"]:
        sin = -sin
    out = []
    for t in (s.q, s.k):
        x = t[:rows].float()
        turn, rest = x[..., :R], x[..., R:]
        a, b = (turn[..., :R // 2], turn[..., R // 2:]) if c["pairs"] == "half" else (turn[..., 0::2], turn[..., 1::2])
        a, b = a * cos - b * sin, b * cos + a * sin
        turn = torch.cat((a, b), -1) if c["pairs"] == "half" else torch.stack((a, b), -1).flatten(-2)
        y = torch.zeros((T, *t.shape[1:]), dtype=BF16, device=DEV)
        y[:rows] = torch.cat((turn, rest), -1).to(BF16)
        out.append(y)
    return {"q": out[0], "k": out[1]}


def _head_groups(case, m):
    """Heads in groups that share keys and whose scores stay within 2 GB."""
    group = case["heads"] // case["kv"]
    step = max(1, (1 << 29) // (m * m * group))
    for i in range(0, case["kv"], step):
        yield i, min(i + step, case["kv"])


def _mask(case, m):
    return torch.ones((m, m), dtype=torch.bool, device=DEV).tril() if case["causal"] else None


def _attend(s):
    c = s.case
    H, K, D = c["heads"], c["kv"], c["D"]
    G = H // K
    out, lse = torch.zeros((_rows(c), H, D), dtype=BF16, device=DEV), torch.zeros((H, _rows(c)), dtype=F32, device=DEV)
    for a, b in _spans(c):
        seen = _mask(c, b - a)
        for i, j in _head_groups(c, b - a):
            q = s.q[a:b, i * G:j * G].float().unflatten(1, (j - i, G)).permute(1, 2, 0, 3)
            k, v = (t[a:b, i:j].float().permute(1, 0, 2)[:, None] for t in (s.k, s.v))
            x = (q @ k.transpose(-1, -2)) * s.scale
            if seen is not None:
                x = x.masked_fill_(~seen, -math.inf)
            top = x.amax(-1, keepdim=True)
            p = (x - top).exp_()
            total = p.sum(-1, keepdim=True)
            o = (p @ v) / total
            out[a:b, i * G:j * G] = o.permute(2, 0, 1, 3).flatten(1, 2).to(BF16)
            lse[i * G:j * G, a:b] = (top + total.log()).flatten(0, 1).squeeze(-1)
    return out, lse


def _attn(s):
    c = s.case
    if own:
        _binding().nb_attention_forward(s.out, s.lse, s.q, s.k, s.v, s.bounds, _rows(c), c["n"], c["heads"], c["kv"], c["D"], s.out.stride(0),
                                        s.q.stride(0), s.k.stride(0), s.v.stride(0), s.scale, c["causal"])
        return {"out": s.out, "lse": s.lse}
    out, lse = _attend(s)
    return {"out": out, "lse": lse if c["train"] else None}


def _attn_bwd(s):
    c = s.case
    if own:
        nb = _binding()
        if s.workspace is None:
            s.workspace = torch.empty(nb.nb_attention_workspace(_rows(c), c["heads"]), dtype=torch.uint8, device=DEV)
        nb.nb_attention_backward(s.dq, s.dk, s.dv, s.dout, s.out, s.lse, s.q, s.k, s.v, s.bounds, _rows(c), c["n"], c["heads"], c["kv"],
                                 c["D"], s.dq.stride(0), s.dk.stride(0), s.dv.stride(0), s.dout.stride(0), s.out.stride(0), s.q.stride(0),
                                 s.k.stride(0), s.v.stride(0), s.scale, c["causal"], s.workspace, s.workspace.numel())
        return {"dq": s.dq, "dk": s.dk, "dv": s.dv}
    H, K, D, T = c["heads"], c["kv"], c["D"], _rows(c)
    G = H // K
    dq = torch.zeros((T, H, D), dtype=BF16, device=DEV)
    dk, dv = (torch.zeros((T, K, D), dtype=BF16, device=DEV) for _ in range(2))
    for a, b in _spans(c):
        seen = _mask(c, b - a)
        for i, j in _head_groups(c, b - a):
            q, do, o = (t[a:b, i * G:j * G].float().unflatten(1, (j - i, G)).permute(1, 2, 0, 3) for t in (s.q, s.dout, s.out))
            k, v = (t[a:b, i:j].float().permute(1, 0, 2)[:, None] for t in (s.k, s.v))
            p = ((q @ k.transpose(-1, -2)) * s.scale - s.lse[i * G:j * G, a:b].unflatten(0, (j - i, G))[..., None]).exp_()
            if seen is not None:
                p = p.masked_fill_(~seen, 0.0)
            delta = (do * o).sum(-1, keepdim=True)
            dv[a:b, i:j] = (p.transpose(-1, -2) @ do).sum(1).permute(1, 0, 2).to(BF16)
            ds = p * (do @ v.transpose(-1, -2) - delta) * s.scale
            dq[a:b, i * G:j * G] = (ds @ k).permute(2, 0, 1, 3).flatten(1, 2).to(BF16)
            dk[a:b, i:j] = (ds.transpose(-1, -2) @ q).sum(1).permute(1, 0, 2).to(BF16)
    return {"dq": dq, "dk": dk, "dv": dv}


def run(s):
    return {"rotary": _rotary, "attn": _attn, "attn_bwd": _attn_bwd}[s.case["kind"]](s)


# ---------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    rows, T, H, K, D = case["rows"], _rows(case), case["heads"], case["kv"], case["D"]
    if case["kind"] == "rotary":
        # pairs as complex numbers, turned by one multiplication
        at = torch.cat([torch.arange(m, device=DEV) for m in lengths(case)]) if s.positions is None else s.positions[:rows]
        R = case["R"]
        f = torch.pow(torch.tensor(BASE, dtype=F64, device=DEV), -2.0 * torch.arange(R // 2, dtype=F64, device=DEV) / R)
        if case["scaled"]:
            ramp = (SCALED["original"] / (2.0 * math.pi) * f - SCALED["low"]) / (SCALED["high"] - SCALED["low"])
            f = torch.lerp(f / SCALED["factor"], f, ramp.clamp(0.0, 1.0))
        angle = torch.outer(at.double(), f)
        turn = torch.polar(torch.full_like(angle, s.scale), -angle if case["inverse"] else angle)[:, None]
        out = []
        for t in (s.q, s.k):
            y = torch.zeros(t.shape, dtype=F64, device=DEV)
            y[:rows] = t[:rows].double()
            first, second = (slice(0, R // 2), slice(R // 2, R)) if case["pairs"] == "half" else (slice(0, R, 2), slice(1, R, 2))
            z = torch.complex(y[:rows, :, first], y[:rows, :, second]) * turn
            y[:rows, :, first], y[:rows, :, second] = z.real, z.imag
            out.append(y)
        return {"q": out[0], "k": out[1]}
    G = H // K
    back = case["kind"] == "attn_bwd"
    out, lse = torch.zeros((T, H, D), dtype=F64, device=DEV), torch.zeros((H, T), dtype=F64, device=DEV)
    dq, dk, dv = (torch.zeros((T, h, D), dtype=F64, device=DEV) for h in (H, K, K))
    for a, b in _spans(case):
        below = torch.triu(torch.full((b - a, b - a), -math.inf, dtype=F64, device=DEV), 1) if case["causal"] else None
        for h in range(H):
            q, k, v = s.q[a:b, h].double(), s.k[a:b, h // G].double(), s.v[a:b, h // G].double()
            x = torch.mm(q * s.scale, k.T)
            if below is not None:
                x += below
            if not back:
                lse[h, a:b] = torch.logsumexp(x, 1)
                out[a:b, h] = torch.softmax(x, 1) @ v
                continue
            do = s.dout[a:b, h].double()
            p = torch.exp(x.sub_(s.lse[h, a:b].double()[:, None]))
            dv[a:b, h // G] += torch.mm(p.T, do)
            p *= torch.mm(do, v.T).sub_(torch.einsum("rd,rd->r", do, s.out[a:b, h].double())[:, None])
            dq[a:b, h] = torch.mm(p, k) * s.scale
            dk[a:b, h // G] += torch.mm(p.T, q) * s.scale
    if back:
        return {"dq": dq, "dk": dk, "dv": dv}
    return {"out": out, "lse": lse if case["train"] else None}


# ---------------------------------------------------------------------------------------- accounting
def work(case):
    rows, H, K, D = case["rows"], case["heads"], case["kv"], case["D"]
    if case["kind"] == "rotary":
        return {"bytes": 4 * rows * (H + K) * D + 4 * case["R"] + (4 * rows if case["far"] else 0), "flops": 3 * rows * (H + K) * case["R"]}
    if case["kind"] == "attn":
        return {"bytes": 2 * rows * (2 * H + 2 * K) * D + (4 * rows * H if case["train"] else 0), "flops": 4 * _products(case)}
    return {"bytes": 2 * rows * (4 * H + 4 * K) * D + 4 * rows * H, "flops": 10 * _products(case)}
