"""The operators next to the linear layers in a training step, as their speed is watched: layer norm with the
residual add in front of it (forward and backward), and the update of the two-dimensional weights by
orthogonalised momentum (the update itself, and its application to the master weights).

`listed()` names the cases, `draw()` gives further ones of the same ranges, `prepare()` makes what a program
holds before a pass, `run()` is one pass, `exact()` the same results in 64 bits, `work()` the bytes and flops
that a pass cannot do without. `own` says whether `run()` computes with elementary operations in 32 bits or
calls this repository's kernels.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda"
F32, BF16 = torch.float32, torch.bfloat16
TYPES = {"f32": F32, "bf16": BF16}
EPS = 1e-5                                    # layer norm
MU, STEPS, NS, NS_EPS = 0.95, 5, (3.4445, -4.7750, 2.0315), 1e-7
STEP, DECAY = 0.02, 1.0 - 0.02 * 0.1          # learning rate 0.02, weight decay 0.1
MOST_ROWS, MOST_ELEMS = 16384, 16384 * 2048   # of a layer norm
MOST_MUON = 12 * 3072 * 768                   # elements of a group of matrices


def listed():
    return [
        # Eight sequences continued by one token each: the smallest call, no statistics kept.
        {"name": "norm_generate_8", "kind": "norm", "rows": 8, "C": 768, "stream": "bf16", "branch": True, "train": False},
        # A ragged batch of no round width, the residual stream in 32 bits.
        {"name": "norm_odd_1003_f32", "kind": "norm", "rows": 1003, "C": 776, "stream": "f32", "branch": True, "train": True},
        # The model's norm between attn_proj and fc at the training batch, B=16, T=1024.
        {"name": "norm_16384", "kind": "norm", "rows": 16384, "C": 768, "stream": "bf16", "branch": True, "train": True},
        # Its backward on one sequence, the last norm of the model: no gradient comes down the stream.
        {"name": "norm_bwd_1024", "kind": "norm_bwd", "rows": 1024, "C": 768, "stream": "bf16", "dres": False, "accumulate": False},
        # Its backward at the training batch, added to the gradients of earlier micro-steps.
        {"name": "norm_bwd_16384", "kind": "norm_bwd", "rows": 16384, "C": 768, "stream": "bf16", "dres": True, "accumulate": True},
        # A wide model's backward, the residual stream and its gradient in 32 bits.
        {"name": "norm_bwd_wide_f32", "kind": "norm_bwd", "rows": 5001, "C": 4096, "stream": "f32", "dres": True, "accumulate": False},
        # One attn_proj weight alone: a chain of short products.
        {"name": "muon_one_768", "kind": "muon", "n": 1, "R": 768, "C": 768, "grad": "f32", "nesterov": True},
        # Three wide matrices of no round size, gradients in 16 bits.
        {"name": "muon_odd_776x1416", "kind": "muon", "n": 3, "R": 776, "C": 1416, "grad": "bf16", "nesterov": False},
        # The attn_proj weights of the twelve blocks.
        {"name": "muon_attn_proj_12", "kind": "muon", "n": 12, "R": 768, "C": 768, "grad": "f32", "nesterov": True},
        # The fc weights of the twelve blocks.
        {"name": "muon_fc_12", "kind": "muon", "n": 12, "R": 3072, "C": 768, "grad": "f32", "nesterov": True},
        # The update of one odd weight, and of the qkv weights of the twelve blocks, applied.
        {"name": "apply_odd_776x1416", "kind": "apply", "n": 1, "R": 776, "C": 1416, "copy": True},
        {"name": "apply_qkv_12", "kind": "apply", "n": 12, "R": 2304, "C": 768, "copy": True},
    ]


def _log(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return max(lo, min(hi, int(round(v / step)) * step))


def draw(rng):
    kind = rng.choice(["norm", "norm", "norm_bwd", "norm_bwd", "muon", "muon", "muon", "apply"])
    if kind in ("norm", "norm_bwd"):
        C = _log(rng, 64, 8192, 8)
        rows = _log(rng, 1, min(MOST_ROWS, MOST_ELEMS // C))
        case = {"kind": kind, "rows": rows, "C": C, "stream": rng.choice(["bf16", "bf16", "f32"])}
        if kind == "norm":
            return {**case, "branch": rng.random() < 0.7, "train": rng.random() < 0.8}
        return {**case, "dres": rng.random() < 0.7, "accumulate": rng.random() < 0.5}
    R, C = _log(rng, 64, 2304, 8), _log(rng, 64, 2304, 8)
    most = MOST_MUON // (R * C)
    if kind == "muon":  # no more products than the largest listed case has
        most = min(most, int(_ns_flops(12, 3072, 768) / _ns_flops(1, R, C)))
        return {"kind": kind, "n": rng.randint(1, max(1, min(28, most))), "R": R, "C": C,
                "grad": rng.choice(["f32", "f32", "bf16"]), "nesterov": rng.random() < 0.7}
    return {"kind": kind, "n": rng.randint(1, max(1, min(28, most))), "R": R, "C": C, "copy": rng.random() < 0.8}


# ---------------------------------------------------------------------------------------- states
class _State:
    pass


def _normal(g, shape, std, dtype=F32, mean=0.0):
    return torch.randn(shape, generator=g, device=DEV, dtype=F32).mul_(std).add_(mean).to(dtype)


def _gradient(g, n, R, C, std):
    """Gradients of weight matrices: what all tokens have in common (a few strong directions, falling off)
    over what they have not."""
    r = min(32, R, C)
    u, v = _normal(g, (n, R, r), 1.0), _normal(g, (n, r, C), 1.0)
    fall = torch.arange(1, r + 1, device=DEV, dtype=F32).rsqrt_()
    common = (u * fall) @ v
    return common.mul_(0.3 * std / math.sqrt(sum(1.0 / j for j in range(1, r + 1)))).add_(_normal(g, (n, R, C), std))


def prepare(case, seed):
    s = _State()
    s.case = case
    s.workspace = None
    kind = case["kind"]
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    if kind in ("norm", "norm_bwd"):
        rows, C, t = case["rows"], case["C"], TYPES[case["stream"]]
        s.weight = _normal(g, (C,), 0.2, BF16, mean=1.0)
        # a residual stream: the rows differ in mean and in spread
        s.inp = (_normal(g, (rows, C), 1.0) * (_normal(g, (rows, 1), 0.5).exp_()) + _normal(g, (rows, 1), 0.3)).to(t)
        s.mean = torch.empty(rows, dtype=F32, device=DEV)
        s.rstd = torch.empty(rows, dtype=F32, device=DEV)
        if kind == "norm":
            s.bias = _normal(g, (C,), 0.1, BF16)
            s.branch = _normal(g, (rows, C), 0.5, BF16) if case["branch"] else None
            s.sum = torch.empty((rows, C), dtype=t, device=DEV) if case["branch"] else None
            s.out = torch.empty((rows, C), dtype=BF16, device=DEV)
            if not case["train"]:
                s.mean = s.rstd = None
        else:
            x = s.inp.double()
            s.mean.copy_(x.mean(1))
            s.rstd.copy_(1.0 / (x.var(1, unbiased=False) + EPS).sqrt())
            s.dout = _normal(g, (rows, C), 1e-3, BF16)
            s.dres = _normal(g, (rows, C), 1e-3, t) if case["dres"] else None
            s.dinp = torch.empty((rows, C), dtype=t, device=DEV)
            # the linear below takes its gradient in bf16: a copy of its own where the stream's is in 32 bits
            s.dbranch = torch.empty((rows, C), dtype=BF16, device=DEV) if case["stream"] == "f32" else None
            s.dweight = _normal(g, (C,), 1e-2)
            s.dbias = _normal(g, (C,), 1e-2)
    elif kind == "muon":
        n, R, C = case["n"], case["R"], case["C"]
        s.grad = [t.clone() for t in _gradient(g, n, R, C, 1e-4).to(TYPES[case["grad"]])]
        s.momentum = [t.clone() for t in _gradient(g, n, R, C, 3e-4)]
        s.update = [torch.empty((R, C), dtype=BF16, device=DEV) for _ in range(n)]
    else:
        n, R, C = case["n"], case["R"], case["C"]
        s.master = [_normal(g, (R, C), 0.02) for _ in range(n)]
        s.weight = [m.to(BF16) for m in s.master] if case["copy"] else None
        s.update = [_normal(g, (R, C), 1.0 / math.sqrt(max(R, C)), BF16) for _ in range(n)]
    return s


# ---------------------------------------------------------------------------------------- a pass
_nb = None


def _binding():
    global _nb
    if _nb is None:
        from paper_2609_28568_b200 import binding
        _nb = binding
    return _nb


def _norm(s):
    c = s.case
    if own:
        nb = _binding()
        nb.nb_layernorm_forward(s.out, s.sum, s.mean, s.rstd, s.inp, s.branch, s.weight, s.bias, c["rows"], c["C"], EPS,
                                nb.DTYPE_F32 if c["stream"] == "f32" else nb.DTYPE_BF16)
        return {"out": s.out, "sum": s.sum, "mean": s.mean, "rstd": s.rstd}
    total = s.inp if s.branch is None else (s.inp.float() + s.branch.float()).to(s.inp.dtype)
    x = total.float()
    mean = x.mean(1, keepdim=True)
    d = x - mean
    rstd = 1.0 / ((d * d).mean(1, keepdim=True) + EPS).sqrt()
    out = (d * rstd * s.weight.float() + s.bias.float()).to(BF16)
    train = s.mean is not None
    return {"out": out, "sum": None if s.branch is None else total, "mean": mean.view(-1) if train else None,
            "rstd": rstd.view(-1) if train else None}


def _norm_bwd(s):
    c = s.case
    if own:
        nb = _binding()
        if s.workspace is None:
            s.workspace = torch.empty(nb.nb_layernorm_workspace(c["rows"], c["C"]), dtype=torch.uint8, device=DEV)
        nb.nb_layernorm_backward(s.dinp, s.dbranch, s.dweight, s.dbias, s.dout, s.dres, s.inp, s.mean, s.rstd, s.weight,
                                 c["rows"], c["C"], c["accumulate"],
                                 nb.DTYPE_F32 if c["stream"] == "f32" else nb.DTYPE_BF16, s.workspace, s.workspace.numel())
    else:
        dy, rstd = s.dout.float(), s.rstd[:, None]
        xh = (s.inp.float() - s.mean[:, None]) * rstd
        g = dy * s.weight.float()
        dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
        if s.dres is not None:
            dx = dx + s.dres.float()
        s.dinp = dx.to(s.inp.dtype)
        s.dbranch = None if s.dbranch is None else dx.to(BF16)
        dw, db = (dy * xh).sum(0), dy.sum(0)
        s.dweight, s.dbias = (s.dweight + dw, s.dbias + db) if c["accumulate"] else (dw, db)
    return {"dinp": s.dinp, "dbranch": s.dbranch, "dweight": s.dweight, "dbias": s.dbias}


def _muon(s):
    c = s.case
    if own:
        nb = _binding()
        if s.workspace is None:
            s.workspace = torch.empty(nb.nb_muon_workspace(c["n"], c["R"], c["C"]), dtype=torch.uint8, device=DEV)
        nb.nb_muon_update(s.update, s.momentum, s.grad, c["n"], c["R"], c["C"], MU, c["nesterov"], STEPS, *NS, NS_EPS,
                          nb.DTYPE_F32 if c["grad"] == "f32" else nb.DTYPE_BF16, s.workspace, s.workspace.numel())
        return {"update": s.update, "momentum": s.momentum}
    a, b, k = NS
    grad = torch.stack(s.grad).float()
    m = MU * torch.stack(s.momentum) + grad
    v = grad + MU * m if c["nesterov"] else m
    x = v / ((v * v).sum((1, 2), keepdim=True).sqrt() + NS_EPS)
    tall = c["R"] > c["C"]
    if tall:
        x = x.transpose(1, 2)
    for _ in range(STEPS):
        p = x @ x.transpose(1, 2)
        x = a * x + (b * p + k * (p @ p)) @ x
    if tall:
        x = x.transpose(1, 2)
    s.momentum, s.update = list(m.unbind()), list(x.to(BF16).unbind())
    return {"update": s.update, "momentum": s.momentum}


def _apply(s):
    c = s.case
    if own:
        nb = _binding()
        nb.nb_muon_apply(s.master, s.weight, s.update, c["n"], c["R"] * c["C"], DECAY, STEP)
    else:
        s.master = [DECAY * m - STEP * u.float() for m, u in zip(s.master, s.update)]
        s.weight = [m.to(BF16) for m in s.master] if c["copy"] else None
    return {"master": s.master, "weight": s.weight}


def run(s):
    return {"norm": _norm, "norm_bwd": _norm_bwd, "muon": _muon, "apply": _apply}[s.case["kind"]](s)


# ---------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "norm":
        x = s.inp.double()
        if s.branch is not None:
            x = (x + s.branch.double()).to(s.inp.dtype).double()  # the norm is that of the stored sum
        var, mean = torch.var_mean(x, 1, correction=0)
        rstd = (var + EPS).rsqrt()
        out = torch.addcmul(s.bias.double(), (x - mean[:, None]) * rstd[:, None], s.weight.double())
        total = None if s.branch is None else s.inp.double() + s.branch.double()
        return {"out": out, "sum": total, "mean": mean if case["train"] else None, "rstd": rstd if case["train"] else None}
    if kind == "norm_bwd":
        # through the Jacobian's two projections, written as sums against xh and against ones
        C, dy = case["C"], s.dout.double()
        xh = (s.inp.double() - s.mean.double()[:, None]) * s.rstd.double()[:, None]
        g = dy * s.weight.double()
        along = torch.einsum("rc,rc->r", g, xh) / C
        dx = (g - along[:, None] * xh - g.sum(1)[:, None] / C) * s.rstd.double()[:, None]
        if s.dres is not None:
            dx += s.dres.double()
        dw, db = torch.einsum("rc,rc->c", dy, xh), dy.sum(0)
        if case["accumulate"]:
            dw, db = dw + s.dweight.double(), db + s.dbias.double()
        return {"dinp": dx, "dbranch": None if s.dbranch is None else dx, "dweight": dw, "dbias": db}
    if kind == "muon":
        a, b, k = NS
        updates, momenta = [], []
        for grad, mom in zip(s.grad, s.momentum):
            m = mom.double() * MU + grad.double()
            x = m * MU + grad.double() if case["nesterov"] else m
            x = x / (torch.linalg.matrix_norm(x) + NS_EPS)
            for _ in range(STEPS):  # from the side that has fewer rows or columns
                if case["R"] <= case["C"]:
                    y = torch.mm(x, x.T)
                    x = torch.mm(torch.addmm(b * y, y, y, alpha=k), x).add_(x, alpha=a)
                else:
                    y = torch.mm(x.T, x)
                    x = torch.mm(x, torch.addmm(b * y, y, y, alpha=k)).add_(x, alpha=a)
            updates.append(x)
            momenta.append(m)
        return {"update": updates, "momentum": momenta}
    master = [m.double() * DECAY - u.double() * STEP for m, u in zip(s.master, s.update)]
    return {"master": master, "weight": master if case["copy"] else None}


# ---------------------------------------------------------------------------------------- accounting
def _ns_flops(n, R, C):
    """Of the products alone, with half of those whose result is symmetric. Two steps at a time may be done on the
    smaller side: x x' once, then five products of the small symmetric matrices, then one product with x."""
    m, k = min(R, C), max(R, C)
    one = 3 * m * m * k + m ** 3
    two = min(2 * one, 3 * m * m * k + 5 * m ** 3)
    return n * ((STEPS // 2) * two + (STEPS % 2) * one)


def work(case):
    kind = case["kind"]
    if kind in ("norm", "norm_bwd"):
        rows, C, t = case["rows"], case["C"], 4 if case["stream"] == "f32" else 2
        if kind == "norm":
            b = rows * C * (t + 2 + (2 + t if case["branch"] else 0)) + 4 * C + (8 * rows if case["train"] else 0)
            return {"bytes": b, "flops": 8 * rows * C}
        b = rows * C * (2 + t + t + (t if case["dres"] else 0) + (2 if t == 4 else 0)) + 2 * C + 8 * rows
        b += 8 * C * (2 if case["accumulate"] else 1)
        return {"bytes": b, "flops": 14 * rows * C}
    elems = case["n"] * case["R"] * case["C"]
    if kind == "muon":
        return {"bytes": elems * ((4 if case["grad"] == "f32" else 2) + 8 + 2), "flops": _ns_flops(case["n"], case["R"], case["C"])}
    return {"bytes": elems * (10 + (2 if case["copy"] else 0)), "flops": 3 * elems}
