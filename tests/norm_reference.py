"""Layer norm and the orthogonalised update from their formulas, in 64 bits."""
import torch

EPS32 = torch.finfo(torch.float32).eps


def norm_forward(s, w, b, eps):
    """s [rows, C], w [C], b [C] or None, all in 64 bits."""
    mean = s.mean(1, keepdim=True)
    d = s - mean
    rstd = 1.0 / torch.sqrt((d * d).mean(1, keepdim=True) + eps)
    out = d * rstd * w
    return {"mean": mean, "rstd": rstd, "xh": d * rstd, "out": out if b is None else out + b}


def norm_backward(dout, s, mean, rstd, w, dres):
    xh = (s - mean) * rstd
    g = dout * w
    dinp = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    return {"xh": xh, "g": g, "dinp": dinp if dres is None else dinp + dres, "dweight": (dout * xh).sum(0), "dbias": dout.sum(0)}


def newton_schulz(v, steps, coefficients, eps):
    """One matrix: v / (|v| + eps), then steps of x <- a x + (b y + c y y) x with y = x x^T."""
    a, b, c = coefficients
    x = v / (v.square().sum().sqrt() + eps)
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    for _ in range(steps):
        y = x @ x.T
        x = a * x + (b * y + c * (y @ y)) @ x
    return x.T if tall else x
