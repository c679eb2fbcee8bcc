"""Attention and rotary positions from their formulas, in 64 bits, with what the roundings of a computation in 32 and 16 bits may add up to."""
import torch

U16 = torch.finfo(torch.bfloat16).eps / 2   # a rounding to bf16, relative to the value
U32 = torch.finfo(torch.float32).eps / 2
EXP = 2.0 ** -21                            # the exponential's own error, relative (2 ulp of the approximate instruction) and its argument's rounding


def spans(bounds):
    return [(a, b) for a, b in zip(bounds, bounds[1:]) if b > a]


def seen(m, causal, device):
    mask = torch.ones((m, m), dtype=torch.bool, device=device)
    return mask.tril() if causal else mask


def forward(q, k, v, bounds, scale, causal):
    """q [T, H, D], k, v [T, K, D]. Returns out, lse [H, T] and bounds of their errors, per element, before out's own rounding is added
    to it. Rows in no sequence are zeros."""
    T, H, D = q.shape
    G = H // k.shape[1]
    q, k, v = q.double(), k.double(), v.double()
    out, e_out = torch.zeros_like(q), torch.zeros_like(q)
    lse, e_lse = (torch.zeros((H, T), dtype=torch.float64, device=q.device) for _ in range(2))
    for a, b in spans(bounds):
        mask = seen(b - a, causal, q.device)
        for h in range(H):
            qq, kk, vv = q[a:b, h], k[a:b, h // G], v[a:b, h // G]
            s = (scale * qq @ kk.T).masked_fill(~mask, -torch.inf)
            lse[h, a:b] = torch.logsumexp(s, 1)
            p = torch.exp(s - lse[h, a:b, None])
            out[a:b, h] = p @ vv
            # a score: D products and sums in fp32 (the tensor core may cut off instead of rounding: 2 U32 each), its scaling
            e_s = ((2 * D + 4) * U32 * scale * (qq.abs() @ kk.abs().T)).masked_fill(~mask, 0.0).amax(1, keepdim=True)
            e_s = e_s + 4 * U32 * lse[h, a:b, None].abs()
            # each probability: its score, the exponential, the rounding to bf16; sums of up to b - a terms; the same for the sum below
            rel = U16 + 2 * e_s + 2 * EXP + 4 * (b - a + 256) * U32
            e_out[a:b, h] = rel * (p @ vv.abs())
            e_lse[h, a:b] = (e_s + EXP + 2 * (b - a + 256) * U32).squeeze(1) + 4 * U32 * lse[h, a:b].abs()
    return out, lse, e_out + U16 * out.abs() * (1 + U16), e_lse


def backward(dout, out, lse, q, k, v, bounds, scale, causal):
    """(dq, dk, dv) and bounds of their errors, with out and lse as they are given."""
    T, H, D = q.shape
    G = H // k.shape[1]
    dout, out, lse, q, k, v = (t.double() for t in (dout, out, lse, q, k, v))
    dq, dk, dv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    eq, ek, ev = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    for a, b in spans(bounds):
        mask = seen(b - a, causal, q.device)
        for h in range(H):
            qq, kk, vv, do, o = q[a:b, h], k[a:b, h // G], v[a:b, h // G], dout[a:b, h], out[a:b, h]
            p = torch.exp(scale * qq @ kk.T - lse[h, a:b, None]).masked_fill(~mask, 0.0)
            dp, delta = do @ vv.T, (do * o).sum(1, keepdim=True)
            ds = p * (dp - delta)
            e_p = (2 * D + 4) * U32 * scale * (qq.abs() @ kk.abs().T) + 6 * U32 * lse[h, a:b, None].abs() + 2 * EXP  # relative
            e_ds = ds.abs() * (U16 + 2 * e_p) + 1.01 * p * ((2 * D + 4) * U32) * (do.abs() @ vv.abs().T + (do * o).abs().sum(1, keepdim=True) + dp.abs() + delta.abs())
            n = 2 * G * (b - a + 256) * U32  # sums of that many terms
            dv[a:b, h // G] += p.T @ do
            ev[a:b, h // G] += (p * (U16 + 2 * e_p + n)).T @ do.abs()
            dq[a:b, h] = scale * ds @ kk
            eq[a:b, h] = scale * (e_ds + n * ds.abs()) @ kk.abs()
            dk[a:b, h // G] += scale * ds.T @ qq
            ek[a:b, h // G] += scale * (e_ds + n * ds.abs()).T @ qq.abs()
    return (dq, dk, dv), tuple(e + U16 * g.abs() * 1.01 for e, g in ((eq, dq), (ek, dk), (ev, dv)))


def frequencies(R, base, factor=1.0, low=1.0, high=32.0, original=0):
    f = torch.tensor([base ** (-2.0 * j / R) for j in range(R // 2)], dtype=torch.float64)
    if not original:
        return f / factor
    keep = ((original * f / (2 * torch.pi) - low) / (high - low)).clamp(0.0, 1.0)
    return f * (keep + (1.0 - keep) / factor)


def rotary(x, freq, at, scale, half, inverse=False):
    """x [T, heads, D], at [T]. The result, and the bound of its error: angle and its sine and cosine to fp32 (4 U32 of a half turn and of the
    value), two products and a sum, the rounding to bf16."""
    R = 2 * freq.numel()
    angle = at.double()[:, None] * freq.to(x.device) * (-1.0 if inverse else 1.0)
    c, s = (scale * f(angle)[:, None] for f in (torch.cos, torch.sin))
    y = x.double().clone()
    first, second = (slice(0, R // 2), slice(R // 2, R)) if half else (slice(0, R, 2), slice(1, R, 2))
    a, b = x.double()[..., first], x.double()[..., second]
    y[..., first], y[..., second] = a * c - b * s, b * c + a * s
    tol = U16 * y.abs() * 1.01
    for part in (first, second):
        tol[..., part] += 20 * U32 * abs(scale) * (a.abs() + b.abs())
    tol[..., R:] = 0.0
    return y, tol
