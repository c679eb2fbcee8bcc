"""Data on which the second piece of dS shows: what the keys (the queries) have in common cancels in dQ (in dK) where dS itself does, but not where its
rounding to one piece does. The few rows that matter lie anywhere in a long sequence; all others are exact zeros, so that no sum of many terms widens the bounds.

Of LIVE queries three at a time are the same, with dout a, b and -(a + b), numbers of few bits: their dS add up to zero for each key. The other queries have dout 0.
LIVE keys have COMMON in a column where queries have 0; the other keys have a score 400 lower, whose probability is 0 in 32 bits. Queries have COMMON in
a column where keys have 0."""
import torch

from attention_reference import EXP, U16, U32

LIVE, COMMON, SCALE = 15, 64.0, 0.125


def make(T, heads, kv, D, seed, device):
    """q, k, v, dout of one sequence [T, ., D] in bf16, and the live rows."""
    g = torch.Generator().manual_seed(seed)
    live = torch.arange(LIVE) * T // LIVE + T // (2 * LIVE)
    draw = lambda *shape: torch.randn(shape, generator=g)  # noqa: E731
    q, k, v = draw(T, heads, D) * 0.5, draw(T, kv, D) * 0.5, draw(T, kv, D)
    q[live] = draw(LIVE // 3, heads, D).repeat_interleave(3, 0) * 0.5
    q[..., 0], q[..., 1], q[..., 2] = 0.0, COMMON, 8.0
    dead = torch.ones(T, dtype=torch.bool)
    dead[live] = False
    k[..., 0], k[..., 1], k[..., 2] = COMMON, 0.0, 0.0
    k[dead, :, 2] = -400.0
    dout = torch.zeros(T, heads, D)
    a, b = (torch.randint(-16, 17, (LIVE // 3, heads, D), generator=g) / 8 for _ in range(2))
    dout[live] = torch.stack((a, b, -(a + b)), 1).flatten(0, 1)
    return *(t.to(torch.bfloat16).to(device) for t in (q, k, v, dout)), live.to(device)


def gradients(q, k, v, dout, out, lse, live, pieces=None):
    """dq and dk of the live rows, of a sequence that sees itself whole: from their formulas in 64 bits, with bounds of a kernel's errors that has dS in two pieces;
    or with dS rounded to so many pieces of bf16."""
    G = q.shape[1] // k.shape[1]
    q, k, v, dout, out = (t[live].double().transpose(0, 1) for t in (q, k, v, dout, out))
    k, v = (t.repeat_interleave(G, 0) for t in (k, v))
    lse, D = lse[:, live].double()[..., None], q.shape[-1]
    p = torch.exp(SCALE * q @ k.mT - lse)
    dp, delta = dout @ v.mT, (dout * out).sum(-1, keepdim=True)
    ds = p * (dp - delta)
    shared = lambda t: t.unflatten(0, (-1, G)).sum(1)  # noqa: E731
    if pieces:
        first = ds.float().bfloat16()
        rounded = first.double() if pieces == 1 else first.double() + (ds.float() - first.float()).bfloat16().double()
        return SCALE * rounded @ k, shared(SCALE * rounded.mT @ q)
    # relative of p; dS with what two roundings leave of it; sums of two terms to each live row (the rows' zeros are added without an error), twice for
    # a tensor core that cuts off
    e_p = (2 * D + 4) * U32 * SCALE * (q.abs() @ k.abs().mT) + 6 * U32 * lse.abs() + 2 * EXP
    e_ds = ds.abs() * (1.01 * U16 ** 2 + 2 * e_p) + 1.01 * p * ((2 * D + 4) * U32) * (dout.abs() @ v.abs().mT + (dout * out).abs().sum(-1, keepdim=True) + dp.abs() + delta.abs())
    e_ds = e_ds + 2 * (2 * LIVE * G + 16) * U32 * ds.abs()
    want = SCALE * ds @ k, shared(SCALE * ds.mT @ q)
    tol = SCALE * e_ds @ k.abs(), shared(SCALE * e_ds.mT @ q.abs())
    return want, tuple(t + 1.01 * U16 * w.abs() + 1e-30 for t, w in zip(tol, want))
