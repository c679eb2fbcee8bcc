"""Gradients where some keys have a score of -infinity: they have no part in a row, and neither value nor key gets a gradient, whatever the length of the sequence
(past its last row a tile is filled with queries of zeros, for which such a key's score is not a number)."""
import math

import pytest
import torch

from paper_2609_28568_b200 import binding as nb
import attention_reference as ref
from test_gpu_attention import rand

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _status_clean():
    yield
    nb.nb_check_status()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("T,heads,kv,D", [(200, 2, 1, 64), (201, 1, 1, 128), (131, 230, 230, 64), (130, 230, 230, 96), (15, 1, 1, 40), (1, 1, 1, 64), (700, 8, 1, 64), (2007, 1, 1, 128),
                                          (208, 2, 2, 64)])
def test_keys_without_a_part(T, heads, kv, D, causal):
    q, k, v, dout = rand(1, (T, heads, D)), rand(2, (T, kv, D)), rand(3, (T, kv, D)), rand(4, (T, heads, D), 0.1)
    q[..., 0] = 1.0
    here = torch.arange(T, device="cuda") % 3 != 1  # the first key among them
    k[~here, :, 0] = -math.inf
    out, lse = nb.attention_forward(q, k, v, causal=causal)
    _, dk, dv = nb.attention_backward(dout, out, lse, q, k, v, causal=causal)
    G, scale = heads // kv, torch.tensor(D ** -0.5, dtype=torch.float32).double().item()
    hidden = ~here | (ref.seen(T, causal, "cuda") == 0)
    qq, do, oo = (t.double().transpose(0, 1) for t in (q, dout, out))
    kk, vv = (t.double().masked_fill(~here[:, None, None], 0.0).transpose(0, 1).repeat_interleave(G, 0) for t in (k, v))
    s = (scale * qq @ kk.mT).masked_fill(hidden, -math.inf)
    p = torch.exp(s - lse.double()[..., None])
    ds = p * (do @ vv.mT - (do * oo).sum(-1, keepdim=True))
    shared = lambda t: t.unflatten(0, (kv, G)).sum(1).transpose(0, 1)  # noqa: E731
    # p and ds: a rounding to bf16 at most, and three tenths of one (1.17e-3) for what is computed in 32 bits: a score's 2 D operations, 4e-5 of p at most, twice, and sums
    # of G (T + 256) terms, 9e-4 of them at most; the result's own rounding. ds besides: what 32 bits leave of the difference, 2 D products and as many sums each
    left = p * (4 * D * ref.U32) * (do.abs() @ vv.abs().mT + (do * oo).abs().sum(-1, keepdim=True))
    for got, want, tol, name in ((dv, shared(p.mT @ do), shared(p.mT @ do.abs()), "dv"),
                                 (dk, scale * shared(ds.mT @ qq), scale * shared((ds.abs() + left / ref.U16).mT @ qq.abs()), "dk")):
        err = (got.double() - want).abs()
        assert torch.isfinite(got[here]).all() and (got[~here] == 0).all(), name
        assert (err <= 1.3 * ref.U16 * (tol + want.abs()) + 1e-30).all(), name
