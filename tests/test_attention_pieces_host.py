"""That the bounds of attention_pieces.py tell one piece of dS from two, without a GPU."""
import pytest
import torch

import attention_pieces as pieces


@pytest.mark.parametrize("T,heads,kv,D", [(200, 3, 3, 64), (333, 6, 2, 40), (700, 4, 1, 128), (90, 2, 2, 96)])
def test_bounds_tell_one_piece_from_two(T, heads, kv, D):
    q, k, v, dout, live = pieces.make(T, heads, kv, D, T, "cpu")
    kk, vv = (t.double().repeat_interleave(heads // kv, 1).transpose(0, 1) for t in (k, v))
    s = pieces.SCALE * q.double().transpose(0, 1) @ kk.mT
    out, lse = (torch.softmax(s, -1) @ vv).transpose(0, 1).bfloat16(), torch.logsumexp(s, -1).float()
    want, tol = pieces.gradients(q, k, v, dout, out, lse, live)
    for one, two, w, t in zip(pieces.gradients(q, k, v, dout, out, lse, live, 1), pieces.gradients(q, k, v, dout, out, lse, live, 2), want, tol):
        assert ((two - w).abs() <= t).all()
        assert ((one - w).abs() > 2 * t).any()
