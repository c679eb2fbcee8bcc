"""dS of the backward pass of attention keeps its second piece, in every form of both passes."""
import pytest
import torch

from paper_2609_28568_b200 import binding as nb
import attention_pieces as pieces

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _status_clean():
    yield
    nb.nb_check_status()


# few items: two warpgroups; shared items (dq by 2 and 4 blocks, dk and dv by 4 and 8); narrow heads in a full batch: one warpgroup
@pytest.mark.parametrize("T,heads,kv,D", [(200, 3, 3, 64), (333, 6, 2, 40), (700, 8, 1, 64), (2000, 1, 1, 128), (4100, 1, 1, 64), (1024, 60, 60, 64), (600, 128, 128, 24),
                                          (600, 60, 60, 128), (500, 8, 4, 96)])
def test_second_piece(T, heads, kv, D):
    q, k, v, dout, live = pieces.make(T, heads, kv, D, T, "cuda")
    out, lse = nb.attention_forward(q, k, v, scale=pieces.SCALE, causal=False)
    grads = nb.attention_backward(dout, out, lse, q, k, v, scale=pieces.SCALE, causal=False)
    want, tol = pieces.gradients(q, k, v, dout, out, lse, live)
    for got, w, t, name in zip(grads, want, tol, ("dq", "dk")):
        err = (got[live].double().transpose(0, 1) - w).abs()
        assert (err <= t).all(), (name, (err / t).max().item())
