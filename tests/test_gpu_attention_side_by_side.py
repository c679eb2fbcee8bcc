"""Passes of the backward pass that run side by side, on inputs that change from step to step in the same memory: the pass that starts early sees this step's."""
import pytest
import torch

from paper_2609_28568_b200 import binding as nb
from test_gpu_attention import BF16, DEV, F32, Case

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _status_clean():
    yield
    nb.nb_check_status()


@pytest.mark.parametrize("lengths,heads,kv,D", [([1], 12, 12, 64), ([200], 12, 12, 64), ([1000], 8, 1, 64), ([1000], 4, 4, 128), ([2000], 2, 1, 128), ([500, 3, 430], 6, 2, 40)])
def test_inputs_of_this_step(lengths, heads, kv, D):
    sets = [Case(lengths, heads, kv, D, seed=s) for s in (3, 4, 5)]
    c = Case(lengths, heads, kv, D, seed=6)
    out, lse = torch.empty((c.T, heads, D), dtype=BF16, device=DEV), torch.empty((heads, c.T), dtype=F32, device=DEV)
    grads = [torch.empty_like(t) for t in (c.q, c.k, c.v)]
    ws = torch.empty(nb.nb_attention_workspace(c.T, heads), dtype=torch.uint8, device=DEV)
    ld, wide, n = [t.stride(0) for t in (c.q, c.k, c.v)], heads * D, len(lengths)

    def step(s):
        for t, x in zip((c.q, c.k, c.v, c.dout), (s.q, s.k, s.v, s.dout)):
            t.copy_(x)
        nb.nb_attention_forward(out, lse, c.q, c.k, c.v, c.cu, c.T, n, heads, kv, D, wide, *ld, D ** -0.5, True)
        nb.nb_attention_backward(*grads, c.dout, out, lse, c.q, c.k, c.v, c.cu, c.T, n, heads, kv, D, *(g.stride(0) for g in grads), wide, wide, *ld, D ** -0.5,
                                 True, ws, ws.numel())
    want = []
    for s in sets:
        step(s)
        torch.cuda.synchronize()
        want.append([g.clone() for g in grads])
    wrong = torch.zeros((), dtype=torch.int64, device=DEV)
    for _ in range(40):
        for s, w in zip(sets, want):
            step(s)
            for a, b in zip(grads, w):
                wrong += (a != b).sum()
    assert wrong.item() == 0
