"""The orthogonalised update and its application on the GPU, against the formulas in 64 bits."""
import pytest
import torch

from paper_2609_28568_b200 import binding as nb
from norm_reference import EPS32
from parity import Guarded

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def _status_clean():
    yield
    nb.nb_check_status()


def rand(seed, shape, std=1.0, dtype=F32):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV).mul_(std).to(dtype)


@pytest.mark.parametrize("copy", [True, False])
@pytest.mark.parametrize("n,count", [(1, 1), (2, 7), (3, 8), (1, 13), (5, 4099), (33, 776), (2, 1416 * 776), (12, 768 * 2304)])
def test_apply_every_element(n, count, copy):
    decay, step = 0.998, 0.02
    start = [rand(10 + i, (count,), 0.02) for i in range(n)]
    update = [rand(200 + i, (count,), 0.05, BF16) for i in range(n)]
    master = [Guarded((count,), F32) for _ in range(n)]
    weight = [Guarded((count,), BF16) for _ in range(n)] if copy else None
    for m, s in zip(master, start):
        m.t.copy_(s)
    nb.nb_muon_apply([m.t for m in master], [w.t for w in weight] if copy else None, update, n, count, decay, step)
    d32, s32 = (torch.tensor(v, dtype=F32).double().item() for v in (decay, step))  # the scalars arrive in 32 bits
    for i in range(n):
        ref = d32 * start[i].double() - s32 * update[i].double()
        # decay * master is rounded, then the difference: half a step each
        bound = EPS32 / 2 * (d32 * start[i].double().abs() + ref.abs() * (1 + EPS32))
        assert ((master[i].t.double() - ref).abs() <= bound).all(), i
        master[i].check("master")
        if copy:
            assert torch.equal(weight[i].t, master[i].t.to(BF16)), i
            weight[i].check("weight")


def test_apply_keeps_what_is_not_finite_where_it_is():
    m = rand(1, (4096,), 0.02)
    u = rand(2, (4096,), 0.05, BF16)
    m[5], u[6], u[4095] = float("inf"), float("nan"), float("-inf")
    w = torch.empty(4096, dtype=BF16, device=DEV)
    nb.nb_muon_apply([m], [w], [u], 1, 4096, 0.998, 0.02)
    bad = ~torch.isfinite(m)
    assert bad.nonzero().view(-1).tolist() == [5, 6, 4095] and torch.equal(~torch.isfinite(w), bad)
    assert m[5] == float("inf") and torch.isnan(m[6]) and m[4095] == float("inf")
