"""What the blocks of an update tell one another when something fails: nothing that another kernel reports or clears."""
import pytest
import torch

from paper_2609_28568_b200 import binding as nb

pytestmark = pytest.mark.gpu
DEV = "cuda"


def gradient(R, C, seed=1):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn((R, C), generator=g, device=DEV)


def test_another_kernels_failure_does_not_end_an_update():
    """A wait that runs out on another stream while updates are under way. Of a 64 x 9216 matrix one block forms x x^T from all 144 k-blocks while
    143 others wait for it, 32 times a call; 144 blocks leave room for the other kernel beside them."""
    grad, calls = [gradient(64, 9216)], 12
    args = (None, grad, 1, 64, 9216, 0.95, 0, 32, 1.5, -0.5, 0.0, 1e-7, nb.DTYPE_F32)
    ws = torch.empty(nb.nb_muon_workspace(1, 64, 9216), dtype=torch.uint8, device=DEV)
    want, *got = [torch.full((64, 9216), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(calls + 1)]
    nb.nb_muon_update([want], *args, ws, ws.numel())
    nb.nb_check_status()
    assert torch.isfinite(want.float()).all()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        nb.nb_debug_wait_timeout(2000)
    for u in got:
        nb.nb_muon_update([u], *args, ws, ws.numel())
    with pytest.raises(nb.NbError) as e:
        nb.nb_check_status()
    assert e.value.code == nb.NB_ERR_TIMEOUT and "wait id 900" in str(e.value)
    nb.nb_check_status()
    assert [i for i, u in enumerate(got) if not torch.equal(u, want)] == []
