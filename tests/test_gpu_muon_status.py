"""What the blocks of an update tell one another when something fails: nothing that another kernel reports or clears."""
import time

import pytest
import torch

from paper_2609_28568_b200 import binding as nb
from norm_reference import newton_schulz
from parity import Guarded

DEV = "cuda"


def gradient(R, C, seed=1):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn((R, C), generator=g, device=DEV)


@pytest.mark.gpu
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


def test_refusals():
    L = nb.lib()
    P = 0x10000  # a fake aligned device address: a refused call never touches it
    need = nb.nb_muon_workspace(1, 128, 128)
    for args in ((None, P, P, need, 1000), (P, None, P, need, 1000), (P, P, None, need, 1000), (P + 8, P, P, need, 1000), (P, P + 4, P, need, 1000),
                 (P, P, P + 64, need, 1000), (P, P, P, need - 1, 1000), (P, P, P, need, 99), (P, P, P, need, 1000001)):
        assert L.nb_debug_muon_timeout(*args) == nb.NB_ERR_INVALID_ARG, args


@pytest.mark.gpu
def test_time_out_exit_and_recovery():
    """Four blocks, three of which store a tile of S before they wait in vain: three for what a tile of P takes, one for what a tile of X takes,
    which P's missing tiles keep from coming. Either may be the first to run out."""
    grad = gradient(128, 128)
    update = Guarded((128, 128), torch.bfloat16)
    update.t.fill_(7.0)
    ws = Guarded((nb.nb_muon_workspace(1, 128, 128) // 4 + 32,), torch.float32)
    at = ws.t[(-ws.t.data_ptr() % 128) // 4:]  # on the boundary that the call asks for
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    nb.nb_debug_muon_timeout(update.t, grad, at, at.numel() * 4, 3000)
    with pytest.raises(nb.NbError) as e:
        nb.nb_check_status()
    took = time.perf_counter() - t0
    assert e.value.code == nb.NB_ERR_TIMEOUT and any(f"wait id {i}" in str(e.value) for i in (701, 702))
    assert torch.all(update.t == 7.0)
    update.check("update of the aborted call")
    ws.check("workspace of the aborted call")
    assert 0.003 <= took < 1.0
    nb.nb_check_status()  # cleared
    # the same workspace again: the word of failure in it does not last
    nb.nb_muon_update([update.t], None, [grad], 1, 128, 128, 0.0, 0, 2, 1.5, -0.5, 0.0, 1e-7, nb.DTYPE_F32, at, at.numel() * 4)
    ref = newton_schulz(grad.double(), 2, (1.5, -0.5, 0.0), 1e-7)
    # two iterates, two S and two P rounded to fp16, at an rms of 2^-11 / sqrt(3) each, and the result to bf16 at 2^-8 / sqrt(3): 2.4e-3
    assert ((update.t.double() - ref).norm() / ref.norm()).item() <= 4e-3
    update.check("update after recovery")
