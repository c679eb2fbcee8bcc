"""The layer norm's bounded waits, made to run out: the kernels leave by themselves, store nothing and say so."""
import time

import pytest
import torch

from paper_2609_28568_b200 import binding as nb
from parity import Guarded
from test_gpu_norm import BF16, DEV, rand, run_backward


def test_refusals():
    L = nb.lib()
    P = 0x10000  # a fake aligned device address: a refused call never touches it
    for args in ((None, P, P, P, 0, 1000), (P, None, P, P, 0, 1000), (P, P, None, P, 1, 1000), (P, P, P, None, 1, 1000), (P + 8, P, P, P, 0, 1000),
                 (P, P, P + 4, P, 0, 1000), (P, P, P, P, 0, 99), (P, P, P, P, 0, 1000001)):
        assert L.nb_debug_layernorm_timeout(*args) == nb.NB_ERR_INVALID_ARG, args


@pytest.mark.gpu
@pytest.mark.parametrize("backward", [False, True])
def test_time_out_exit_and_recovery(backward):
    rows, C = 5000, 64
    x, w = rand(1, (rows, C)), rand(2, (C,), 0.2, 1.0)
    stats = torch.ones(rows, device=DEV)
    out = Guarded((rows, C), BF16)
    out.t.fill_(7.0)
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    nb.nb_debug_layernorm_timeout(out.t, x, w, stats, backward, 3000)
    with pytest.raises(nb.NbError) as e:
        nb.nb_check_status()
    took = time.perf_counter() - t0
    assert e.value.code == nb.NB_ERR_TIMEOUT and f"wait id {810 if backward else 811}" in str(e.value)
    assert torch.all(out.t == 7.0)  # two or three rows of each team: none is stored
    out.check("aborted norm")
    assert 0.003 <= took < 1.0  # one limit, not one for each row
    nb.nb_check_status()  # cleared
    run_backward(rows, C, "bf16", True, True, True)
    got, _, mean, _ = nb.layernorm_forward(x, w)
    ref = torch.nn.functional.layer_norm(x.double(), (C,), w.double(), None, 1e-5)
    # one rounding to bf16, and 32-bit arithmetic (values of about 4 at most)
    assert ((got.double() - ref).abs() <= torch.finfo(BF16).eps / 2 * ref.abs() + 1e-5).all()
