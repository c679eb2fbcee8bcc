"""Layer norm at batches whose rows pass through the ring of bulk copies, every form of it: each team's slots are filled again at least
twice, so that their barriers change phase, and the last round leaves some teams without a row."""
import pytest
import torch

from paper_2609_28568_b200 import binding as nb
from norm_reference import norm_forward
from parity import Guarded
from test_gpu_norm import BF16, DEV, F32, HALF_STEP, TYPES, EPS32, forward_bounds, rand, run_backward, within

pytestmark = pytest.mark.gpu
# Rows of up to 1024 elements belong to a warp, with one to four vectors per thread; to 2048, 4096, 8192 to 4, 8, 16 warps. 148 blocks
# of sixteen warps have 2368, 592, 296, 148 teams of at most four slots: nine rows for each and a few teams have ten. Each form with full rows
# and with rows that end inside a thread's vectors.
SIZES = [(2368 * 9 + 7, 8), (2368 * 9 + 7, 248), (2368 * 9 + 1, 256), (2368 * 9 + 5, 264), (2368 * 9 + 1203, 512), (2368 * 9 + 1, 520),
         (2368 * 9 + 9, 776), (2368 * 9 + 3, 1024), (592 * 9 + 5, 1032), (592 * 9 + 1, 1600), (592 * 9 + 301, 2048), (296 * 9 + 3, 2056),
         (296 * 9 + 1, 4096), (148 * 9 + 1, 4104), (148 * 9 + 71, 8192)]


@pytest.fixture(autouse=True)
def _status_clean():
    yield
    nb.nb_check_status()


@pytest.mark.parametrize("stream", ["bf16", "f32"])
@pytest.mark.parametrize("rows,C", SIZES)
def test_forward(rows, C, stream):
    dtype, code = TYPES[stream]
    x, br = rand(1, (rows, C), 1.5, 0.3, dtype), rand(2, (rows, C), 0.7)
    w, b = rand(3, (C,), 0.2, 1.0), rand(4, (C,), 0.1)
    for branch, bias, stats in ((br, b, True), (None, None, False)):
        out = Guarded((rows, C), BF16)
        total = Guarded((rows, C), dtype) if branch is not None else None
        mean, rstd = (Guarded((rows,), F32), Guarded((rows,), F32)) if stats else (None, None)
        nb.nb_layernorm_forward(out.t, total.t if total else None, mean.t if stats else None, rstd.t if stats else None, x, branch,
                                w, bias, rows, C, 1e-5, code)
        if branch is not None:
            assert torch.equal(total.t, (x.float() + branch.float()).to(dtype))  # one rounding: no tolerance
            total.check("sum")
        s = (x if branch is None else total.t).double()
        bd = None if bias is None else bias.double()
        r = norm_forward(s, w.double(), bd, 1e-5)
        dmean, drstd, slack = forward_bounds(s, r, w.double(), bd, C)
        within(out.t, r["out"], HALF_STEP * (r["out"].abs() + slack) + slack, "out")
        out.check("out")
        if stats:
            within(mean.t[:, None], r["mean"], dmean + EPS32 * r["mean"].abs(), "mean")
            within(rstd.t[:, None], r["rstd"], drstd, "rstd")
            mean.check("mean")
            rstd.check("rstd")


@pytest.mark.parametrize("stream", ["bf16", "f32"])
@pytest.mark.parametrize("rows,C", SIZES)
def test_backward(rows, C, stream):
    """A column's sum adds a team's rows (at most rows // 148 + 1), the sixteen teams of a block or fewer, five blocks and 32 groups: 54 +
    rows // 148 roundings, within the 64 + rows // 148 that the bound counts."""
    run_backward(rows, C, stream, dres=True, copy=True, accumulate=True)
    run_backward(rows, C, stream, dres=False, copy=False, accumulate=False, seed=30)


@pytest.mark.parametrize("stream", ["bf16", "f32"])
@pytest.mark.parametrize("rows,C", [(2368 * 9 + 7, 248), (2368 * 9 + 3, 1024), (592 * 9 + 5, 1600), (296 * 9 + 3, 4096), (148 * 9 + 1, 8192)])
def test_in_place(rows, C, stream):
    """Rows are stored over their own memory while copies of later rows are under way."""
    dtype, code = TYPES[stream]
    x, br, w, b = rand(1, (rows, C), 1.0, 0.0, dtype), rand(2, (rows, C)), rand(3, (C,), 0.2, 1.0), rand(4, (C,), 0.1)
    out, total, mean, rstd = nb.layernorm_forward(x, w, b, branch=br)
    x2, br2 = x.clone(), br.clone()
    nb.nb_layernorm_forward(br2, x2, None, None, x2, br2, w, b, rows, C, 1e-5, code)
    assert torch.equal(x2, total) and torch.equal(br2, out)
    dout, dres = rand(5, (rows, C), 1e-3), rand(6, (rows, C), 1e-3, 0.0, dtype)
    dinp, dbranch, dw, db = nb.layernorm_backward(dout, total, mean, rstd, w, dres=dres)
    dres2, dout2, dw2, db2 = dres.clone(), dout.clone(), torch.empty_like(dw), torch.empty_like(db)
    ws = torch.empty(nb.nb_layernorm_workspace(rows, C), dtype=torch.uint8, device=DEV)
    nb.nb_layernorm_backward(dres2, dout2, dw2, db2, dout2, dres2, total, mean, rstd, w, rows, C, 0, code, ws, ws.numel())
    assert torch.equal(dres2, dinp) and torch.equal(dout2, dbranch) and torch.equal(dw2, dw) and torch.equal(db2, db)
