"""Layer norm of finite rows whose sums leave fp32's range."""
import pytest
import torch

from paper_2609_28568_b200 import binding as nb

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def test_norm_of_rows_whose_squares_leave_fp32():
    """As the header has it; rows beside them are not touched."""
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x = torch.randn((5, 264), generator=g, device="cuda")
    w = torch.randn(264, generator=g, device="cuda").to(BF16)
    b = torch.randn(264, generator=g, device="cuda").to(BF16)
    good, _, _, _ = nb.layernorm_forward(x, w, b)
    x[1] *= 1e25
    x[3] = 3e38
    out, _, _, rstd = nb.layernorm_forward(x, w, b)
    assert torch.equal(out[1], b) and rstd[1] == 0.0
    assert torch.isnan(out[3].float()).all()
    assert all(torch.equal(out[i], good[i]) for i in (0, 2, 4))
