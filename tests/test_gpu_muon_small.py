"""Updates of gradients that eps outweighs: where the figures of full precision end, and what holds from there on."""
import pytest
import torch

from paper_2609_28568_b200 import binding as nb
from norm_reference import newton_schulz
from test_gpu_muon import BF16, COEFFICIENTS, close, gradients

pytestmark = pytest.mark.gpu
R, C = 136, 264


@pytest.fixture(autouse=True)
def _status_clean():
    yield
    nb.nb_check_status()


def update(std, eps):
    grad = gradients(50, 1, R, C, std)
    return nb.muon_update(grad, eps=eps)[0], newton_schulz(grad[0].double(), 5, COEFFICIENTS, eps)


@pytest.mark.parametrize("std", [1e-10, 1e-14, 1e-15])
def test_precision_of_larger_gradients_down_to_1e_6_of_eps(std):
    """136 x 264 values of std have a norm of 190 std or more: 1e-15 gives |v| / eps = 2e-6 and values of x of 1e-8, which fp16 at 2^12 holds
    to 2^-37 / sqrt(3) = 4e-12: 4e-4 of them, within what the bound has to spare over the roundings it counts."""
    close(*update(std, 1e-7), f"std {std}")


@pytest.mark.parametrize("std", [1e-16, 1e-17, 1e-18, 1e-19, 1e-24])
def test_stated_bound_below(std):
    """x x^T is below 1e-13 and P = a I: the steps multiply by a. Each of the five x and five P takes a rounding of 2^-11 of its value, x where it
    is subnormal one of 2^-37 instead, multiplied by a in each step that follows; the result one of 2^-8 to bf16."""
    got, ref = update(std, 1e-7)
    a = COEFFICIENTS[0]
    absolute = 2.0 ** -37 * sum(a ** k for k in range(1, 6))
    relative = (1 + 2.0 ** -11) ** 10 * (1 + torch.finfo(BF16).eps / 2) - 1
    assert absolute < 5.1e-9  # as the header has it
    err = (got.double() - ref).abs()
    # what S adds to P: |b| x^2 beside a, 1e-13 of it at most
    assert (err <= absolute * (1 + relative) + ref.abs() * (relative + 1e-12)).all(), (err - ref.abs() * relative).max().item()


@pytest.mark.parametrize("std", [1e-30, 1e-12, 1e30])
def test_without_eps_any_gradient_is_one_like_another(std):
    close(*update(std, 0.0), f"std {std}")
