"""Updates of matrices whose singular values are much alike, as those of thin ones are: rounding errors where a step is steep."""
import pytest
import torch

from paper_2609_28568_b200 import binding as nb
from norm_reference import newton_schulz
from test_gpu_muon import BF16, COEFFICIENTS, gradients

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _status_clean():
    yield
    nb.nb_check_status()


def predicted(x):
    """2-norm that the roundings to fp16 leave of the update, relative to it. In the direction of a singular value x a step takes x to f(x) = x p(x^2), with
    p(s) = a + b s + c s^2, and a relative error to x f'(x) / f(x) times itself: up to 5 near x = 1.2. Each rounding has an rms of 2^-11 / sqrt(3)
    at most. Those of x and P pass as they are, that of S = x^2 as s p'(s) / p(s) of itself; each is multiplied in the steps that follow."""
    a, b, c = COEFFICIENTS
    r = 2.0 ** -11 / 3 ** 0.5
    square = torch.zeros_like(x)
    for _ in range(5):
        s = x * x
        p, slope = a + b * s + c * s * s, b * s + 2 * c * s * s
        gain = 1 + 2 * slope / p
        square = (square + r * r) * gain ** 2 + r * r * (1 + (slope / p) ** 2)
        x = x * p
    return ((square * x * x).sum() / (x * x).sum()).sqrt().item()


@pytest.mark.parametrize("R,C", [(8, 64), (16, 264), (24, 1000), (32, 608), (608, 32), (40, 520), (48, 2000), (64, 4096), (2304, 64), (128, 1024)])
def test_thin_matrices(R, C):
    grad = gradients(40, 6, R, C, 1e-4)
    half = torch.finfo(BF16).eps / 2 / 3 ** 0.5  # rms of the result's rounding, at most
    for g, got in zip(grad, nb.muon_update(grad)):
        v = g.double()
        ref = newton_schulz(v, 5, COEFFICIENTS, 1e-7)
        want = predicted(torch.linalg.svdvals(v) / v.norm())
        err = ((got.double() - ref).norm() / ref.norm()).item()
        # twice the rms: of a few directions one may take most
        assert err <= 2 * (want ** 2 + half ** 2) ** 0.5, (err, want)
        assert want <= 5e-3  # as the header has it


def test_rows_at_right_angles_and_of_one_length():
    """All singular values the same: 1 / sqrt(m) at first, which is steep in one step or another by m."""
    half = torch.finfo(BF16).eps / 2 / 3 ** 0.5
    for m in (8, 24, 32, 40, 64, 96, 200):
        g = torch.Generator(device="cuda")
        g.manual_seed(m)
        v = torch.linalg.qr(torch.randn((1024, m), generator=g, device="cuda", dtype=torch.float64))[0].T.float().contiguous()
        got, ref = nb.muon_update([v])[0], newton_schulz(v.double(), 5, COEFFICIENTS, 1e-7)
        want = predicted(torch.linalg.svdvals(v.double()) / v.double().norm())
        assert ((got.double() - ref).norm() / ref.norm()).item() <= 2 * (want ** 2 + half ** 2) ** 0.5, (m, want)
