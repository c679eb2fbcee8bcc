"""Rotary positions against their formula in 64 bits (bounds: attention_reference.py)."""
import math

import pytest
import torch

from paper_2609_28568_b200 import binding as nb
import attention_reference as ref
from test_gpu_attention import BF16, DEV, Case, cumulated, rand, within

pytestmark = pytest.mark.gpu
HALF, NEIGHBOURS = nb.ROTARY_HALF, nb.ROTARY_NEIGHBOURS


@pytest.fixture(autouse=True)
def _status_clean():
    yield
    nb.nb_check_status()


def places(bounds, T):
    at = torch.zeros(T, dtype=torch.int64)
    for a, b in ref.spans(bounds):
        at[a:b] = torch.arange(b - a)
    return at.to(DEV)


def check(c, R, layout, positions=None, scale=1.0, inverse=False, **freq):
    f = nb.rotary_frequencies(R, **freq)
    at = places(c.bounds, c.T) if positions is None else positions
    out = [torch.full((c.T, h, c.D), 7.0, dtype=BF16, device=DEV) for h in (c.heads, c.kv)]
    nb.nb_rotary(*out, c.q, c.k, f, positions, c.cu, c.T, len(c.bounds) - 1, c.heads, c.kv, c.D, R, c.heads * c.D, c.kv * c.D, c.q.stride(0), c.k.stride(0),
                 scale, layout, inverse)
    rows = slice(c.bounds[0], c.bounds[-1])
    scale32 = torch.tensor(scale, dtype=torch.float32).item()
    want = ref.frequencies(R, **{"base": 10000.0, **freq})
    for got, x in zip(out, (c.q, c.k)):
        assert (c.outside(got) == 7.0).all()
        y, tol = ref.rotary(x, want, at, scale32, layout == HALF, inverse)
        within(got[rows], y[rows], tol[rows], "rotary")


@pytest.mark.parametrize("D,R,layout", [(64, 64, HALF), (128, 128, HALF), (128, 128, NEIGHBOURS), (80, 32, HALF), (80, 80, HALF), (80, 72, NEIGHBOURS), (16, 16, HALF),
                                        (8, 8, NEIGHBOURS), (128, 16, HALF), (104, 96, NEIGHBOURS), (120, 48, HALF)])
@pytest.mark.parametrize("inverse", [False, True])
def test_widths(D, R, layout, inverse):
    check(Case([50, 0, 1, 33], 3, 1, D, first=2, pad=7, fused=True), R, layout, inverse=inverse)
    check(Case([9], 4, 4, D), R, layout, inverse=inverse, scale=1.4)


@pytest.mark.parametrize("T", [1, 2, 7, 148, 593, 1200, 5000])
def test_rows(T):
    check(Case([T], 2, 2, 32, seed=T), 32, HALF)


@pytest.mark.parametrize("n", [1, 31, 32, 33, 1000])
def test_sequences(n):
    g = torch.Generator().manual_seed(n)
    check(Case(torch.randint(0, 4, (n,), generator=g).tolist(), 2, 1, 16, first=1, pad=3), 16, HALF)


@pytest.mark.parametrize("far", [1 << 12, 1 << 17, 1 << 24, (1 << 31) - 1])
@pytest.mark.parametrize("layout", [HALF, NEIGHBOURS])
def test_far_positions(far, layout):
    """An angle formed in 32 bits would be off by far 2^-24 radians: of another turn altogether. In 64 bits 2^31 positions cost
    2^31 2^-52 radians more than fp32 has."""
    c = Case([64], 2, 1, 64)
    g = torch.Generator().manual_seed(1)
    at = (torch.rand(64, generator=g, dtype=torch.float64) * far).long().to(torch.int32)
    at[:2] = torch.tensor([far, 0], dtype=torch.int64).to(torch.int32)
    check(c, 64, layout, at.to(DEV))
    check(c, 64, layout, -at.to(DEV))


@pytest.mark.parametrize("freq", [dict(base=1.0e6), dict(factor=8.0), dict(base=5.0e5, factor=16.0, original=4096), dict(factor=4.0, low=2.0, high=8.0, original=512)])
def test_scaled_contexts(freq):
    check(Case([3000], 1, 1, 64), 64, HALF, scale=1.2, **freq)


def test_in_place_and_queries_alone():
    c = Case([70, 30], 4, 2, 80, fused=True)
    f = nb.rotary_frequencies(48)
    q, k = nb.rotary(c.q, c.k, f, cu_seqlens=c.cu)
    alone, none = nb.rotary(c.q, None, f, cu_seqlens=c.cu)
    assert none is None and torch.equal(alone, q)
    v = c.v.clone()
    got = nb.rotary(c.q, c.k, f, cu_seqlens=c.cu, in_place=True)
    assert got[0] is c.q and torch.equal(c.q, q) and torch.equal(c.k, k) and torch.equal(c.v, v)


def test_of_one_length():
    c = Case([25] * 4, 2, 2, 32)
    f = nb.rotary_frequencies(32)
    for a, b in zip(nb.rotary(c.q, c.k, f, n=4), nb.rotary(c.q, c.k, f, cu_seqlens=c.cu)):
        assert torch.equal(a, b)
    assert nb.rotary(c.q[:0], c.k[:0], f)[0].shape == (0, 2, 32)


def test_not_finite_values_stay_where_they_are():
    c = Case([40], 2, 1, 32)
    f = nb.rotary_frequencies(32)
    q, _ = nb.rotary(c.q, c.k, f)
    c.q[7, 1, 3], c.q[9, 0, 20] = math.nan, math.inf
    q2, _ = nb.rotary(c.q, c.k, f)
    same = q == q2
    assert not same[7, 1, 3] and not same[7, 1, 19] and not same[9, 0, 4] and not same[9, 0, 20] and same.sum() == same.numel() - 4


@pytest.mark.parametrize("bounds", [[0, 400], [-5, 300], [0, 200, 100, 300], [300, 0], [0, 1 << 30, 300]])
def test_bad_bounds_are_reported(bounds):
    whole = torch.full((300 + 128, 2, 32), 3.0, dtype=BF16, device=DEV)
    q = whole[64:-64]
    nb.nb_rotary(q, None, q, None, nb.rotary_frequencies(32), None, torch.tensor(bounds, dtype=torch.int32, device=DEV), 300, len(bounds) - 1, 2, 2, 32, 32,
                 64, 64, 64, 64, 1.0, HALF, 0)
    with pytest.raises(nb.NbError) as e:
        nb.nb_check_status()
    assert e.value.code == nb.NB_ERR_INVALID_ARG and "cu_seqlens" in str(e.value)
    assert (whole[:64] == 3.0).all() and (whole[-64:] == 3.0).all()


def test_gradient():
    """The outputs' gradient turned back is the inputs' gradient, by autograd through the formula."""
    bounds = cumulated([33, 12])
    x, dy = rand(1, (45, 3, 64)), rand(2, (45, 3, 64))
    cu = torch.tensor(bounds, dtype=torch.int32, device=DEV)
    f = nb.rotary_frequencies(48)
    got, _ = nb.rotary(dy, None, f, cu_seqlens=cu, scale=1.3, inverse=True)
    xd = x.double().requires_grad_()
    angle = places(bounds, 45).double()[:, None] * ref.frequencies(48, 10000.0).to(DEV)
    c, s = 1.3 * torch.cos(angle)[:, None], 1.3 * torch.sin(angle)[:, None]
    a, b, rest = xd[..., :24], xd[..., 24:48], xd[..., 48:]
    torch.cat((a * c - b * s, b * c + a * s, rest), -1).backward(dy.double())
    _, tol = ref.rotary(dy, ref.frequencies(48, 10000.0), places(bounds, 45), 1.3, True, True)
    # 1.3 is not a number of 32 bits
    within(got, xd.grad, tol + 2 * ref.U32 * dy.double().abs().amax() * 2, "gradient")


def test_captured():
    c = Case([120, 30], 4, 2, 64)
    f = nb.rotary_frequencies(64)
    nb.rotary(c.q, c.k, f, cu_seqlens=c.cu)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        held = nb.rotary(c.q, c.k, f, cu_seqlens=c.cu)
    c.q.mul_(2.0)
    g.replay()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        want = nb.rotary(c.q, c.k, f, cu_seqlens=c.cu)
    side.synchronize()
    torch.cuda.synchronize()
    for a, b in zip(held, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("D,R,layout", [(80, 32, NEIGHBOURS), (96, 64, HALF), (128, 64, HALF), (128, 32, NEIGHBOURS), (72, 16, NEIGHBOURS), (24, 8, NEIGHBOURS), (40, 16, HALF),
                                        (48, 48, NEIGHBOURS), (104, 80, HALF)])
def test_part_of_a_head(D, R, layout):
    """Columns that are copied, in pieces of one or two vectors; in place they are left alone, NaN among them."""
    c = Case([70, 1, 30], 6, 2, D, first=3, pad=9, fused=True)
    check(c, R, layout)
    check(c, R, layout, inverse=True, scale=0.75)
    f = nb.rotary_frequencies(R)
    want = nb.rotary(c.q, c.k, f, cu_seqlens=c.cu, layout=layout)
    v = c.v.clone()
    if R < D:
        c.q[20, 1, R], c.k[20, 1, D - 1] = math.nan, math.inf
        want[0][20, 1, R], want[1][20, 1, D - 1] = math.nan, math.inf
    nb.rotary(c.q, c.k, f, cu_seqlens=c.cu, layout=layout, in_place=True)
    rows = slice(3, 104)
    for got, w in zip((c.q, c.k, c.v), (*want, v)):
        assert torch.equal(got[rows].nan_to_num(nan=9.0, posinf=8.0), w[rows].nan_to_num(nan=9.0, posinf=8.0))
        assert torch.isnan(got[:3]).all() and torch.isnan(got[104:]).all()
