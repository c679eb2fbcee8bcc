"""Layer norm and the orthogonalised update, without a GPU: refusals, workspace sizes, and the references that the GPU tests use."""
import ctypes

import pytest
import torch

from paper_2609_28568_b200 import binding as nb
from paper_2609_28568_b200 import build
from norm_reference import norm_backward, norm_forward

P = 0x10000  # a fake aligned device address: a refused call never touches it


def at(i):
    """The i-th of fake tensors that lie apart."""
    return P + (i << 20)


@pytest.fixture(scope="module")
def L():
    build.build()
    return nb.lib()


def test_norm_forward_refusals(L):
    def call(out=at(0), total=at(1), mean=at(2), rstd=at(3), inp=at(4), branch=at(5), w=at(6), b=at(7), BT=4, C=64, eps=1e-5, dtype=nb.DTYPE_BF16):
        return L.nb_layernorm_forward(out, total, mean, rstd, inp, branch, w, b, BT, C, eps, dtype, None)
    bad = nb.NB_ERR_INVALID_ARG
    for kw in (dict(out=None), dict(inp=None), dict(w=None), dict(total=None), dict(branch=None), dict(mean=None), dict(rstd=None),
               dict(BT=-1), dict(C=0), dict(eps=-1e-5), dict(eps=float("nan")), dict(eps=float("inf")), dict(dtype=2), dict(out=P + 8), dict(total=P + 2),
               dict(inp=P + 4), dict(branch=P + 2), dict(w=P + 2), dict(b=P + 2), dict(mean=P + 2), dict(rstd=P + 1)):
        assert call(**kw) == bad, kw
        assert nb.nb_last_error()
    for kw in (dict(out=at(4)), dict(out=at(1)), dict(total=at(5)), dict(out=at(5) + 16), dict(total=at(4) + 16), dict(mean=at(3) + 8), dict(rstd=at(4) + 32),
               dict(out=at(6)), dict(total=at(7), branch=at(7))):  # overlaps
        assert call(**kw) == bad and b"overlap" in L.nb_last_error(), kw
    for kw in (dict(C=12), dict(C=8200), dict(BT=1 << 31), dict(BT=(1 << 31) - 1, C=8192)):
        assert call(**kw) == nb.NB_ERR_UNSUPPORTED, kw
    assert call(BT=0) == nb.NB_OK


def test_norm_backward_refusals(L):
    need = nb.nb_layernorm_workspace(4, 64)

    def call(dinp=at(0), dbranch=at(1), dw=at(2), db=at(3), dout=at(4), dres=at(5), inp=at(6), mean=at(7), rstd=at(8), w=at(9), BT=4,
             C=64, acc=0, dtype=nb.DTYPE_F32, ws=at(10), size=need):
        return L.nb_layernorm_backward(dinp, dbranch, dw, db, dout, dres, inp, mean, rstd, w, BT, C, acc, dtype, ws, size, None)
    for kw in (dict(dinp=None), dict(dout=None), dict(inp=None), dict(mean=None), dict(rstd=None), dict(w=None), dict(ws=None),
               dict(size=need - 1), dict(size=0), dict(dw=None, size=0), dict(BT=-4), dict(C=-8), dict(dtype=7), dict(dinp=P + 4), dict(dbranch=P + 2), dict(dw=P + 4),
               dict(db=P + 8), dict(dout=P + 2), dict(dres=P + 4), dict(inp=P + 8), dict(w=P + 2), dict(ws=P + 8), dict(mean=P + 3),
               dict(rstd=P + 2)):
        assert call(**kw) == nb.NB_ERR_INVALID_ARG, kw
    for kw in (dict(dinp=at(6)), dict(dinp=at(5) + 16), dict(dbranch=at(0)), dict(dbranch=at(5)), dict(dw=at(3) + 16), dict(ws=at(4)), dict(ws=at(2)),
               dict(dw=at(9))):
        assert call(**kw) == nb.NB_ERR_INVALID_ARG and b"overlap" in L.nb_last_error(), kw
    for kw in (dict(C=20), dict(C=8200)):
        assert call(**kw) == nb.NB_ERR_UNSUPPORTED, kw
    assert call(BT=0, acc=1) == nb.NB_OK


def test_norm_workspace(L):
    assert L.nb_layernorm_workspace(-1, 64) == -1 and L.nb_layernorm_workspace(4, 12) == -1 and L.nb_layernorm_workspace(4, 8200) == -1
    with pytest.raises(nb.NbError):
        nb.nb_layernorm_workspace(4, 12)
    assert nb.nb_layernorm_workspace(0, 64) == 0
    for C in (8, 64, 768, 1024, 1032, 2048, 4096, 8192):
        sizes = [nb.nb_layernorm_workspace(rows, C) for rows in (1, 8, 9, 100, 4096, 1 << 30)]
        assert all(s > 0 and s % (8 * C) == 0 for s in sizes) and sizes == sorted(sizes)
        assert sizes[0] == 8 * C  # one block's sums


def _array(*addresses):
    return (ctypes.c_void_p * len(addresses))(*addresses)


def test_update_refusals(L):
    need = nb.nb_muon_workspace(2, 64, 128)

    def call(u=_array(at(0), at(1)), m=_array(at(2), at(3)), g=_array(at(4), at(5)), n=2, R=64, C=128, mu=0.95, nesterov=1, steps=5,
             co=nb.MUON_COEFFICIENTS, eps=1e-7, dtype=nb.DTYPE_F32, ws=at(9), size=need):
        return L.nb_muon_update(u, m, g, n, R, C, mu, nesterov, steps, *co, eps, dtype, ws, size, None)
    for kw in (dict(u=None), dict(g=None), dict(n=-1), dict(R=0), dict(C=-8), dict(mu=float("nan")), dict(eps=-1.0), dict(eps=float("nan")),
               dict(steps=-1), dict(steps=33), dict(co=(1.0, float("inf"), 0.0)), dict(dtype=3), dict(ws=None), dict(ws=P + 64),
               dict(size=need - 1), dict(u=_array(P, None)), dict(m=_array(None, P)), dict(g=_array(P, None)), dict(u=_array(P, P + 8)),
               dict(m=_array(P + 4, P)), dict(g=_array(P, P + 2))):
        assert call(**kw) == nb.NB_ERR_INVALID_ARG, kw
        assert nb.nb_last_error()
    for kw in (dict(R=12), dict(C=100), dict(n=1025), dict(R=32776), dict(co=(40.0, 0.0, 0.0)), dict(co=(3.0, 0.0, 0.0)), dict(co=(1.0, 50.0, -50.0))):
        assert call(**kw) == nb.NB_ERR_UNSUPPORTED, kw
    for kw in (dict(u=_array(at(0), at(0))), dict(u=_array(at(0), at(4))), dict(m=_array(at(2), at(2) + 16)), dict(m=_array(at(4), at(3))),
               dict(u=_array(at(2) + 1024, at(1))), dict(g=_array(at(9) + 128, at(5))), dict(u=_array(at(9), at(1)))):
        assert call(**kw) == nb.NB_ERR_INVALID_ARG and b"overlap" in L.nb_last_error(), kw
    assert call(n=0) == nb.NB_OK
    # polynomials in use: they keep [0, 1] near itself
    for co in (nb.MUON_COEFFICIENTS, (2.0, -1.5, 0.5), (1.5, -0.5, 0.0), (1.875, -1.25, 0.375)):
        assert call(n=0, co=co) == nb.NB_OK, co


def test_update_workspace(L):
    for bad in ((-1, 64, 64), (1, 0, 64), (1, 64, 12), (1025, 64, 64), (1, 32776, 64)):
        assert L.nb_muon_workspace(*bad) == -1
        with pytest.raises(nb.NbError):
            nb.nb_muon_workspace(*bad)
    assert nb.nb_muon_workspace(0, 64, 64) == 0
    # two iterates, two symmetric matrices
    assert nb.nb_muon_workspace(1, 768, 3072) >= 4 * 768 * 3072 + 4 * 768 * 768
    assert nb.nb_muon_workspace(33, 64, 64) == nb.nb_muon_workspace(32, 64, 64)
    assert nb.nb_muon_workspace(3, 64, 128) == nb.nb_muon_workspace(3, 128, 64)


def test_update_binding_refusals(L):
    t = torch.zeros(8, 8)
    with pytest.raises(ValueError, match="one shape"):
        nb.muon_update([t, torch.zeros(8, 16)])
    with pytest.raises(ValueError, match="one shape"):
        nb.muon_update([t, t.bfloat16()])
    with pytest.raises(ValueError, match="momenta"):
        nb.muon_update([t], [t.bfloat16()])
    assert nb.muon_update([]) == []


def test_norm_conveniences_refuse_other_types_and_shapes(L):
    """Before anything is launched: none of these tensors is on a device."""
    x, w, b16 = torch.zeros(4, 16), torch.zeros(16, dtype=torch.bfloat16), torch.zeros(4, 16, dtype=torch.bfloat16)
    m = torch.zeros(4)
    for kw in (dict(weight=w.float()), dict(weight=w[:8]), dict(weight=w, bias=w.float()), dict(weight=w, branch=x), dict(weight=w, branch=b16[:2])):
        with pytest.raises(ValueError, match="is wanted"):
            nb.layernorm_forward(x, **kw)
    good = dict(dout=b16, inp=x, mean=m, rstd=m, weight=w)
    for kw in (dict(dout=x), dict(mean=m.double()), dict(rstd=m[:3]), dict(weight=w.float()), dict(dres=b16), dict(dweight=w), dict(dbias=torch.zeros(8))):
        with pytest.raises(ValueError, match="is wanted"):
            nb.layernorm_backward(**{**good, **kw})
    with pytest.raises(TypeError):
        nb.layernorm_forward(x.half(), w)


def test_apply_refusals(L):
    def call(m=_array(at(0), at(1)), w=_array(at(2), at(3)), u=_array(at(4), at(5)), n=2, count=10):
        return L.nb_muon_apply(m, w, u, n, count, 0.9, 0.1, None)
    for kw in (dict(m=None), dict(u=None), dict(n=-1), dict(count=-1), dict(m=_array(P, None)), dict(u=_array(None, P)),
               dict(w=_array(P, None)), dict(m=_array(P, P + 4)), dict(u=_array(P + 2, P)), dict(w=_array(P, P + 8))):
        assert call(**kw) == nb.NB_ERR_INVALID_ARG, kw
    for kw in (dict(m=_array(at(0), at(0))), dict(w=_array(at(2), at(2) + 16)), dict(w=_array(at(0), at(3))), dict(u=_array(at(4), at(1) + 32)),
               dict(m=_array(at(0), at(0) + 32))):
        assert call(**kw) == nb.NB_ERR_INVALID_ARG and b"overlap" in L.nb_last_error(), kw
    assert call(n=1025) == nb.NB_ERR_UNSUPPORTED
    assert call(count=1 << 40) == nb.NB_ERR_UNSUPPORTED
    assert call(n=0) == nb.NB_OK and call(count=0) == nb.NB_OK
    assert L.nb_muon_apply(None, None, None, 0, 10, 0.9, 0.1, None) == nb.NB_OK


def test_binding_refusals(L):
    with pytest.raises(ValueError, match="master"):
        nb.nb_muon_apply([P], None, [P, P], 2, 0, 0.9, 0.1, 0)
    with pytest.raises(TypeError):
        nb.nb_muon_apply(P, None, [P], 1, 0, 0.9, 0.1, 0)
    with pytest.raises(nb.NbError):
        nb.nb_muon_apply([P], None, [None], 1, 8, 0.9, 0.1, 0)
    with pytest.raises(AssertionError):  # a CPU tensor
        nb.nb_muon_apply([torch.zeros(8)], None, [P], 1, 0, 0.9, 0.1, 0)
    with pytest.raises(TypeError):
        nb._stream_dtype(torch.zeros(1, dtype=torch.float16))
    nb.nb_muon_apply([P], None, (P,), 1, 0, 0.9, 0.1, 0)  # nothing to do
    nb.nb_muon_apply([], [], [], 0, 8, 0.9, 0.1, 0)


def test_reference_gradients_against_differences():
    g = torch.Generator().manual_seed(3)
    s, w, b, r = (torch.randn(shape, generator=g, dtype=torch.float64) for shape in ((3, 16), (16,), (16,), (3, 16)))
    f = lambda s_, w_, b_: (norm_forward(s_, w_, b_, 1e-5)["out"] * r).sum()  # noqa: E731
    fw = norm_forward(s, w, b, 1e-5)
    got = norm_backward(r, s, fw["mean"], fw["rstd"], w, None)
    h = 1e-6
    for name, at, grad in (("s", s, got["dinp"]), ("w", w, got["dweight"]), ("b", b, got["dbias"])):
        for i in range(at.numel()):
            d = torch.zeros_like(at)
            d.view(-1)[i] = h
            args = [(x + d if x is at else x, x - d if x is at else x) for x in (s, w, b)]
            diff = (f(*(a[0] for a in args)) - f(*(a[1] for a in args))) / (2 * h)
            # central differences: third derivatives times h^2, and 64-bit cancellation over h
            assert abs(diff - grad.view(-1)[i]) < 1e-8 * max(1.0, grad.abs().max().item()), (name, i)
