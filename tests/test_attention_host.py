"""Rotary positions and attention, without a GPU: refusals, workspace sizes, frequencies, and the references that the GPU tests use."""
import ctypes
import math

import pytest
import torch

from paper_2609_28568_b200 import binding as nb
from paper_2609_28568_b200 import build
import attention_reference as ref

P = 0x10000  # a fake aligned device address: a refused call never touches it


def at(i):
    """The i-th of fake tensors that lie apart."""
    return P + (i << 24)


@pytest.fixture(scope="module")
def L():
    build.build()
    return nb.lib()


def forward(L, out=at(0), lse=at(1), q=at(2), k=at(3), v=at(4), cu=at(5), T=64, n=3, heads=4, kv=2, D=64, ld_out=256, ld_q=512, ld_k=512, ld_v=512,
            scale=0.125, causal=1):
    return L.nb_attention_forward(out, lse, q, k, v, cu, T, n, heads, kv, D, ld_out, ld_q, ld_k, ld_v, scale, causal, None)


def backward(L, dq=at(0), dk=at(1), dv=at(2), dout=at(3), out=at(4), lse=at(5), q=at(6), k=at(7), v=at(8), cu=at(9), T=64, n=3, heads=4, kv=2, D=64,
             ld=(256, 128, 128, 256, 256, 512, 512, 512), scale=0.125, causal=1, ws=at(10), size=64 * 4 * 4):
    return L.nb_attention_backward(dq, dk, dv, dout, out, lse, q, k, v, cu, T, n, heads, kv, D, *ld, scale, causal, ws, size, None)


def rotary(L, oq=at(0), ok=at(1), q=at(2), k=at(3), freq=at(4), pos=at(5), cu=at(6), T=64, n=3, heads=4, kv=2, D=64, R=32, ld_oq=256, ld_ok=128, ld_q=256,
           ld_k=128, scale=1.0, layout=nb.ROTARY_HALF, inverse=0):
    return L.nb_rotary(oq, ok, q, k, freq, pos, cu, T, n, heads, kv, D, R, ld_oq, ld_ok, ld_q, ld_k, scale, layout, inverse, None)


SIZES_INVALID = [dict(T=-1), dict(n=-1), dict(heads=0), dict(kv=0), dict(kv=-2), dict(D=0), dict(heads=4, kv=3), dict(cu=None, n=3)]
SIZES_UNSUPPORTED = [dict(D=60), dict(D=136), dict(T=2147483001, n=1), dict(n=2147483001), dict(heads=1026, kv=2)]


@pytest.mark.parametrize("call", [forward, backward, rotary])
def test_sizes_refused(L, call):
    for kw in SIZES_INVALID:
        assert call(L, **kw) == nb.NB_ERR_INVALID_ARG and nb.nb_last_error(), kw
    for kw in SIZES_UNSUPPORTED:
        assert call(L, **kw) == nb.NB_ERR_UNSUPPORTED, kw
    for kw in (dict(T=0), dict(n=0), dict(T=0, n=0, cu=None)):
        assert call(L, **kw) == nb.NB_OK, kw


def test_forward_refusals(L):
    bad = nb.NB_ERR_INVALID_ARG
    for kw in (dict(out=None), dict(q=None), dict(k=None), dict(v=None), dict(out=P + 8), dict(q=P + 2), dict(k=P + 4), dict(v=P + 8), dict(lse=P + 2),
               dict(cu=P + 1), dict(ld_out=248), dict(ld_q=248), dict(ld_k=120), dict(ld_v=0), dict(ld_v=-512), dict(scale=0.0), dict(scale=-1.0),
               dict(scale=math.nan), dict(scale=math.inf)):
        assert forward(L, **kw) == bad, kw
    for kw in (dict(ld_out=260), dict(ld_k=132), dict(ld_q=(1 << 32) + 8)):
        assert forward(L, **kw) == nb.NB_ERR_UNSUPPORTED, kw
    # columns of one buffer are apart where neither reaches into the other
    for kw in (dict(out=at(2)), dict(out=at(2) + 496, ld_out=512), dict(lse=at(3) + 64), dict(out=at(5)), dict(lse=at(5)), dict(out=at(1)), dict(out=at(2) + 512)):
        assert forward(L, **kw) == bad and b"overlap" in L.nb_last_error(), kw


def test_backward_refusals(L):
    bad = nb.NB_ERR_INVALID_ARG
    for name in ("dq", "dk", "dv", "dout", "out", "q", "k", "v"):
        assert backward(L, **{name: None}) == bad and backward(L, **{name: P + 8}) == bad, name
    for i in range(8):
        ld = [256, 128, 128, 256, 256, 512, 512, 512]
        ld[i] = 120
        assert backward(L, ld=ld) == bad, i
        ld[i] = 516
        assert backward(L, ld=ld) == nb.NB_ERR_UNSUPPORTED, i
    for kw in (dict(lse=None), dict(lse=P + 2), dict(cu=P + 2), dict(ws=None), dict(ws=P + 8), dict(size=64 * 4 * 4 - 1), dict(size=-1), dict(scale=0.0),
               dict(scale=math.nan)):
        assert backward(L, **kw) == bad, kw
    fused = (512, 512, 512, 256, 256, 512, 512, 512)
    for kw in (dict(dq=at(1)), dict(dv=at(8)), dict(dk=at(10)), dict(ws=at(5)), dict(dq=at(3)), dict(ws=at(9)), dict(dk=at(0) + 496, ld=fused), dict(dq=at(4)),
               dict(dv=at(0) + 1024 - 16, ld=fused)):
        assert backward(L, **kw) == bad and b"overlap" in L.nb_last_error(), kw


def test_rotary_refusals(L):
    bad = nb.NB_ERR_INVALID_ARG
    for kw in (dict(oq=None), dict(q=None), dict(freq=None), dict(ok=None), dict(k=None), dict(oq=P + 8), dict(ok=P + 2), dict(q=P + 4), dict(k=P + 8),
               dict(freq=P + 4), dict(pos=P + 2), dict(cu=P + 1), dict(layout=2), dict(layout=-1), dict(R=0), dict(R=-16), dict(R=80), dict(scale=math.nan),
               dict(scale=math.inf), dict(ld_oq=248), dict(ld_ok=120), dict(ld_q=0), dict(ld_k=8)):
        assert rotary(L, **kw) == bad, kw
    for kw in (dict(R=24), dict(R=8), dict(R=20, layout=nb.ROTARY_NEIGHBOURS), dict(ld_q=260)):
        assert rotary(L, **kw) == nb.NB_ERR_UNSUPPORTED, kw
    for kw in (dict(oq=at(3)), dict(ok=at(2)), dict(oq=at(1)), dict(oq=at(2), ld_oq=512), dict(oq=at(2) + 16), dict(oq=at(5)), dict(ok=at(6)), dict(oq=at(4))):
        assert rotary(L, **kw) == bad and b"overlap" in L.nb_last_error(), kw


def test_workspace(L):
    for bad in ((-1, 4), (4, 0), (2147483001, 4), (4, 1025)):
        assert L.nb_attention_workspace(*bad) == -1
        with pytest.raises(nb.NbError):
            nb.nb_attention_workspace(*bad)
    assert nb.nb_attention_workspace(0, 4) == 0 and nb.nb_attention_workspace(1000, 12) == 48000


def test_timeout_refusals(L):
    tensors = (ctypes.c_void_p * 10)(*(at(i) for i in range(10)))
    broken = (ctypes.c_void_p * 10)(*(at(i) for i in range(9)), None)
    for args in ((None, 0, 1000), (broken, 0, 1000), (tensors, 3, 1000), (tensors, 0, 99), (tensors, 0, 1000001)):
        assert L.nb_debug_attention_timeout(*args) == nb.NB_ERR_INVALID_ARG, args


@pytest.mark.parametrize("R,kw", [(2, {}), (64, {}), (128, dict(base=1.0e6)), (128, dict(base=5.0e5, factor=8.0)), (64, dict(factor=4.0, original=8192)),
                                  (128, dict(base=1.0e6, factor=32.0, low=1.0, high=4.0, original=2048))])
def test_frequencies(L, R, kw):
    got = torch.tensor(nb.nb_rotary_frequencies(R, **kw), dtype=torch.float64)
    want = ref.frequencies(R, **{"base": 10000.0, **kw})
    assert (got - want).abs().max() <= 1e-15 * want.abs().max() and ((got / want - 1).abs() <= 1e-13).all()
    if kw.get("original"):  # fast pairs stay, slow ones are divided
        plain = ref.frequencies(R, kw.get("base", 10000.0))
        assert got[0] == plain[0] and abs(got[-1] * kw["factor"] / plain[-1] - 1) < 1e-13


def test_frequencies_refused(L):
    for kw, rc in ((dict(R=0), nb.NB_ERR_INVALID_ARG), (dict(R=7), nb.NB_ERR_UNSUPPORTED), (dict(R=130), nb.NB_ERR_UNSUPPORTED),
                   (dict(R=64, base=0.0), nb.NB_ERR_INVALID_ARG), (dict(R=64, base=math.inf), nb.NB_ERR_INVALID_ARG), (dict(R=64, factor=0.0), nb.NB_ERR_INVALID_ARG),
                   (dict(R=64, factor=-2.0), nb.NB_ERR_INVALID_ARG), (dict(R=64, original=-1), nb.NB_ERR_INVALID_ARG),
                   (dict(R=64, original=10, low=4.0, high=4.0), nb.NB_ERR_INVALID_ARG), (dict(R=64, original=10, low=math.nan), nb.NB_ERR_INVALID_ARG)):
        with pytest.raises(nb.NbError) as e:
            nb.nb_rotary_frequencies(**kw)
        assert e.value.code == rc, kw
    assert L.nb_rotary_frequencies(None, 64, 1e4, 1.0, 1.0, 32.0, 0) == nb.NB_ERR_INVALID_ARG


def test_conveniences_refuse_other_types_and_shapes(L):
    """Before anything is launched: none of these tensors is on a device."""
    q, k = torch.zeros(6, 4, 64, dtype=torch.bfloat16), torch.zeros(6, 2, 64, dtype=torch.bfloat16)
    o, lse, cu = torch.zeros_like(q), torch.zeros(4, 6), torch.zeros(3, dtype=torch.int32)
    freq = torch.zeros(32, dtype=torch.float64)
    for args in ((q.float(), k, k), (q, k.half(), k), (q, k, k[:, :1]), (q, k[..., :32], k), (q[:, 0], k, k), (q, k[:5], k), (q, k, k[:5]), (q[:3], k, k)):
        with pytest.raises(ValueError):
            nb.attention_forward(*args)
    for bad in (cu.long(), cu[None], torch.zeros(0, dtype=torch.int32)):
        with pytest.raises(ValueError, match="cu_seqlens"):
            nb.attention_forward(q, k, k, bad)
    good = dict(dout=o, out=o, lse=lse, q=q, k=k, v=k)
    for kw in (dict(dout=o.float()), dict(out=o[:5]), dict(lse=lse.double()), dict(lse=lse.T), dict(grads=(o, k, k.float())), dict(grads=(o, o, k))):
        with pytest.raises(ValueError):
            nb.attention_backward(**{**good, **kw})
    for kw in (dict(freq=freq.float()), dict(positions=torch.zeros(6)), dict(positions=torch.zeros(5, dtype=torch.int32)), dict(k=k[:5]), dict(k=k[..., :32])):
        with pytest.raises(ValueError):
            nb.rotary(**{**dict(q=q, k=k, freq=freq), **kw})


def test_binding_refuses_other_strides(L):
    args = [at(0), None, at(2), at(3), at(4), at(5), 0, 3, 4, 2, 64, 256, 512, 512, 512, 0.125, 1, 0]
    nb.nb_attention_forward(*args)  # no rows: nothing to do
    with pytest.raises(AssertionError, match="dense rows"):
        nb.nb_attention_forward(*args[:2], torch.zeros(6, 4, 64, dtype=torch.bfloat16), *args[3:])  # not on a device
    with pytest.raises(TypeError):
        nb.nb_attention_forward(*args[:-3])
    with pytest.raises(nb.NbError):
        nb.nb_attention_forward(*args[:8], 3, *args[9:])


@pytest.mark.parametrize("causal", [False, True])
def test_reference_gradients_against_differences(causal):
    g = torch.Generator().manual_seed(3)
    bounds, scale = [0, 3, 3, 7], 0.7
    q, dout = (torch.randn((8, 4, 5), generator=g, dtype=torch.float64) for _ in range(2))
    k, v = (torch.randn((8, 2, 5), generator=g, dtype=torch.float64) for _ in range(2))
    out, lse, _, _ = ref.forward(q, k, v, bounds, scale, causal)
    got, _ = ref.backward(dout, out, lse, q, k, v, bounds, scale, causal)
    h = 1e-5
    for x, grad in zip((q, k, v), got):
        for i in range(0, x.numel(), 7):
            d = torch.zeros_like(x)
            d.view(-1)[i] = h
            up, down = (ref.forward(*(t + f * d if t is x else t for t in (q, k, v)), bounds, scale, causal)[0] for f in (1, -1))
            # central differences: third derivatives times h^2, and 64-bit cancellation over h
            assert abs(((up - down) * dout).sum() / (2 * h) - grad.view(-1)[i]) < 1e-8


def test_reference_turns_back():
    g = torch.Generator().manual_seed(4)
    x, w = (torch.randn((6, 2, 24), generator=g, dtype=torch.float64) for _ in range(2))
    f, where = ref.frequencies(16, 100.0), torch.arange(6) * 5
    for half in (False, True):
        y, _ = ref.rotary(x, f, where, 1.5, half)
        back, _ = ref.rotary(w, f, where, 1.5, half, inverse=True)
        assert abs((y * w).sum() - (x * back).sum()) < 1e-12  # the gradient's way back is the transposed turn
        assert (ref.rotary(y, f, where, 1 / 1.5, half, inverse=True)[0][..., :16] - x[..., :16]).abs().max() < 1e-14
