"""Attention whose blocks of rows are shared by clusters of thread blocks (few of them, with much to walk over), and whose backward
passes run side by side. Sizes are chosen by the number of thread blocks that share one: see the marks of each case."""
import math

import pytest
import torch

from paper_2609_28568_b200 import binding as nb
from test_gpu_attention import BF16, DEV, F32, Case, check, rand

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _status_clean():
    yield
    nb.nb_check_status()


@pytest.mark.parametrize("lengths,heads,kv,D,causal", [
    ([2000], 1, 1, 128, False),             # forward 4, dq 2, dk and dv 4
    ([1999], 1, 1, 120, True),
    ([3100], 1, 1, 64, True),               # 8, 2, 4
    ([3073], 1, 1, 72, False),              # one row in the last tile
    ([4100], 1, 1, 64, True),               # 8, 4, 4
    ([4097], 2, 1, 128, True),              # 4, 2, 4 of all heads' tiles
    ([9000], 1, 1, 64, True),               # 4, 2, 4
    ([700], 8, 1, 64, True),                # 2, 1, 8
    ([641], 8, 1, 128, False),
    ([700], 5, 1, 40, True),                # parts that begin and end inside a head's tiles
    ([1100], 12, 2, 96, True),
    ([1500, 3, 0, 260], 6, 2, 40, True),    # some thread blocks have nothing to do
    ([1, 1, 3000, 1], 3, 1, 128, True),
    ([900, 128, 1290], 4, 1, 8, False),
    ([310], 4, 1, 64, True),
])
def test_shared(lengths, heads, kv, D, causal):
    check(Case(lengths, heads, kv, D, seed=heads + D, first=5, pad=77, fused=D % 16 == 0), causal)


@pytest.mark.parametrize("D", [64, 128])
def test_large_scores(D):
    """Rows whose maximum grows from part to part by more than the type's range of exponentials."""
    c = Case([2300], 2, 1, D, seed=3, std=3.0)
    ramp = torch.linspace(0.2, 6.0, c.T, device=DEV)[:, None, None]
    c.k.copy_((c.k.float() * ramp).to(BF16))
    check(c, True)
    c.k.copy_((c.k.float() / ramp).to(BF16))
    c.k.copy_((c.k.float() * ramp.flip(0)).to(BF16))
    check(c, False)


@pytest.mark.parametrize("D", [64, 128])
def test_infinite_scores(D):
    """Keys of whole parts without a probability; a row that sees nothing else has no result, as without parts."""
    T = 2048
    q = rand(1, (T, 1, D)).abs()
    k = rand(2, (T, 1, D))
    v = rand(3, (T, 1, D))
    k[:600, :, 0] = -math.inf                     # scores of -infinity
    out, lse = torch.empty((T, 1, D), dtype=BF16, device=DEV), torch.empty((1, T), dtype=F32, device=DEV)
    nb.nb_attention_forward(out, lse, q, k, v, None, T, 1, 1, 1, D, D, D, D, D, D ** -0.5, False)
    x = (q[:, 0].double() @ k[600:, 0].double().T) * D ** -0.5
    want = torch.softmax(x, 1) @ v[600:, 0].double()
    assert (out[:, 0].double() - want).abs().max() <= 2.0 ** -6 * v.abs().max().double()
    assert (lse[0].double() - torch.logsumexp(x, 1)).abs().max() <= 1e-3
    nb.nb_attention_forward(out, lse, q, k, v, None, T, 1, 1, 1, D, D, D, D, D, D ** -0.5, True)
    assert torch.isnan(out[:600]).all() and torch.isfinite(out[640:]).all()


def tensors(c):
    out, lse = torch.zeros((c.T, c.heads, c.D), dtype=BF16, device=DEV), torch.zeros((c.heads, c.T), dtype=F32, device=DEV)
    grads = [torch.zeros_like(t) for t in (c.q, c.k, c.v)]
    ws = torch.empty((nb.nb_attention_workspace(c.T, c.heads),), dtype=torch.uint8, device=DEV)
    return out, lse, grads, ws


def passes(c, out, lse, grads, ws, cu, n):
    ld, wide = [t.stride(0) for t in (c.q, c.k, c.v)], c.heads * c.D
    nb.nb_attention_forward(out, lse, c.q, c.k, c.v, cu, c.T, n, c.heads, c.kv, c.D, wide, *ld, c.D ** -0.5, True)
    nb.nb_attention_backward(*grads, c.dout, out, lse, c.q, c.k, c.v, cu, c.T, n, c.heads, c.kv, c.D, *(g.stride(0) for g in grads), wide, wide, *ld,
                             c.D ** -0.5, True, ws, ws.numel())


SIZES = [([1], 12, 12, 64), ([200], 12, 12, 64), ([1000], 8, 1, 64), ([1000], 4, 4, 128), ([2000], 2, 1, 128)]


@pytest.mark.parametrize("lengths,heads,kv,D", SIZES)
def test_successors_wait_for_both_passes(lengths, heads, kv, D):
    """What follows on the stream, launched while the passes still run, reads all of their gradients; so do passes that follow with the same workspace."""
    c = Case(lengths, heads, kv, D, seed=4)
    out, lse, grads, ws = tensors(c)
    freq = torch.tensor(nb.nb_rotary_frequencies(D // 16 * 16), dtype=torch.float64, device=DEV)
    turned = [torch.zeros_like(g) for g in grads[:2]]

    def step():
        passes(c, out, lse, grads, ws, c.cu, 1)
        nb.nb_rotary(*turned, *grads[:2], freq, None, c.cu, c.T, 1, heads, kv, D, D // 16 * 16, *(t.stride(0) for t in turned),
                     *(t.stride(0) for t in grads[:2]), 1.0, nb.ROTARY_HALF, True)
    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in (*grads, *turned)]
    wrong = torch.zeros((), dtype=torch.int64, device=DEV)
    for _ in range(60):
        for t in (*grads, *turned):
            t.zero_()
        step()
        for t, w in zip((*grads, *turned), want):
            wrong += (t != w).sum()
    assert wrong.item() == 0
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            for t in (*grads, *turned):
                t.zero_()
            step()
        for _ in range(20):
            graph.replay()
            for t, w in zip((*grads, *turned), want):
                wrong += (t != w).sum()
    torch.cuda.synchronize()
    assert wrong.item() == 0


@pytest.mark.parametrize("lengths,heads,kv,D", SIZES)
def test_two_streams(lengths, heads, kv, D):
    """Passes on two streams at once, with a workspace each."""
    c = [Case(lengths, heads, kv, D, seed=s) for s in (5, 6)]
    t = [tensors(x) for x in c]
    want = []
    for x, y in zip(c, t):
        passes(x, *y, x.cu, 1)
        torch.cuda.synchronize()
        want.append([g.clone() for g in (y[0], y[1], *y[2])])
    streams = [torch.cuda.Stream() for _ in c]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(30):
        for s, x, y in zip(streams, c, t):
            with torch.cuda.stream(s):
                passes(x, *y, x.cu, 1)
    torch.cuda.synchronize()
    for y, w in zip(t, want):
        for a, b in zip((y[0], y[1], *y[2]), w):
            assert torch.equal(a, b)


def test_sequences_of_one_length():
    c = Case([1500, 1500], 1, 1, 64, seed=8)
    a, b = tensors(c), tensors(c)
    passes(c, *a, None, 2)
    passes(c, *b, c.cu, 2)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    for x, y in zip(a[2], b[2]):
        assert torch.equal(x, y)


@pytest.mark.parametrize("which", [8, 9, 10])
def test_timeout(which):
    t = [rand(i, (512, 64)) for i in range(3)]
    out, dout, dq, dk, dv = (torch.full((512, 64), 5.0, dtype=BF16, device=DEV) for _ in range(5))
    lse, ws = (torch.full((512,), 5.0, dtype=F32, device=DEV) for _ in range(2))
    nb.nb_debug_attention_timeout([*t, out, lse, dout, dq, dk, dv, ws], which, 2000)
    with pytest.raises(nb.NbError) as e:
        nb.nb_check_status()
    assert e.value.code == nb.NB_ERR_TIMEOUT and "wait id 300" in str(e.value)
    for x in (out, lse, dq, dk, dv):
        assert (x == 5.0).all()
    check(Case([2000], 1, 1, 64))  # and the device is as it was


@pytest.mark.parametrize("heads,kv,D", [(3, 3, 64), (8, 1, 64), (4, 2, 128), (12, 1, 128), (300, 300, 64)])
@pytest.mark.parametrize("causal", [True, False])
def test_one_key_alone_has_no_gradient(heads, kv, D, causal):
    """Its probability is one whatever its score. (dP and delta, summed in different orders, differ in their last bits.)"""
    lengths = [1, 1, 40, 1, 300]
    c = Case(lengths, heads, kv, D, seed=7, pad=3)
    out, lse, grads, ws = tensors(c)
    ld, wide = [t.stride(0) for t in (c.q, c.k, c.v)], c.heads * c.D
    nb.nb_attention_forward(out, lse, c.q, c.k, c.v, c.cu, c.T, 5, heads, kv, D, wide, *ld, D ** -0.5, causal)
    nb.nb_attention_backward(*grads, c.dout, out, lse, c.q, c.k, c.v, c.cu, c.T, 5, heads, kv, D, *(g.stride(0) for g in grads), wide, wide, *ld, D ** -0.5, causal,
                             ws, ws.numel())
    dq, dk, dv = grads
    for row in (0, 1, 42):
        assert (dq[row] == 0).all() and (dk[row] == 0).all()
        want = c.dout[row].double().unflatten(0, (kv, heads // kv)).sum(1)
        assert ((dv[row].double() - want).abs() <= want.abs() * 2.0 ** -8 + c.dout[row].abs().max().double() * heads * 2.0 ** -20).all()
    for row in (2, 43):
        assert (dq[row] == 0).all() == causal
