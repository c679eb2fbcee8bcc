"""Attention over packed sequences, forward and backward, against its formulas in 64 bits (bounds: attention_reference.py)."""
import math

import pytest
import torch

from paper_2609_28568_b200 import binding as nb
import attention_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def _status_clean():
    yield
    nb.nb_check_status()


def rand(seed, shape, std=1.0, dtype=BF16):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV).mul_(std).to(dtype)


def cumulated(lengths, first=0):
    b = [first]
    for m in lengths:
        b.append(b[-1] + m)
    return b


class Case:
    """Inputs of T rows, `first` before the first sequence and `pad` behind the last one; all of them NaN outside the sequences."""

    def __init__(self, lengths, heads, kv, D, seed=1, first=0, pad=0, fused=False, std=1.0):
        self.bounds = cumulated(lengths, first)
        T = self.T = self.bounds[-1] + pad
        self.heads, self.kv, self.D = heads, kv, D
        self.cu = torch.tensor(self.bounds, dtype=torch.int32, device=DEV)
        if fused:
            whole = rand(seed, (T, (heads + 2 * kv), D), std)
            self.q, self.k, self.v = whole.split([heads, kv, kv], 1)
        else:
            self.q, self.k, self.v = (rand(seed + i, (T, h, D), std) for i, h in enumerate((heads, kv, kv)))
        self.dout = rand(seed + 9, (T, heads, D), 0.1)
        for t in (self.q, self.k, self.v, self.dout):
            t[self.bounds[-1]:] = math.nan
            t[:first] = math.nan

    def outside(self, t, dim=0):
        """The rows of a result that belong to no sequence."""
        t = t if dim == 0 else t.transpose(0, dim)
        return torch.cat((t[:self.bounds[0]], t[self.bounds[-1]:]))


def within(got, want, tol, what):
    err = (got.double() - want).abs()
    assert torch.isfinite(err).all(), what
    assert (err <= tol + 1e-30).all(), (what, (err - tol).max().item(), (err / (tol + 1e-30)).max().item())


def check(c, causal=True, scale=None, backward=True):
    scale = c.D ** -0.5 if scale is None else scale
    out, lse = torch.full((c.T, c.heads, c.D), 7.0, dtype=BF16, device=DEV), torch.full((c.heads, c.T), 7.0, dtype=F32, device=DEV)
    ld = [t.stride(0) for t in (c.q, c.k, c.v)]
    nb.nb_attention_forward(out, lse, c.q, c.k, c.v, c.cu, c.T, len(c.bounds) - 1, c.heads, c.kv, c.D, c.heads * c.D, *ld, scale, causal)
    scale32 = torch.tensor(scale, dtype=F32).item()
    zeroed = [torch.nan_to_num(t) for t in (c.q, c.k, c.v, c.dout)]
    want, want_lse, tol, tol_lse = ref.forward(*zeroed[:3], c.bounds, scale32, causal)
    assert (c.outside(out) == 7.0).all() and (c.outside(lse, 1) == 7.0).all()
    rows = slice(c.bounds[0], c.bounds[-1])
    within(out[rows], want[rows], tol[rows], "out")
    within(lse[:, rows], want_lse[:, rows], tol_lse[:, rows], "lse")
    if not backward:
        return
    c.outside(out).fill_(math.nan)
    grads = [torch.full_like(t, 7.0) for t in (c.q, c.k, c.v)]
    ws = torch.full((nb.nb_attention_workspace(c.T, c.heads),), 255, dtype=torch.uint8, device=DEV)  # NaN
    nb.nb_attention_backward(*grads, c.dout, out, lse, c.q, c.k, c.v, c.cu, c.T, len(c.bounds) - 1, c.heads, c.kv, c.D, *(g.stride(0) for g in grads),
                             c.heads * c.D, c.heads * c.D, *ld, scale, causal, ws, ws.numel())
    wants, tols = ref.backward(zeroed[3], torch.nan_to_num(out), torch.nan_to_num(lse), *zeroed[:3], c.bounds, scale32, causal)
    for g, w, t, name in zip(grads, wants, tols, ("dq", "dk", "dv")):
        assert (c.outside(g) == 7.0).all(), name
        within(g[rows], w[rows], t[rows], name)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("m", [1, 2, 15, 16, 17, 127, 128, 129, 255, 256, 257, 384, 700])
def test_lengths(m, causal):
    check(Case([m], 2, 2, 64, seed=m), causal)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("D", [8, 16, 24, 40, 56, 64, 72, 96, 120, 128])
def test_widths(D, causal):
    check(Case([130, 19], 2, 1, D, seed=D, fused=True), causal)


@pytest.mark.parametrize("heads,kv", [(1, 1), (3, 3), (4, 2), (8, 1), (6, 2), (12, 12)])
@pytest.mark.parametrize("D", [64, 128])
def test_shared_heads(heads, kv, D):
    check(Case([140, 33], heads, kv, D, seed=heads, fused=True, pad=5))


@pytest.mark.parametrize("lengths", [[0], [0, 0, 5, 0], [1] * 40, [300, 0, 1, 17, 128, 513], [0, 129], [256, 256], [1, 128, 127, 255, 2], [640] + [1] * 70 + [130]])
@pytest.mark.parametrize("causal,D", [(True, 64), (False, 64), (True, 128)])
def test_packed(lengths, causal, D):
    check(Case(lengths, 4, 2, D, seed=len(lengths), first=3, pad=150), causal)


def test_many_sequences():
    """More than a warp's first look into cu_seqlens takes in, and more than two of them."""
    g = torch.Generator().manual_seed(5)
    check(Case(torch.randint(0, 4, (3000,), generator=g).tolist(), 1, 1, 32, first=1, pad=2))


def test_sequences_of_one_length():
    c = Case([130] * 3, 3, 3, 64)
    whole = nb.attention_forward(c.q, c.k, c.v, c.cu)
    even = nb.attention_forward(c.q, c.k, c.v, n=3)
    for a, b in zip(whole, even):
        assert torch.equal(a, b)
    for a, b in zip(nb.attention_backward(c.dout, *whole, c.q, c.k, c.v, c.cu), nb.attention_backward(c.dout, *whole, c.q, c.k, c.v, n=3)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("scale", [1e-3, 1.0, 3.0])
def test_scales(scale):
    """Flat rows; rows of one key, whose maximum jumps by hundreds between tiles."""
    check(Case([520], 2, 2, 64, seed=3), scale=scale, backward=scale < 2.0)


@pytest.mark.parametrize("D", [64, 128])
def test_rising_maxima(D):
    """The largest score of every row comes in its last tile, in the first, or by steps that ask for no rescaling."""
    for step in (0.0, 0.02, 0.4, -0.4):
        c = Case([900], 1, 1, D, seed=7, std=0.3)
        c.q[:, :, 0], c.k[:, 0, 0] = 4.0, torch.arange(900, device=DEV) * step
        check(c)
        check(c, causal=False)


def test_without_statistics():
    c = Case([300, 77], 4, 2, 64)
    out, lse = nb.attention_forward(c.q, c.k, c.v, c.cu)
    alone, none = nb.attention_forward(c.q, c.k, c.v, c.cu, train=False)
    assert none is None and torch.equal(out, alone)


def test_same_bits_whatever_else_is_in_the_batch():
    c = Case([200, 150, 90], 4, 2, 64, seed=11)
    out, lse = nb.attention_forward(c.q, c.k, c.v, c.cu)
    grads = nb.attention_backward(c.dout, out, lse, c.q, c.k, c.v, c.cu)
    again = nb.attention_backward(c.dout, out, lse, c.q, c.k, c.v, c.cu)
    assert all(torch.equal(a, b) for a, b in zip(grads, again))
    a, b = c.bounds[1:3]
    q, k, v, dout = (t[a:b].contiguous() for t in (c.q, c.k, c.v, c.dout))
    o, s = nb.attention_forward(q, k, v)
    assert torch.equal(o, out[a:b]) and torch.equal(s, lse[:, a:b])
    for x, y in zip(grads, nb.attention_backward(dout, o, s, q, k, v)):
        assert torch.equal(x[a:b], y)


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
def test_other_sequences_are_not_reached(value):
    """What one sequence holds changes no bit of its neighbours, before and behind."""
    c = Case([150, 70, 140], 2, 1, 64, seed=13)
    out, lse = nb.attention_forward(c.q, c.k, c.v, c.cu)
    grads = nb.attention_backward(c.dout, out, lse, c.q, c.k, c.v, c.cu)
    for t in (c.q, c.k, c.v, c.dout):
        t[150:220] = value
    out2, lse2 = nb.attention_forward(c.q, c.k, c.v, c.cu)
    grads2 = nb.attention_backward(c.dout, out2, lse2, c.q, c.k, c.v, c.cu)
    for rows in (slice(0, 150), slice(220, 360)):
        assert torch.equal(out[rows], out2[rows]) and torch.equal(lse[:, rows], lse2[:, rows])
        for a, b in zip(grads, grads2):
            assert torch.equal(a[rows], b[rows])


def test_later_rows_are_not_seen():
    c = Case([400], 2, 2, 64, seed=17)
    out, lse = nb.attention_forward(c.q, c.k, c.v)
    for t in (c.k, c.v):
        t[250:] = 100.0
    out2, lse2 = nb.attention_forward(c.q, c.k, c.v)
    assert torch.equal(out[:250], out2[:250]) and torch.equal(lse[:, :250], lse2[:, :250])
    assert not torch.equal(out[250:], out2[250:])


def test_infinite_scores():
    """Keys that no query can see for their infinite distance: they have no part in the result, wherever they stand."""
    c = Case([200], 1, 1, 64, seed=18)
    c.q[:, 0, 0] = 1.0
    want, lse = nb.attention_forward(c.q[150:], c.k[150:], c.v[150:], causal=False)
    c.k[:150, 0] = 0.0
    c.k[:150, 0, 0] = -math.inf
    got, lse2 = nb.attention_forward(c.q, c.k, c.v, causal=False)
    # the sums are made up of the same numbers, in other pieces: probabilities, lse and the result each rounded anew
    e, tol = (got[150:].double() - want.double()).abs(), 4 * ref.U16 * (want.double().abs() + c.v[150:].double().abs().mean(0))
    assert (e <= tol).all() and (lse2[:, 150:] - lse).abs().max() < 1e-5


def test_offsets_past_32_bits():
    """Rows so far apart that the last lies 5 GB behind the first."""
    ld, T = 1 << 23, 300
    far = torch.empty(T * ld, dtype=BF16, device=DEV).view(T, ld)
    c = Case([170, 130], 2, 1, 64, seed=19)
    q, k, v, out, dq, dk, dv, dout = (far[:, i * 128:i * 128 + 128] for i in range(8))
    k, v, dk, dv = (t[:, :64] for t in (k, v, dk, dv))
    for view, t in ((q, c.q), (k, c.k), (v, c.v), (dout, c.dout)):
        view.copy_(t.flatten(1))
    lse = torch.empty((2, T), dtype=F32, device=DEV)
    nb.nb_attention_forward(out, lse, q, k, v, c.cu, T, 2, 2, 1, 64, ld, ld, ld, ld, 0.125, 1)
    ws = torch.empty(nb.nb_attention_workspace(T, 2), dtype=torch.uint8, device=DEV)
    nb.nb_attention_backward(dq, dk, dv, dout, out, lse, q, k, v, c.cu, T, 2, 2, 1, 64, *(ld,) * 8, 0.125, 1, ws, ws.numel())
    o, s = nb.attention_forward(c.q, c.k, c.v, c.cu, scale=0.125)
    assert torch.equal(o.flatten(1), out) and torch.equal(s, lse)
    for got, want in zip((dq, dk, dv), nb.attention_backward(c.dout, o, s, c.q, c.k, c.v, c.cu, scale=0.125)):
        assert torch.equal(got, want.flatten(1))


@pytest.mark.parametrize("bounds", [[0, 400], [-5, 100, 300], [0, 200, 100, 300], [0, 1 << 30, 300], [300, 0], [0, 300, -(1 << 31)], [1 << 30, 1 << 30, 1 << 30]])
def test_bad_bounds_are_reported(bounds):
    """Sequences that fall or leave the tensors are cut: nothing outside is touched, and the status says so."""
    T, guard = 300, 64
    whole = [torch.full((T + 2 * guard, 2, 64), 3.0, dtype=BF16, device=DEV) for _ in range(8)]
    q, k, v, out, dq, dk, dv, dout = (t[guard:-guard] for t in whole)
    stats = torch.full((2, T), 3.0, dtype=F32, device=DEV)
    cu = torch.tensor(bounds, dtype=torch.int32, device=DEV)
    n = len(bounds) - 1
    nb.nb_attention_forward(out, stats, q, k, v, cu, T, n, 2, 2, 64, 128, 128, 128, 128, 0.125, 1)
    with pytest.raises(nb.NbError) as e:
        nb.nb_check_status()
    assert e.value.code == nb.NB_ERR_INVALID_ARG and "cu_seqlens" in str(e.value)
    ws = torch.empty(nb.nb_attention_workspace(T, 2), dtype=torch.uint8, device=DEV)
    nb.nb_attention_backward(dq, dk, dv, dout, out, stats, q, k, v, cu, T, n, 2, 2, 64, *(128,) * 8, 0.125, 1, ws, ws.numel())
    with pytest.raises(nb.NbError) as e:
        nb.nb_check_status()
    assert e.value.code == nb.NB_ERR_INVALID_ARG
    for t in whole:
        assert (t[:guard] == 3.0).all() and (t[-guard:] == 3.0).all()


def test_nothing_to_do():
    q = torch.empty((0, 2, 64), dtype=BF16, device=DEV)
    out, lse = nb.attention_forward(q, q, q)
    assert out.shape == q.shape and lse.shape == (2, 0)
    assert all(g.shape == q.shape for g in nb.attention_backward(out, out, lse, q, q, q))
    c = Case([5], 2, 2, 64)
    out, lse = nb.attention_forward(c.q, c.k, c.v, torch.zeros(1, dtype=torch.int32, device=DEV))
    assert (out == 0).all() and (lse == 0).all()


def test_on_another_stream_and_in_graphs():
    """Two captured passes with workspaces of their own, replayed at the same time on changed inputs."""
    cases = [Case([260, 40], 4, 2, 64, seed=23), Case([100, 333], 4, 2, 64, seed=29)]
    graphs, held = [], []
    for c in cases:
        for _ in range(1):  # first use of every kernel: attributes are set outside the capture
            o, s = nb.attention_forward(c.q, c.k, c.v, c.cu)
            nb.attention_backward(c.dout, o, s, c.q, c.k, c.v, c.cu)
    torch.cuda.synchronize()
    for c in cases:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            o, s = nb.attention_forward(c.q, c.k, c.v, c.cu)
            held.append((o, s, *nb.attention_backward(c.dout, o, s, c.q, c.k, c.v, c.cu)))
        graphs.append(g)
    for c in cases:
        for t in (c.q, c.k, c.v, c.dout):
            t.mul_(-0.5)
    streams = [torch.cuda.Stream() for _ in cases]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for c, h in zip(cases, held):
        with torch.cuda.stream(side):
            o, s = nb.attention_forward(c.q, c.k, c.v, c.cu)
            grads = nb.attention_backward(c.dout, o, s, c.q, c.k, c.v, c.cu)
        side.synchronize()
        for a, b in zip(h, (o, s, *grads)):
            assert torch.equal(a, b)


def test_gradients_against_differences():
    """Along a direction, on scores so flat that roundings of the probabilities matter little."""
    c = Case([150], 2, 1, 64, seed=31)
    out, lse = nb.attention_forward(c.q, c.k, c.v)
    grads = nb.attention_backward(c.dout, out, lse, c.q, c.k, c.v)
    for i, (x, g) in enumerate(zip((c.q, c.k, c.v), grads)):
        d = rand(40 + i, x.shape, 1.0, F32).double()
        h = 1e-4
        up, down = (ref.forward(*(t.double() + f * h * d if t is x else t.double() for t in (c.q, c.k, c.v)), [0, 150], 0.125, True)[0] for f in (1, -1))
        want = ((up - down) * c.dout.double()).sum() / (2 * h)
        # the gradient's roundings (out in delta, p, ds, the result: 2^-8 each at most) are independent over the elements of the sum
        assert abs((g.double() * d).sum() - want) <= 6 * 4 * ref.U16 * (g.double() * d).norm()


@pytest.mark.parametrize("which", [0, 1, 2])
def test_timeout(which):
    t = [rand(i, (256, 64)) for i in range(3)]
    out, dout, dq, dk, dv = (torch.full((256, 64), 5.0, dtype=BF16, device=DEV) for _ in range(5))
    lse, ws = (torch.full((256,), 5.0, dtype=F32, device=DEV) for _ in range(2))
    nb.nb_debug_attention_timeout([*t, out, lse, dout, dq, dk, dv, ws], which, 2000)
    with pytest.raises(nb.NbError) as e:
        nb.nb_check_status()
    assert e.value.code == nb.NB_ERR_TIMEOUT and "wait id 300" in str(e.value)
    for x in (out, lse, dq, dk, dv):
        assert (x == 5.0).all()
    check(Case([200], 1, 1, 64))  # and the device is as it was
