"""Layer norm with its residual add on the GPU, against the formulas in 64 bits."""
import pytest
import torch

from paper_2609_28568_b200 import binding as nb
from norm_reference import EPS32, norm_backward, norm_forward
from parity import Guarded

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32
TYPES = {"bf16": (BF16, nb.DTYPE_BF16), "f32": (F32, nb.DTYPE_F32)}
HALF_STEP = torch.finfo(BF16).eps / 2   # one rounding to bf16, relative
# (rows, C): one row, partial blocks, one vector, rows that end inside a warp's, a block's and the widest team's vectors
SIZES = [(1, 8), (1, 768), (2, 64), (7, 248), (8, 768), (9, 256), (33, 264), (5, 520), (127, 776), (64, 1024), (3, 1032), (12, 2048),
         (5, 2056), (40, 4096), (7, 4104), (6, 8192), (1003, 776), (2500, 768)]


@pytest.fixture(autouse=True)
def _status_clean():
    yield
    nb.nb_check_status()


def rand(seed, shape, std=1.0, mean=0.0, dtype=BF16):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV).mul_(std).add_(mean).to(dtype)


def within(x, ref, bound, name):
    err = (x.double() - ref).abs()
    assert torch.isfinite(x.double()).all(), name
    worst = (err - bound).max().item()
    assert worst <= 0, f"{name}: {int((err > bound).sum())} of {err.numel()} values past the bound, by {worst:.3e} at most"


def forward_bounds(s, r, w, b, C):
    """What 32-bit arithmetic may be off by, before the rounding of the output. A sum over a row adds at most 64 times in sequence
    (32 elements of a thread and the shuffles, or 16 and 9 + 8 across warps), so the mean is off by 64 e mean|s|, the
    variance (of deviations from that mean) by 66 e of itself plus the mean's error squared, rstd by half that and its own
    three roundings; then four roundings to the output."""
    e = EPS32 / 2
    dmean = 64 * e * s.abs().mean(1, keepdim=True)
    xh = r["xh"].abs()
    drstd = 0.5 * (66 * e + (dmean * r["rstd"]) ** 2) + 3 * e
    slack = (dmean * r["rstd"] + xh * (drstd + 4 * e)) * w.abs()
    if b is not None:
        slack = slack + e * b.abs()
    return dmean, drstd * r["rstd"], slack


@pytest.mark.parametrize("stream", ["bf16", "f32"])
@pytest.mark.parametrize("rows,C", SIZES)
def test_forward_every_element(rows, C, stream):
    dtype, code = TYPES[stream]
    x, br = rand(1, (rows, C), 1.5, 0.3, dtype), rand(2, (rows, C), 0.7)
    w, b = rand(3, (C,), 0.2, 1.0), rand(4, (C,), 0.1)
    for branch, bias, stats in ((br, b, True), (None, b, True), (br, None, False), (None, None, False)):
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


def run_backward(rows, C, stream, dres, copy, accumulate, seed=10, w_mean=1.0):
    dtype, code = TYPES[stream]
    x, w = rand(seed, (rows, C), 1.5, 0.3, dtype), rand(seed + 1, (C,), 0.2, w_mean)
    dout = rand(seed + 2, (rows, C), 1e-3)
    res = rand(seed + 3, (rows, C), 1e-3, 0.0, dtype) if dres else None
    f = norm_forward(x.double(), w.double(), None, 1e-5)
    mean, rstd = f["mean"].float().view(-1), f["rstd"].float().view(-1)
    before = (rand(seed + 4, (C,), 0.5, 0.0, F32), rand(seed + 5, (C,), 0.5, 0.0, F32))
    dinp, db16 = Guarded((rows, C), dtype), Guarded((rows, C), BF16) if copy else None
    dw, db = Guarded((C,), F32), Guarded((C,), F32)
    dw.t.copy_(before[0])
    db.t.copy_(before[1])
    ws = Guarded((nb.nb_layernorm_workspace(rows, C) // 4,), F32)
    nb.nb_layernorm_backward(dinp.t, db16.t if copy else None, dw.t, db.t, dout, res, x, mean, rstd, w, rows, C, int(accumulate), code,
                             ws.t, ws.t.numel() * 4)
    for name, t in (("dinp", dinp), ("dbranch", db16), ("dweight", dw), ("dbias", db), ("workspace", ws)):
        if t is not None:
            t.check(name)
    r = norm_backward(dout.double(), x.double(), mean.double()[:, None], rstd.double()[:, None], w.double(),
                      None if res is None else res.double())
    # 32-bit arithmetic: the two row means add 64 times in sequence, xh takes two roundings, g one; then five operations
    # to dx
    e = EPS32 / 2
    xh = r["xh"].abs()
    dxh = 2 * e * xh
    g = r["g"].abs()
    m1, m2 = g.mean(1, keepdim=True), (g * (xh + dxh)).mean(1, keepdim=True)
    d2 = 68 * e * m2 + (g * dxh).mean(1, keepdim=True)
    slack = rstd.double()[:, None] * (e * g + 66 * e * m1 + xh * d2 + dxh * m2 + 5 * e * (g + m1 + xh * m2))
    if res is not None:
        slack = slack + e * (res.double().abs() + r["dinp"].abs())
    step = HALF_STEP if dtype == BF16 else e
    within(dinp.t, r["dinp"], step * (r["dinp"].abs() + slack) + slack, "dinp")
    if copy:
        within(db16.t, r["dinp"], HALF_STEP * (r["dinp"].abs() + slack) + slack, "dbranch")
    # a column's sum: the rows of a team, then eight warps, then every eighth of the blocks and eight again
    adds = 64 + rows // 148
    for name, got, ref, terms, old in (("dweight", dw.t, r["dweight"], dout.double().abs() * xh, before[0]),
                                       ("dbias", db.t, r["dbias"], dout.double().abs(), before[1])):
        bound = adds * e * terms.sum(0)
        if name == "dweight":
            bound = bound + (dout.double().abs() * dxh).sum(0)
        if accumulate:
            ref = ref + old.double()
            bound = bound + e * ref.abs()
        within(got, ref, bound + e * ref.abs(), name)
    return dinp.t, dw.t, db.t


@pytest.mark.parametrize("stream", ["bf16", "f32"])
@pytest.mark.parametrize("rows,C", SIZES)
def test_backward_every_element(rows, C, stream):
    run_backward(rows, C, stream, dres=True, copy=True, accumulate=False)
    run_backward(rows, C, stream, dres=False, copy=False, accumulate=True, seed=30)


def test_many_short_rows_and_the_training_batch():
    run_backward(70001, 8, "bf16", True, False, True)
    run_backward(16384, 768, "bf16", True, False, True)
    run_backward(5001, 4096, "f32", True, True, False)


def test_backward_gives_the_same_bits_every_time_and_on_two_streams_at_once():
    first = run_backward(3000, 768, "bf16", True, False, False)
    again = run_backward(3000, 768, "bf16", True, False, False)
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    x, w, dout = rand(1, (3000, 768), 1.0), rand(2, (768,), 0.2, 1.0), rand(3, (3000, 768), 1e-3)
    out, _, mean, rstd = nb.layernorm_forward(x, w)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for s in streams:  # each call has a workspace of its own
        with torch.cuda.stream(s):
            for _ in range(5):
                got.append(nb.layernorm_backward(dout, x, mean, rstd, w))
    torch.cuda.synchronize()
    for g in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], g))


@pytest.mark.parametrize("stream", ["bf16", "f32"])
def test_in_place(stream):
    dtype, code = TYPES[stream]
    rows, C = 37, 1040
    x, br, w, b = rand(1, (rows, C), 1.0, 0.0, dtype), rand(2, (rows, C)), rand(3, (C,), 0.2, 1.0), rand(4, (C,), 0.1)
    out, total, mean, rstd = nb.layernorm_forward(x, w, b, branch=br)
    x2, br2 = x.clone(), br.clone()
    nb.nb_layernorm_forward(br2, x2, None, None, x2, br2, w, b, rows, C, 1e-5, code)
    assert torch.equal(x2, total) and torch.equal(br2, out)
    dout, dres = rand(5, (rows, C), 1e-3), rand(6, (rows, C), 1e-3, 0.0, dtype)
    dinp, dbranch, _, _ = nb.layernorm_backward(dout, total, mean, rstd, w, dres=dres, need_dweight=False, need_dbias=False)
    dres2, dout2 = dres.clone(), dout.clone()
    nb.nb_layernorm_backward(dres2, dout2, None, None, dout2, dres2, total, mean, rstd, w, rows, C, 0, code, None, 0)
    assert torch.equal(dres2, dinp) and torch.equal(dout2, dbranch)


def test_gradients_that_are_not_asked_for():
    rows, C = 300, 768
    x, w, dout = rand(1, (rows, C)), rand(2, (C,), 0.2, 1.0), rand(3, (rows, C), 1e-3)
    _, _, mean, rstd = nb.layernorm_forward(x, w)
    full = nb.layernorm_backward(dout, x, mean, rstd, w)
    only_w = nb.layernorm_backward(dout, x, mean, rstd, w, need_dbias=False)
    only_b = nb.layernorm_backward(dout, x, mean, rstd, w, need_dweight=False)
    assert torch.equal(only_w[2], full[2]) and only_w[3] is None
    assert torch.equal(only_b[3], full[3]) and only_b[2] is None
    assert torch.equal(only_w[0], full[0])


def test_no_rows():
    C = 64
    w, g, h = rand(1, (C,)), torch.full((C,), 3.0, device=DEV), torch.full((C,), 4.0, device=DEV)
    e = torch.empty((0, C), dtype=BF16, device=DEV)
    out, _, mean, rstd = nb.layernorm_forward(e, w)
    assert out.shape == (0, C) and mean.shape == (0,)
    one = torch.empty(8, dtype=F32, device=DEV)
    args = (one, None, g, h, one, None, one, one, one, w, 0, C)
    nb.nb_layernorm_backward(*args, 1, nb.DTYPE_BF16, None, 0)
    assert torch.all(g == 3.0) and torch.all(h == 4.0)
    nb.nb_layernorm_backward(*args, 0, nb.DTYPE_BF16, None, 0)
    assert torch.all(g == 0.0) and torch.all(h == 0.0)


def test_rows_that_are_hard():
    """Constant rows, a large common offset, tiny and huge values, and a row that holds an infinity or a NaN: it alone is lost."""
    rows, C = 9, 776
    x = rand(1, (rows, C), 1.0, 0.0, F32)
    x[1] = 2.5
    x[2] = 0.0
    x[3] += 4096.0
    x[4] *= 1e-18
    x[5] *= 1e15
    x[6, 5] = float("inf")
    x[7, 770] = float("nan")
    w, b = rand(3, (C,), 0.2, 1.0), rand(4, (C,), 0.1)
    out, _, mean, rstd = nb.layernorm_forward(x, w, b)
    fine = [0, 1, 2, 3, 4, 5, 8]
    s = x[fine].double()
    r = norm_forward(s, w.double(), b.double(), 1e-5)
    _, _, slack = forward_bounds(s, r, w.double(), b.double(), C)
    within(out[fine], r["out"], HALF_STEP * (r["out"].abs() + slack) + slack, "out")
    assert torch.isnan(out[6].float()).all() and torch.isnan(out[7].float()).all()
    assert torch.equal(out[1], b) and torch.equal(out[2], b)  # no spread: the deviations are exact zeros


def test_offsets_past_32_bits():
    """The last rows of a batch of more than 2^31 elements."""
    C = 8192
    rows = (1 << 31) // C + 5
    x = torch.zeros((rows, C), dtype=BF16, device=DEV)
    w, b = rand(3, (C,), 0.2, 1.0), rand(4, (C,), 0.1)
    tail = rand(5, (9, C), 1.5, 0.3)
    x[-9:] = tail
    out, _, mean, rstd = nb.layernorm_forward(x, w, b)
    r = norm_forward(tail.double(), w.double(), b.double(), 1e-5)
    _, _, slack = forward_bounds(tail.double(), r, w.double(), b.double(), C)
    within(out[-9:], r["out"], HALF_STEP * (r["out"].abs() + slack) + slack, "out")
    assert torch.equal(out[rows // 2], b)
    dout = torch.zeros((rows, C), dtype=BF16, device=DEV)
    dout[-9:] = rand(6, (9, C), 1e-3)
    small = nb.layernorm_backward(dout[-9:], tail, mean[-9:].clone(), rstd[-9:].clone(), w)
    dinp, _, dw, db = nb.layernorm_backward(dout, x, mean, rstd, w)
    assert torch.equal(dinp[-9:], small[0])
    # the other rows add zeros: only the order of nine terms differs
    for a, c in ((dw, small[2]), (db, small[3])):
        assert (a - c).abs().max() <= 16 * EPS32 * c.abs().max()
    assert not dinp[:100].any()


def test_captured_and_replayed_beside_an_eager_call():
    rows, C = 520, 768
    x, br, w, b = rand(1, (rows, C)), rand(2, (rows, C)), rand(3, (C,), 0.2, 1.0), rand(4, (C,), 0.1)
    dout = rand(5, (rows, C), 1e-3)

    def step():
        out, s, mean, rstd = nb.layernorm_forward(x, w, b, branch=br)
        return (out, s, *nb.layernorm_backward(dout, s, mean, rstd, w, dres=dout))

    eager = step()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            held = step()
        graphs.append((g, held))
    side = [torch.cuda.Stream() for _ in graphs]
    for _ in range(3):
        for st, (g, _) in zip(side, graphs):  # two graphs at once, each with its own workspace
            with torch.cuda.stream(st):
                g.replay()
        again = step()
    torch.cuda.synchronize()
    for got in (again, graphs[0][1], graphs[1][1]):
        assert all(torch.equal(a, c) for a, c in zip(eager, got))
