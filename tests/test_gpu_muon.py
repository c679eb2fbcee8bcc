"""The orthogonalised update and its application on the GPU, against the formulas in 64 bits."""
import pytest
import torch

from paper_2609_28568_b200 import binding as nb
from norm_reference import EPS32, newton_schulz
from parity import Guarded

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def _status_clean():
    yield
    nb.nb_check_status()


def rand(seed, shape, std=1.0, dtype=F32):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV).mul_(std).to(dtype)


COEFFICIENTS = nb.MUON_COEFFICIENTS


def gradients(seed, n, R, C, std, dtype=F32):
    """A few strong directions over noise of full rank."""
    r = min(8, R, C)
    return [(rand(seed + 3 * i, (R, r)) @ rand(seed + 3 * i + 1, (r, C)) * (0.3 * std / r ** 0.5) +
             rand(seed + 3 * i + 2, (R, C), std)).to(dtype) for i in range(n)]


def close(got, ref, name):
    """Roundings to fp16 have an rms of at most 2^-11 / sqrt(3) = 2.8e-4 of a value. Each of the five iterates, S and P is rounded once and,
    as signal and error grow alike from there, each adds as much: sqrt(15) * 2.8e-4 = 1.1e-3. The result's rounding to bf16
    adds an rms of at most 2^-8 / sqrt(3) = 2.3e-3: together 2.5e-3 over the matrix. Single rows and columns, of which there are
    many and some short, may be off by a few times that; one that is wrong is off by about 1."""
    err = got.double() - ref
    whole = (err.norm() / ref.norm()).item()
    assert whole <= 4e-3, f"{name}: off by {whole:.2e}"
    for d in (0, 1):
        off, size = err.norm(dim=d), ref.norm(dim=d)
        assert not off[size == 0].any(), f"{name}: rows or columns of zeros"
        worst = (off[size > 0] / size[size > 0]).max().item()
        assert worst <= 1.6e-2, f"{name}: a {'column' if d == 0 else 'row'} is off by {worst:.2e}"


# (matrices, rows, columns): tiles of 64 (a few matrices), of 128, of 256 (many), wide, tall and square ones, sides that end inside a
# tile, inside a k-block and inside a piece of a tile; more matrices than one launch takes; several short tiles of a phase per
# block, which loads far ahead of what it computes
SHAPES = [(28, 64, 2304), (28, 2304, 64), (32, 128, 1024), (32, 1024, 72), (32, 8, 4096), (24, 776, 520), (18, 520, 776), (3, 520, 200), (2, 72, 776), (1, 8, 8), (1, 64, 64), (2, 16, 264), (2, 264, 16), (3, 136, 72), (1, 128, 256), (2, 256, 128), (1, 776, 1416),
          (2, 1416, 776), (3, 768, 768), (1, 3072, 768), (33, 72, 136), (1, 2056, 2048), (12, 768, 768), (5, 264, 1000), (28, 520, 264)]


def run_update(n, R, C, dtype, nesterov, momentum, steps=5, std=1e-4, mu=0.95, seed=50):
    grad = gradients(seed, n, R, C, std, dtype)
    old = gradients(seed + 1000, n, R, C, 3 * std) if momentum else None
    mom = [Guarded((R, C), F32) for _ in range(n)] if momentum else None
    out = [Guarded((R, C), BF16) for _ in range(n)]
    ws = Guarded((nb.nb_muon_workspace(n, R, C) // 4 + 32,), F32)
    at = ws.t[(-ws.t.data_ptr() % 128) // 4:]  # on the boundary that the call asks for
    for i in range(n if momentum else 0):
        mom[i].t.copy_(old[i])
    nb.nb_muon_update([o.t for o in out], [m.t for m in mom] if momentum else None, grad, n, R, C, mu, int(nesterov), steps,
                      *COEFFICIENTS, 1e-7, nb.DTYPE_F32 if dtype == F32 else nb.DTYPE_BF16, at, at.numel() * 4)
    ws.check("workspace")
    mu32 = torch.tensor(mu, dtype=F32).double().item()
    refs = []
    for i in range(n):
        g = grad[i].double()
        m = mu32 * old[i].double() + g if momentum else g
        v = g + mu32 * m if nesterov and momentum else m
        refs.append(newton_schulz(v, steps, COEFFICIENTS, 1e-7))
        out[i].check("update")
        if momentum:
            mom[i].check("momentum")
            assert ((mom[i].t.double() - m).abs() <= EPS32 / 2 * m.abs()).all(), i  # one rounding
    return [o.t for o in out], refs


@pytest.mark.parametrize("n,R,C", SHAPES)
def test_update_every_matrix(n, R, C):
    for dtype, nesterov, momentum in ((F32, True, True), (BF16, False, True), (F32, True, False)):
        for i, (got, ref) in enumerate(zip(*run_update(n, R, C, dtype, nesterov, momentum))):
            close(got, ref, f"{n} x [{R}, {C}], {dtype}, matrix {i}")


@pytest.mark.parametrize("R,C", [(264, 520), (520, 264)])
@pytest.mark.parametrize("steps", [0, 1, 2, 7])
def test_other_numbers_of_steps(R, C, steps):
    for got, ref in zip(*run_update(2, R, C, F32, True, True, steps=steps)):
        close(got, ref, f"{steps} steps")


@pytest.mark.parametrize("std", [1e-30, 1e-12, 1e12, 1e30])
def test_gradients_of_any_size(std):
    """eps is 1e-7: what is far smaller comes out smaller, by the formula."""
    for got, ref in zip(*run_update(1, 136, 264, F32, False, False, std=std)):
        if std > 1e-20:
            close(got, ref, f"std {std}")
        else:  # x below fp16's smallest values: the update vanishes beside an orthogonal one
            assert got.double().abs().max() <= 1e-6 and ref.abs().max() <= 1e-6


@pytest.mark.parametrize("R,C", [(256, 512), (768, 520)])
def test_steeply_falling_singular_values(R, C):
    """Singular values 1 / j^2. The first rounding to fp16 leaves noise of 2^-11 / sqrt(3) of each value of x, whose norm is one: spread over the
    matrix its singular values reach 2.8e-4 (1 / sqrt(R) + 1 / sqrt(C)), and five steps multiply small ones by 485. Beside an update whose
    singular values are of the order of one that is up to 1.5e-2 (256 x 512) of its norm; the later iterates' roundings,
    multiplied by 140, 41, 12 and 3.4, add less than as much again."""
    m = min(R, C)
    u, v = torch.linalg.qr(rand(60, (R, m), dtype=torch.float64))[0], torch.linalg.qr(rand(61, (C, m), dtype=torch.float64))[0]
    g = (u * torch.arange(1, m + 1, device=DEV, dtype=torch.float64) ** -2 @ v.T).float()
    got, ref = nb.muon_update([g])[0], newton_schulz(g.double(), 5, COEFFICIENTS, 1e-7)
    noise = 485 * 2 ** -11 / 3 ** 0.5 * (R ** -0.5 + C ** -0.5)
    assert ((got.double() - ref).norm() / ref.norm()).item() <= 2 * noise + 2.5e-3


def test_matrices_do_not_touch_each_other():
    n, R, C = 4, 264, 136
    grad = gradients(70, n, R, C, 1e-3)
    good = nb.muon_update(grad)
    grad[1] = torch.zeros_like(grad[1])
    grad[2][5, 7] = float("nan")
    got = nb.muon_update(grad)
    assert torch.equal(got[0], good[0]) and torch.equal(got[3], good[3])
    assert not got[1].any() and torch.isnan(got[2].float()).all()
    grad[2][5, 7] = float("inf")
    got = nb.muon_update(grad)
    assert torch.equal(got[0], good[0]) and torch.equal(got[3], good[3]) and torch.isnan(got[2].float()).all()


def test_singular_values_come_near_one():
    got = nb.muon_update(gradients(80, 2, 768, 1536, 1e-4))
    for u in got:
        s = torch.linalg.svdvals(u.double())
        assert s.min() > 0.6 and s.max() < 1.25


def test_update_gives_the_same_bits_every_time_on_streams_and_in_graphs():
    grad = gradients(90, 3, 776, 520, 1e-4)
    first = nb.muon_update(grad)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            held = nb.muon_update(grad)
        graphs.append((g, held))
    streams = [torch.cuda.Stream() for _ in graphs]
    got = []
    for _ in range(3):
        for st, (g, _) in zip(streams, graphs):  # each graph has a workspace of its own
            with torch.cuda.stream(st):
                g.replay()
        got.append(nb.muon_update(grad))
    torch.cuda.synchronize()
    for other in got + [held for _, held in graphs]:
        assert all(torch.equal(a, b) for a, b in zip(first, other))


@pytest.mark.parametrize("copy", [True, False])
@pytest.mark.parametrize("n,count", [(1, 1), (2, 7), (3, 8), (1, 13), (5, 4099), (33, 776), (2, 1416 * 776), (12, 768 * 2304)])
def test_apply_every_element(n, count, copy):
    decay, step = 0.998, 0.02
    start = [rand(10 + i, (count,), 0.02) for i in range(n)]
    update = [rand(200 + i, (count,), 0.05, BF16) for i in range(n)]
    master = [Guarded((count,), F32) for _ in range(n)]
    weight = [Guarded((count,), BF16) for _ in range(n)] if copy else None
    for m, s in zip(master, start):
        m.t.copy_(s)
    nb.nb_muon_apply([m.t for m in master], [w.t for w in weight] if copy else None, update, n, count, decay, step)
    d32, s32 = (torch.tensor(v, dtype=F32).double().item() for v in (decay, step))  # the scalars arrive in 32 bits
    for i in range(n):
        ref = d32 * start[i].double() - s32 * update[i].double()
        # decay * master is rounded, then the difference: half a step each
        bound = EPS32 / 2 * (d32 * start[i].double().abs() + ref.abs() * (1 + EPS32))
        assert ((master[i].t.double() - ref).abs() <= bound).all(), i
        master[i].check("master")
        if copy:
            assert torch.equal(weight[i].t, master[i].t.to(BF16)), i
            weight[i].check("weight")


def test_apply_keeps_what_is_not_finite_where_it_is():
    m = rand(1, (4096,), 0.02)
    u = rand(2, (4096,), 0.05, BF16)
    m[5], u[6], u[4095] = float("inf"), float("nan"), float("-inf")
    w = torch.empty(4096, dtype=BF16, device=DEV)
    nb.nb_muon_apply([m], [w], [u], 1, 4096, 0.998, 0.02)
    bad = ~torch.isfinite(m)
    assert bad.nonzero().view(-1).tolist() == [5, 6, 4095] and torch.equal(~torch.isfinite(w), bad)
    assert m[5] == float("inf") and torch.isnan(m[6]) and m[4095] == float("inf")


def test_apply_past_32_bits():
    count = (1 << 31) + 13
    m = torch.zeros(count, dtype=F32, device=DEV)
    u = torch.zeros(count, dtype=BF16, device=DEV)
    u[-9:] = torch.arange(1, 10, device=DEV)
    u[5] = 3.0
    nb.nb_muon_apply([m], None, [u], 1, count, 0.5, 2.0)
    assert torch.equal(m[-9:], -2.0 * torch.arange(1, 10, device=DEV).float()) and m[5] == -6.0
    assert int((m != 0).sum()) == 10


def test_workspace_past_32_bits():
    """Thirty-two matrices whose iterates take 4 GB each way: the first one again as the last gives the same bits."""
    grad = gradients(95, 2, 8192, 8192, 1e-4, BF16)
    grad = grad[:1] + [grad[1].clone() for _ in range(30)] + [grad[0].clone()]
    update = nb.muon_update(grad, steps=2)
    assert torch.equal(update[0], update[31]) and torch.equal(update[1], update[30]) and not torch.equal(update[0], update[1])
    close(update[31], newton_schulz(grad[31].double(), 2, COEFFICIENTS, 1e-7), "the last")
