"""The operators of a training step together: norm -> fc (GELU) -> proj -> add and norm -> head with loss, backward through all of
them over two micro-steps, and the update of the weights, against 64-bit autograd and the update's formula."""
import pytest
import torch

from paper_2609_28568_b200 import binding as nb
from norm_reference import newton_schulz
from test_gpu_muon import close

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(autouse=True)
def _status_clean():
    yield
    nb.nb_check_status()


def rand(seed, shape, std, dtype=BF16, mean=0.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV).mul_(std).add_(mean).to(dtype)


class Model:
    """One MLP block between two norms, and a head of Vp columns, V of them real."""

    def __init__(self, C, H, Vp, stream):
        self.C, self.H, self.Vp, self.V, self.stream = C, H, Vp, Vp - 7, stream
        self.master = {"fc": rand(1, (H, C), 0.05, F32), "proj": rand(2, (C, H), 0.05, F32), "head": rand(3, (Vp, C), 0.05, F32)}
        self.w = {k: v.to(BF16) for k, v in self.master.items()}
        self.w |= {"fc_b": rand(4, (H,), 0.1), "proj_b": rand(5, (C,), 0.1), "n1": rand(6, (C,), 0.2, mean=1.0), "n1_b": rand(7, (C,), 0.1),
                   "n2": rand(8, (C,), 0.2, mean=1.0), "n2_b": rand(9, (C,), 0.1)}
        self.grad = {k: torch.zeros(v.shape, dtype=F32, device=DEV) for k, v in self.w.items()}
        self.momentum = {k: torch.zeros_like(v) for k, v in self.master.items()}

    def micro_step(self, x, targets, scale, accumulate):
        """Loss per row, the gradient of x; gradients of all parameters into self.grad."""
        w, g, BT = self.w, self.grad, x.shape[0]
        y1, _, m1, r1 = nb.layernorm_forward(x, w["n1"], w["n1_b"])
        h, pre = nb.linear_forward(y1, w["fc"], w["fc_b"], nb.ACT_GELU)
        z, _ = nb.linear_forward(h, w["proj"], w["proj_b"])
        y2, s, m2, r2 = nb.layernorm_forward(x, w["n2"], w["n2_b"], branch=z)
        logits = torch.empty((BT, self.Vp), dtype=BF16, device=DEV)
        loss, lse = torch.empty(BT, dtype=F32, device=DEV), torch.empty(BT, dtype=F32, device=DEV)
        nb.nb_lm_head_ce_forward(logits, loss, lse, y2, w["head"], targets, BT, self.C, self.Vp, self.V)
        nb.nb_ce_backward(logits, logits, lse, targets, scale, BT, self.Vp, self.V)
        acc = dict(accumulate=accumulate)
        dy2, _, _ = nb.linear_backward(logits, y2, w["head"], dweight=g["head"], need_dbias=False, **acc)
        ds, dz, _, _ = nb.layernorm_backward(dy2, s, m2, r2, w["n2"], dweight=g["n2"], dbias=g["n2_b"], **acc)
        dpre, _, _ = nb.linear_backward(dz, h, w["proj"], inp_pre_act=pre, dweight=g["proj"], dbias=g["proj_b"], **acc)
        dy1, _, _ = nb.linear_backward(dpre, y1, w["fc"], dweight=g["fc"], dbias=g["fc_b"], **acc)
        dx, _, _, _ = nb.layernorm_backward(dy1, x, m1, r1, w["n1"], dres=ds, dweight=g["n1"], dbias=g["n1_b"], **acc)
        return loss, dx

    def update(self, lr=0.02):
        """fc and proj^T have one shape, and the head's: one call each, as a program groups its weights by shape."""
        ups = {}
        for names in (("fc",), ("proj",), ("head",)):
            got = nb.muon_update([self.grad[k] for k in names], [self.momentum[k] for k in names])
            ups |= dict(zip(names, got))
            nb.nb_muon_apply([self.master[k] for k in names], [self.w[k] for k in names], got, len(names), got[0].numel(), 1.0 - 0.1 * lr, lr)
        return ups

    def reference(self, batches, scale):
        """(losses, gradients of x, gradients of the parameters) in 64 bits."""
        p = {k: v.double().requires_grad_() for k, v in self.w.items()}
        norm = lambda t, k: torch.nn.functional.layer_norm(t, (self.C,), p[k], p[k + "_b"], 1e-5)  # noqa: E731
        losses, dxs = [], []
        for x, t in batches:
            xd = x.double().requires_grad_()
            h = torch.nn.functional.gelu(norm(xd, "n1") @ p["fc"].T + p["fc_b"], approximate="tanh")
            logits = norm(xd + h @ p["proj"].T + p["proj_b"], "n2") @ p["head"].T
            loss = torch.nn.functional.cross_entropy(logits[:, :self.V], t.long(), reduction="none")
            (loss.sum() * scale).backward()
            losses.append(loss.detach())
            dxs.append(xd.grad)
        return losses, dxs, {k: v.grad for k, v in p.items()}


def rel(a, b):
    return ((a.double() - b).norm() / b.norm()).item()


# Ten roundings to bf16 lie between the input and a gradient (norms, activation, sum, logits, their gradient, and the way back), each with an
# rms of at most 2^-8 / sqrt(3) = 2.3e-3 of its values: 7.2e-3 where all of them reach the result alike. Twice that, and the
# derivative of the approximated tanh.
TOL = 1.5e-2


@pytest.mark.parametrize("stream", [BF16, F32])
@pytest.mark.parametrize("BT,C,H,Vp", [(96, 64, 256, 512), (301, 264, 520, 1000)])
def test_training_steps(BT, C, H, Vp, stream):
    model = Model(C, H, Vp, stream)
    batches = [(rand(20 + i, (BT, C), 1.0, stream), torch.randint(0, Vp - 7, (BT,), dtype=torch.int32, device=DEV)) for i in range(2)]
    for step in range(2):  # the second with the updated weights
        scale = 1.0 / (2 * BT)
        losses, dxs, grads = model.reference(batches, scale)
        for i, (x, t) in enumerate(batches):
            loss, dx = model.micro_step(x, t, scale, accumulate=i > 0)
            assert dx.dtype == stream
            assert rel(loss, losses[i]) <= TOL and rel(dx, dxs[i]) <= TOL, (step, i)
        for k, g in grads.items():
            assert rel(model.grad[k], g) <= TOL, (step, k, rel(model.grad[k], g))
        before = {k: (v.clone(), model.momentum[k].clone()) for k, v in model.master.items()}
        ups = model.update()
        for k, u in ups.items():
            mu = torch.tensor(0.95, dtype=F32).double()
            m = mu * before[k][1].double() + model.grad[k].double()
            close(u, newton_schulz(model.grad[k].double() + mu * m, 5, nb.MUON_COEFFICIENTS, 1e-7), k)
            want = (1.0 - 0.1 * 0.02) * before[k][0].double() - 0.02 * u.double()
            assert ((model.master[k].double() - want).abs() <= 1e-7 * (before[k][0].double().abs() + want.abs() + u.double().abs())).all(), k
            assert torch.equal(model.w[k], model.master[k].to(BF16)), k


def test_step_in_a_graph():
    """The whole step captured, replayed on changed inputs beside eager steps of another model."""
    model, other = Model(264, 520, 1000, F32), Model(264, 520, 1000, F32)
    x, t = rand(20, (301, 264), 1.0, F32), torch.randint(0, 993, (301,), dtype=torch.int32, device=DEV)
    x2 = rand(30, (301, 264), 1.0, F32)
    nb.nb_workspace_reserve(64 << 20)  # before capturing: the head's partials

    def step(m, x_):
        loss, dx = m.micro_step(x_, t, 1.0 / 301, accumulate=False)
        return loss, dx, m.update()

    step(other, x2)  # first use of every kernel: attributes are set outside the capture
    torch.cuda.synchronize()
    held_x = x.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step(model, held_x)
    graph.replay()
    held_x.copy_(x2)
    graph.replay()
    torch.cuda.synchronize()
    fresh = Model(264, 520, 1000, F32)
    step(fresh, x)
    want = step(fresh, x2)
    torch.cuda.synchronize()
    # the linears' weight gradients are summed in no fixed order: last bits of fp32, which the update's roundings may turn into some of its own
    assert rel(held[0], want[0].double()) <= 1e-3 and rel(held[1], want[1].double()) <= 1e-2
    for k in model.master:
        assert rel(model.master[k], fresh.master[k].double()) <= 1e-3, k
        assert rel(held[2][k], want[2][k].double()) <= 1e-2, k
