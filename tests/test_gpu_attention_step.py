"""The operators together as a layer uses them: qkv linear -> rotary positions in place -> attention -> attn_proj, and back into the qkv linear's
gradients, over packed sequences with rows left over, against 64-bit autograd."""
import math

import pytest
import torch

from paper_2609_28568_b200 import binding as nb
from attention_reference import frequencies
from test_gpu_attention import BF16, DEV, cumulated, rand

pytestmark = pytest.mark.gpu
F32 = torch.float32


@pytest.fixture(autouse=True)
def _status_clean():
    yield
    nb.nb_check_status()


class Layer:
    def __init__(self, C, heads, kv, D, lengths, pad, rotate):
        self.C, self.heads, self.kv, self.D, self.rotate = C, heads, kv, D, rotate
        self.bounds = cumulated(lengths)
        self.T = self.bounds[-1] + pad
        self.cu = torch.tensor(self.bounds, dtype=torch.int32, device=DEV)
        self.wide = (heads + 2 * kv) * D
        self.w = {"qkv": rand(1, (self.wide, C), C ** -0.5), "qkv_b": rand(2, (self.wide,), 0.1), "proj": rand(3, (C, heads * D), (heads * D) ** -0.5),
                  "proj_b": rand(4, (C,), 0.1)}
        self.freq = nb.rotary_frequencies(D, base=1000.0)
        self.grad = {k: torch.zeros(v.shape, dtype=F32, device=DEV) for k, v in self.w.items()}

    def split(self, t):
        return t.view(self.T, -1, self.D).split([self.heads, self.kv, self.kv], 1)

    def step(self, x, dy):
        """(y, dx); the parameters' gradients into self.grad."""
        w, g = self.w, self.grad
        qkv, _ = nb.linear_forward(x, w["qkv"], w["qkv_b"])
        q, k, v = self.split(qkv)
        if self.rotate:
            nb.rotary(q, k, self.freq, cu_seqlens=self.cu, in_place=True)
        out, lse = nb.attention_forward(q, k, v, self.cu)
        flat = out.view(self.T, -1)
        y, _ = nb.linear_forward(flat, w["proj"], w["proj_b"])
        dout, _, _ = nb.linear_backward(dy, flat, w["proj"], dweight=g["proj"], dbias=g["proj_b"])
        dqkv = torch.zeros_like(qkv)
        dq, dk, dv = self.split(dqkv)
        nb.attention_backward(dout.view(out.shape), out, lse, q, k, v, self.cu, grads=(dq, dk, dv))
        if self.rotate:
            nb.rotary(dq, dk, self.freq, cu_seqlens=self.cu, inverse=True, in_place=True)
        dx, _, _ = nb.linear_backward(dqkv, x, w["qkv"], dweight=g["qkv"], dbias=g["qkv_b"])
        return y, dx

    def reference(self, x, dy):
        p = {k: v.double().requires_grad_() for k, v in self.w.items()}
        x = x.double().requires_grad_()
        q, k, v = self.split(x @ p["qkv"].T + p["qkv_b"])
        f = frequencies(self.D, 1000.0).to(DEV)
        parts = []
        for a, b in zip(self.bounds, self.bounds[1:]):
            qq, kk, vv = (t[a:b] for t in (q, k, v))
            if self.rotate:
                angle = torch.arange(b - a, device=DEV).double()[:, None] * f
                c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
                turn = lambda t: torch.cat((t[..., :self.D // 2] * c - t[..., self.D // 2:] * s, t[..., self.D // 2:] * c + t[..., :self.D // 2] * s), -1)  # noqa: E731
                qq, kk = turn(qq), turn(kk)
            kk, vv = (t.repeat_interleave(self.heads // self.kv, 1) for t in (kk, vv))
            scores = torch.einsum("ihd,jhd->hij", qq, kk) / math.sqrt(self.D)
            hidden = torch.ones((b - a, b - a), dtype=torch.bool, device=DEV).triu(1)
            parts.append(torch.einsum("hij,jhd->ihd", scores.masked_fill(hidden, -math.inf).softmax(-1), vv).flatten(1))
        rest = torch.zeros((self.T - self.bounds[-1], self.heads * self.D), dtype=torch.float64, device=DEV)
        y = torch.cat((*parts, rest)) @ p["proj"].T + p["proj_b"]
        y.backward(dy.double())
        return y.detach(), x.grad, {k: v.grad for k, v in p.items()}


def rel(a, b):
    return ((a.double() - b).norm() / b.norm()).item()


# Eight roundings to bf16 lie between x and its gradient (qkv, turned q and k, probabilities, out, dout, p and ds, the gradients of q, k and v, turned
# back), each with an rms of at most 2^-8 / sqrt(3) = 2.3e-3 of its values: 6.4e-3 where all of them reach the result alike, twice that at most.
TOL = 1.3e-2


@pytest.mark.parametrize("C,heads,kv,D,rotate", [(96, 3, 3, 64, False), (128, 4, 2, 128, True), (72, 4, 1, 80, True)])
@pytest.mark.parametrize("lengths,pad", [([300, 1, 129, 0, 64], 0), ([70, 200], 30)])
def test_layer(C, heads, kv, D, rotate, lengths, pad):
    layer = Layer(C, heads, kv, D, lengths, pad, rotate)
    x, dy = rand(10, (layer.T, C)), rand(11, (layer.T, C), 0.1)
    want_y, want_dx, want = layer.reference(x, dy)
    y, dx = layer.step(x, dy)
    assert rel(y, want_y) <= TOL and rel(dx[:layer.bounds[-1]], want_dx[:layer.bounds[-1]]) <= TOL
    assert (dx[layer.bounds[-1]:] == 0).all()
    for k, g in want.items():
        assert rel(layer.grad[k], g) <= TOL, (k, rel(layer.grad[k], g))


def test_layer_in_a_graph():
    """Captured once and replayed on other sequences of the same sum: their bounds are read on the device."""
    layer = Layer(128, 4, 2, 64, [130, 70, 100], 20, True)
    x, dy = rand(10, (layer.T, 128)), rand(11, (layer.T, 128), 0.1)
    layer.step(x, dy)  # first use of every kernel: attributes are set outside the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = layer.step(x, dy)
    other = Layer(128, 4, 2, 64, [1, 250, 49], 20, True)
    layer.cu.copy_(other.cu)
    graph.replay()
    torch.cuda.synchronize()
    want_y, want_dx, want = other.reference(x, dy)
    assert rel(held[0], want_y) <= TOL and rel(held[1][:300], want_dx[:300]) <= TOL
    for k, g in want.items():
        assert rel(layer.grad[k], g) <= TOL, k
