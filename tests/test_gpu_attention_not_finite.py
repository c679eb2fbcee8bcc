"""How far a value that is not finite reaches inside its own sequence: to what sees it or is seen by it, and, for some, no further than the 128 rows beside it."""
import math

import pytest
import torch

from paper_2609_28568_b200 import binding as nb
from test_gpu_attention import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _status_clean():
    yield
    nb.nb_check_status()


@pytest.mark.parametrize("heads,kv,D", [(2, 1, 64), (2, 2, 128), (130, 130, 64), (6, 1, 40)])
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_reach_within_a_sequence(heads, kv, D, value):
    c, row, last = Case([450], heads, kv, D, seed=D), 200, 256  # the blocks of 128 rows around: [128, 256)
    out, lse = nb.attention_forward(c.q, c.k, c.v)
    grads = nb.attention_backward(c.dout, out, lse, c.q, c.k, c.v)

    def changed(name):
        t = getattr(c, name)
        kept = t[row].clone()
        t[row] = value
        got = nb.attention_forward(c.q, c.k, c.v), nb.attention_backward(c.dout, out, lse, c.q, c.k, c.v)
        t[row] = kept
        return got
    same = lambda a, b, *rows: all(torch.equal(a[r], b[r]) for r in rows)  # noqa: E731
    (o, s), (dq, dk, dv) = changed("q")  # its own row of out and dq; keys from the first to its own, and up to 55 after it
    others = slice(0, row), slice(row + 1, 450)
    assert same(o, out, *others) and same(s.T, lse.T, *others) and same(dq, grads[0], *others)
    assert same(dk, grads[1], slice(last, 450)) and same(dv, grads[2], slice(last, 450))
    (o, s), (dq, dk, dv) = changed("k")  # rows from its own on; of dq from 72 before it on
    assert same(o, out, slice(0, row)) and same(s.T, lse.T, slice(0, row)) and same(dq, grads[0], slice(0, 128))
    assert same(dk, grads[1], *others) and same(dv, grads[2], *others)
    (o, s), (dq, dk, dv) = changed("v")
    assert same(o, out, slice(0, 128)) and torch.equal(s, lse) and same(dq, grads[0], slice(0, row))
    assert same(dk, grads[1], *others) and torch.equal(dv, grads[2])
    _, (dq, dk, dv) = changed("dout")
    assert same(dq, grads[0], *others) and same(dk, grads[1], slice(last, 450)) and same(dv, grads[2], slice(last, 450))
