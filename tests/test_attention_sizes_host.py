"""Attention of sizes at the ends of what is taken, without a GPU: what is refused is refused by its sizes, before a device is asked for."""
import pytest

from paper_2609_28568_b200 import binding as nb
from paper_2609_28568_b200 import build

MOST = 2147483000


def at(i):
    """The i-th of fake tensors that lie far apart; a refused call never touches them."""
    return (i + 1) << 46


@pytest.fixture(scope="module")
def L():
    build.build()
    return nb.lib()


def forward(L, T, n, heads, D=8, cu=at(5), scale=0.125):
    return L.nb_attention_forward(at(0), at(1), at(2), at(3), at(4), cu, T, n, heads, heads, D, *(heads * D,) * 4, scale, 1, None)


def backward(L, T, n, heads, D=8, cu=at(9), scale=0.125):
    return L.nb_attention_backward(*(at(i) for i in range(9)), cu, T, n, heads, heads, D, *(heads * D,) * 8, scale, 1, at(10), 4 * T * heads, None)


# blocks of 128 rows, one more to each sequence: more than a launch has (the first sum is beyond 32 bits itself)
@pytest.mark.parametrize("T,n,heads", [(MOST, MOST, 1), (MOST, MOST, 2), (1 << 30, 1 << 30, 2), (128, MOST, 1024), (1 << 24, 1 << 21, 1024)])
@pytest.mark.parametrize("call", [forward, backward])
def test_too_many_blocks(L, call, T, n, heads):
    assert call(L, T, n, heads) == nb.NB_ERR_UNSUPPORTED and b"too many tiles" in L.nb_last_error()


@pytest.mark.parametrize("scale", [1.8e38, 2.5e38, 3.2e38])
@pytest.mark.parametrize("call", [forward, backward])
def test_scales_that_leave_the_type(L, call, scale):
    """Scores are formed in units of log 2, for which 1.44 times the scale has to be a number too."""
    assert call(L, 300, 2, 4, scale=scale) == nb.NB_ERR_INVALID_ARG and b"scale" in L.nb_last_error()
