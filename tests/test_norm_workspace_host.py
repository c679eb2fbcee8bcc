"""Layer norm, without a GPU: the workspace is asked for by the same rule of sizes as the calls."""
import pytest

from paper_2609_28568_b200 import binding as nb
from paper_2609_28568_b200 import build

P = 0x10000  # a fake aligned device address: a refused call never touches it


def at(i):
    """The i-th of fake tensors that lie apart."""
    return P + (i << 48)


@pytest.fixture(scope="module")
def L():
    build.build()
    return nb.lib()


@pytest.mark.parametrize("BT,C", [(-1, 64), (4, 0), (4, -8), (4, 12), (4, 8200), (1 << 31, 8), (1 << 31, 8192), ((1 << 31) - 1, 8192),
                                  ((1 << 30) + 1, 8192), ((1 << 43) // 4104 + 1, 4104), ((1 << 63) - 1, 8), ((1 << 63) - 1, 8192)])
def test_no_size_for_what_the_calls_refuse(L, BT, C):
    assert L.nb_layernorm_workspace(BT, C) == -1
    with pytest.raises(nb.NbError):
        nb.nb_layernorm_workspace(BT, C)
    refused = (nb.NB_ERR_INVALID_ARG, nb.NB_ERR_UNSUPPORTED)
    assert L.nb_layernorm_forward(at(0), None, None, None, at(1), None, at(2), None, BT, C, 1e-5, nb.DTYPE_BF16, None) in refused
    assert L.nb_layernorm_backward(at(0), None, at(1), at(2), at(3), None, at(4), at(5), at(6), at(7), BT, C, 0, nb.DTYPE_BF16, at(8),
                                   1 << 40, None) in refused


@pytest.mark.parametrize("BT,C", [((1 << 31) - 1, 8), (1 << 30, 8192), ((1 << 43) // 4104, 4104), (0, 8192), (1, 8)])
def test_a_size_for_the_largest_and_smallest(L, BT, C):
    size = nb.nb_layernorm_workspace(BT, C)
    assert size % (8 * C) == 0 and size <= 148 * 8 * C and (size > 0) == (BT > 0)
