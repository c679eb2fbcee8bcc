"""Layer norm, without a GPU: which arguments may be the same memory, tensor by tensor."""
import pytest

from paper_2609_28568_b200 import binding as nb
from paper_2609_28568_b200 import build

P = 0x10000  # a fake aligned device address: a refused call never touches it


def at(i):
    """The i-th of fake tensors that lie apart."""
    return P + (i << 20)


@pytest.fixture(scope="module")
def L():
    build.build()
    return nb.lib()


@pytest.mark.parametrize("dtype", [nb.DTYPE_BF16, nb.DTYPE_F32])
def test_forward_only_sum_over_inp_and_out_over_branch(L, dtype):
    """The two pairs that may be one tensor do not open that memory to a third argument."""
    def call(out=at(0), total=at(1), mean=at(2), rstd=at(3), inp=at(4), branch=at(5), w=at(6), b=at(7)):
        return L.nb_layernorm_forward(out, total, mean, rstd, inp, branch, w, b, 4, 64, 1e-5, dtype, None)
    for kw in (dict(total=at(4), w=at(4)),            # blocks would store sum where others still read the weight
               dict(total=at(4), b=at(4)),
               dict(total=at(4), branch=at(4)),       # fp32: a row of sum covers two rows of branch
               dict(out=at(5), inp=at(5)),
               dict(out=at(5), w=at(5)),
               dict(out=at(5), b=at(5)),
               dict(out=at(4), inp=at(4), branch=at(4)),
               dict(out=at(4)), dict(total=at(5))):   # the pairs crossed
        assert call(**kw) == nb.NB_ERR_INVALID_ARG and b"overlap" in L.nb_last_error(), kw


@pytest.mark.parametrize("dtype", [nb.DTYPE_BF16, nb.DTYPE_F32])
def test_backward_only_dinp_over_dres_and_dbranch_over_dout(L, dtype):
    need = nb.nb_layernorm_workspace(4, 64)

    def call(dinp=at(0), dbranch=at(1), dw=at(2), db=at(3), dout=at(4), dres=at(5), inp=at(6), mean=at(7), rstd=at(8), w=at(9),
             ws=at(10)):
        return L.nb_layernorm_backward(dinp, dbranch, dw, db, dout, dres, inp, mean, rstd, w, 4, 64, 0, dtype, ws, need, None)
    for kw in (dict(dinp=at(5), inp=at(5)),
               dict(dinp=at(5), dout=at(5)),
               dict(dinp=at(5), w=at(5)),
               dict(dinp=at(5), mean=at(5)),
               dict(dinp=at(5), rstd=at(5)),
               dict(dbranch=at(4), inp=at(4)),
               dict(dbranch=at(4), dres=at(4)),
               dict(dbranch=at(4), w=at(4)),
               dict(dinp=at(4)), dict(dbranch=at(5)),
               dict(dinp=at(6), dres=at(6), inp=at(6))):
        assert call(**kw) == nb.NB_ERR_INVALID_ARG and b"overlap" in L.nb_last_error(), kw
