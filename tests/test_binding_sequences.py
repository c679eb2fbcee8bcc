"""Sequences of tensors as arguments of the binding, without a GPU: what the call is given lives until it has been made."""
import weakref

import pytest

from paper_2609_28568_b200 import binding as nb
from paper_2609_28568_b200 import build

P = 0x10000


class Tensor:
    """What the binding takes for a tensor."""
    is_cuda = True

    def __init__(self, at):
        self.at = at

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return self.at


class Stream:
    """A stream object, which the binding asks for its address last: it notes which tensors are alive then."""

    def __init__(self, refs):
        self.refs, self.alive = refs, None

    @property
    def _as_parameter_(self):
        self.alive = [r() is not None for r in self.refs]
        return 0


@pytest.fixture(scope="module", autouse=True)
def built():
    build.build()


def made_on_the_fly(n, refs, first=0):
    for i in range(n):
        t = Tensor(P + ((first + i) << 20))
        refs.append(weakref.ref(t))
        yield t


def test_tensors_of_an_iterator_live_until_the_call():
    refs = []
    s = Stream(refs)
    nb.nb_muon_apply(made_on_the_fly(2, refs), made_on_the_fly(2, refs, 2), made_on_the_fly(2, refs, 4), 2, 0, 0.9, 0.1, s)
    assert s.alive == [True] * 6
    assert all(r() is None for r in refs)  # and no longer
    refs.clear()
    nb.nb_muon_update(made_on_the_fly(0, refs), None, made_on_the_fly(0, refs), 0, 8, 8, 0.9, 1, 5, *nb.MUON_COEFFICIENTS, 1e-7,
                      nb.DTYPE_F32, None, 0, s)


def test_references_are_given_back_where_the_call_is_refused():
    refs = []
    s = Stream(refs)
    with pytest.raises(nb.NbError):  # fp32 [8, 8]: no workspace
        nb.nb_muon_update(made_on_the_fly(2, refs), made_on_the_fly(2, refs, 2), made_on_the_fly(2, refs, 4), 2, 8, 8, 0.9, 1, 5,
                          *nb.MUON_COEFFICIENTS, 1e-7, nb.DTYPE_F32, None, 0, s)
    assert s.alive == [True] * 6 and all(r() is None for r in refs)
    refs.clear()
    with pytest.raises(ValueError, match="weight"):
        nb.nb_muon_apply(made_on_the_fly(2, refs), made_on_the_fly(3, refs, 2), made_on_the_fly(2, refs, 5), 2, 0, 0.9, 0.1, s)
    assert all(r() is None for r in refs)
