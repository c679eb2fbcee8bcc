"""What the conveniences of the binding return where there is no sequence: every row is in none of them, and zero."""
import math

import pytest
import torch

from paper_2609_28568_b200 import binding as nb
from test_gpu_attention import BF16, DEV, rand

pytestmark = pytest.mark.gpu


def test_no_sequences():
    T, H, D = 300, 4, 64
    q, dout, freq = rand(1, (T, H, D)), rand(2, (T, H, D)), nb.rotary_frequencies(D)

    def used():  # memory that an allocation is likely to be given next
        t = [torch.full((T, H, D), math.nan, dtype=BF16, device=DEV) for _ in range(4)] + [torch.full((H, T), math.nan, device=DEV)]
        torch.cuda.synchronize()
        del t
    used()
    out, lse = nb.attention_forward(q, q, q, n=0)
    assert (out == 0).all() and (lse == 0).all()
    used()
    for g in nb.attention_backward(dout, out, lse, q, q, q, n=0):
        assert (g == 0).all()
    used()
    for t in nb.rotary(q, q, freq, n=0):
        assert (t == 0).all()
    nb.nb_check_status()
