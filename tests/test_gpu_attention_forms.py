"""Attention's kernels as full batches use them: more items than blocks find an SM, so that a block goes from one item of several tiles to the next, and the
form of the backward pass that narrow heads have only then; and sequences of one length whose number lies on both sides of what one warp orders."""
import pytest
import torch

from paper_2609_28568_b200 import binding as nb
from test_gpu_attention import Case, check

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _status_clean():
    yield
    nb.nb_check_status()


LENGTHS = [700, 513, 129, 384, 640, 257]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,kv,D", [(48, 48, 64), (48, 48, 40), (48, 24, 64), (40, 40, 8), (48, 48, 128), (48, 24, 96)])
def test_full_batches(heads, kv, D, causal):
    c = Case(LENGTHS, heads, kv, D, seed=D + kv, first=2, pad=9, fused=D % 16 == 0)
    # blocks of 128 rows that the rule of sizes counts, in both passes more than three to an SM (at most two blocks run on one)
    slots, sms = c.T // 128 + len(LENGTHS), torch.cuda.get_device_properties(0).multi_processor_count
    assert slots * kv > 3 * sms
    check(c, causal)


@pytest.mark.parametrize("m", [1, 130, 257])
@pytest.mark.parametrize("n", [97, 128, 129, 300])
def test_many_sequences_of_one_length(n, m):
    """Without bounds, bit for bit what the same bounds give (a search of its own beyond 128 sequences), and what the formulas do."""
    c = Case([m] * n, 2, 1, 32, seed=n + m)
    whole = nb.attention_forward(c.q, c.k, c.v, c.cu)
    even = nb.attention_forward(c.q, c.k, c.v, n=n)
    for a, b in zip(whole, even):
        assert torch.equal(a, b)
    for a, b in zip(nb.attention_backward(c.dout, *whole, c.q, c.k, c.v, c.cu), nb.attention_backward(c.dout, *whole, c.q, c.k, c.v, n=n)):
        assert torch.equal(a, b)
    check(c)
