"""How exact packed attention of bfloat16 tensors is, by the root mean square of its errors against that of rounding the exact values.

Where the weights are kept to 16 bits, what is left is the rounding of the results: weights of 16 bits and a sign are off by 2^-17 of
themselves, 2^-8 of what their rounding to 8 bits adds, and the sums are float32: the error is that of rounding alone to a few
thousandths, at most 1.1 times.  Weights rounded to bfloat16, each by itself, add as much again for values without a common mean:
about sqrt(2) times (these formulas with those roundings in float64: 1.37 to 1.47 times in all four results).  With d left as the
rounding of out has it, dQ and dK had 1.72 to 2.15 times so: 1.6 is between the two."""
import pytest
import torch

from tests.test_packed_precision import NAMES, _case, _rms, _run, formulas

pytestmark = pytest.mark.gpu


def _times(H, H_kv, q_lens, k_lens, causal):
    """Error of out, dQ, dK and dV over the error of rounding."""
    tensors, q_off, k_off = _case(H, H_kv, q_lens, k_lens, torch.bfloat16)
    want = formulas(tensors, q_off, k_off, causal)
    return {what: _rms(g.double() - w) / _rms(w.to(torch.bfloat16).double() - w)
            for what, g, w in zip(NAMES, _run(tensors, q_off, k_off, causal), want) if what != "lse"}


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("H,H_kv,q_lens,k_lens", [
    (8, 8, [1] * 8, [20] * 8),                          # one query to a short sequence
    (4, 4, list(range(1, 41)), list(range(1, 41))),     # short sequences
    (4, 4, [1 + i % 60 for i in range(100)], [1 + i % 60 for i in range(100)]),       # ... and many of them
    (4, 4, [60] * 8, [60] * 8),
    (4, 2, [90, 140], [90, 140]),
    (8, 2, [3, 1, 2], [400, 700, 129]),                 # new queries of longer sequences
    (4, 2, [1, 1], [3000, 900]),
    (8, 1, [700, 0, 1, 333], [700, 5, 1, 333]),         # many rows to a key head
    (2, 2, [2100], [2100])])
def test_weights_of_small_calls_have_16_bits(H, H_kv, q_lens, k_lens, causal):
    times = _times(H, H_kv, q_lens, k_lens, causal)
    assert max(times.values()) <= 1.1, times


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("H,H_kv,q_lens,k_lens", [(64, 32, [200, 290], [200, 290]), (32, 32, [500, 401], [500, 401]), (96, 32, [111, 222, 90], [170, 222, 150])])
def test_weights_of_large_calls_are_rounded_once(H, H_kv, q_lens, k_lens, causal):
    times = _times(H, H_kv, q_lens, k_lens, causal)
    assert max(times.values()) <= 1.6, times
