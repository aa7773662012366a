"""Rotary positions as far as the header promises angles that are exact to float32: 2^26."""
import pytest
import torch

from paper_2106_09236_amd import binding as psa
from tests.operator_bounds import assert_within, rotary

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layout", [psa.ROTARY_HALF, psa.ROTARY_INTERLEAVED])
@pytest.mark.parametrize("dim", [64, 30])
def test_far_positions(dim, layout):
    L = 200
    g = torch.Generator().manual_seed(dim)
    X = torch.randn(1, 3, L, 64, generator=g)
    spec = psa.make_rotary(dim, layout=layout)
    where = torch.randint((1 << 26) - (1 << 20), 1 << 26, (1, L), generator=g, dtype=torch.int32)
    first = (1 << 26) - L
    for positions, at in ((where, where), (None, torch.arange(first, 1 << 26)[None])):
        # the angle itself in float64 is off by 2^-53 of 2^26: half of a half step of float32, beside the 12 that the bound counts
        angle = at.double()[..., None] * torch.tensor(psa.rotary_frequencies(spec), dtype=torch.float64)
        want, bound = rotary(X, angle, 1.0, dim, layout == psa.ROTARY_INTERLEAVED)
        assert_within(psa.probsparse_rotary_fwd(X.cuda(), None, spec, positions=None if positions is None else positions.cuda(), first=first), want, bound)
