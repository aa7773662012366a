"""Layer norm forward of both types at both sides of the number of rows from which half as many threads share a row."""
import pytest
import torch

from paper_2106_09236_amd import binding as psa
from tests.operator_bounds import assert_within, layer_norm

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,cols", [(torch.float32, 130), (torch.float32, 255), (torch.float32, 256), (torch.bfloat16, 257), (torch.bfloat16, 512)])
@pytest.mark.parametrize("rows", [32767, 32768, 131071, 131073])
def test_rows_at_the_limits(rows, cols, dtype):
    period = 521
    g = torch.Generator().manual_seed(cols)
    X = torch.randn(period, cols, generator=g).to(dtype)
    gamma, beta = (1 + 0.3 * torch.randn(cols, generator=g)).to(dtype), (0.3 * torch.randn(cols, generator=g)).to(dtype)
    Xd = X.cuda().repeat((rows + period - 1) // period, 1)[:rows].contiguous()
    Y, mean, rstd = psa.probsparse_layer_norm_fwd(Xd, gamma.cuda(), beta.cuda(), 1e-5)
    for got, want, bound, what in zip((Y, mean, rstd), *(layer_norm(X, gamma, beta, 1e-5)[i:i + 3] for i in (0, 3)), ("Y", "mean", "rstd")):
        assert_within(got[:period], want, bound, what)
        whole = rows // period * period
        assert (got[:whole].view(-1, period, *got.shape[1:]) == got[:period]).all() and torch.equal(got[whole:], got[:rows - whole])
