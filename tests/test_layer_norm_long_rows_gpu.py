"""Layer norm of more rows beyond 8192 elements than there are work-groups: each takes several of them."""
import pytest
import torch

from paper_2106_09236_amd import binding as psa
from tests.operator_bounds import assert_within, layer_norm, layer_norm_grad

pytestmark = pytest.mark.gpu
EPS = 1e-5


def test_more_long_rows_than_work_groups():
    """2^17 + 77 rows (a work-group's second row in the last 77), which repeat every 1013; the gradient, then the norm in place."""
    rows, cols, period = (1 << 17) + 77, 8193, 1013
    g = torch.Generator().manual_seed(2)
    X, dY = (torch.randn(period, cols, generator=g).to(torch.bfloat16) for _ in range(2))
    gamma, beta = (1 + 0.3 * torch.randn(cols, generator=g)).to(torch.bfloat16), (0.3 * torch.randn(cols, generator=g)).to(torch.bfloat16)
    whole = rows // period * period

    def repeated(x):
        return x.cuda().repeat((rows + period - 1) // period, *[1] * (x.dim() - 1))[:rows].contiguous()

    def check(got, want, bound, what):
        assert_within(got[:period], want, bound, what)
        assert (got[:whole].view(-1, period, *got.shape[1:]) == got[:period]).all() and torch.equal(got[whole:], got[:rows - whole])
    Xd, gd, bd = repeated(X), gamma.cuda(), beta.cuda()
    y, mean, rstd, e_y, e_mean, e_rstd = layer_norm(X, gamma, beta, EPS)
    _, mean_d, rstd_d = psa.probsparse_layer_norm_fwd(Xd[:period], gd, bd, EPS)
    dX, _, _ = psa.probsparse_layer_norm_bwd(repeated(dY), Xd, gd, repeated(mean_d), repeated(rstd_d))
    want = layer_norm_grad(dY, X, gamma, EPS)
    check(dX, want[0], want[3], "dX")
    del dX
    _, mean_d, rstd_d = psa.probsparse_layer_norm_fwd(Xd, gd, bd, EPS, Y=Xd)
    check(Xd, y, e_y, "Y")
    check(mean_d, mean, e_mean, "mean")
    check(rstd_d, rstd, e_rstd, "rstd")
