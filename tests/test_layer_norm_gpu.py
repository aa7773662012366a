"""Layer norm and its gradients against float64."""
import pytest
import torch

from paper_2106_09236_amd import binding as psa
from tests.operator_bounds import assert_within, layer_norm, layer_norm_grad

pytestmark = pytest.mark.gpu
EPS = 1e-5


def _inputs(rows, cols, dtype, seed, offset=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=g) * (0.2 + 2 * torch.rand(rows, 1, generator=g)) + offset * torch.randn(rows, 1, generator=g)
    gamma = 1 + 0.3 * torch.randn(cols, generator=g)
    return [t.to(dtype) for t in (x, torch.randn(rows, cols, generator=g), gamma, 0.3 * torch.randn(cols, generator=g))]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 2), (1, 512), (5, 7), (33, 64), (257, 65), (100, 256), (1025, 257), (19, 512), (7, 777),
                                       (300, 1001), (4, 1024), (9, 2048), (3, 2049), (2, 4097), (5, 8192), (3, 8193), (70, 9001), (2, 40000)])
def test_norm_and_gradients(rows, cols, dtype):
    X, dY, gamma, beta = _inputs(rows, cols, dtype, rows * 100003 + cols)
    Xd, dYd, gd, bd = (t.cuda() for t in (X, dY, gamma, beta))
    Y, mean, rstd = psa.probsparse_layer_norm_fwd(Xd, gd, bd, EPS)
    y, m, r, e_y, e_m, e_r = layer_norm(X, gamma, beta, EPS)
    assert_within(Y, y, e_y, "Y")
    assert_within(mean, m, e_m, "mean")
    assert_within(rstd, r, e_r, "rstd")
    assert torch.equal(psa.probsparse_layer_norm_fwd(Xd, gd, bd, EPS, stats=False), Y)
    dX, dgamma, dbeta = psa.probsparse_layer_norm_bwd(dYd, Xd, gd, mean, rstd)
    dx, dg, db, e_x, e_g, e_b = layer_norm_grad(dY, X, gamma, EPS)
    assert_within(dX, dx, e_x, "dX")
    assert_within(dgamma, dg, e_g, "dgamma")
    assert_within(dbeta, db, e_b, "dbeta")
    assert dgamma.dtype == dbeta.dtype == torch.float32
    # the same again, bit for bit: no order of atomics
    again = psa.probsparse_layer_norm_bwd(dYd, Xd, gd, mean, rstd)
    assert all(torch.equal(a, b) for a, b in zip(again, (dX, dgamma, dbeta)))


@pytest.mark.parametrize("rows,cols", [(40000, 256), (9000, 512), (66000, 24), (66000, 300)])
def test_many_rows(rows, cols):
    X, dY, gamma, beta = _inputs(rows, cols, torch.bfloat16, rows + cols)
    Xd, dYd, gd, bd = (t.cuda() for t in (X, dY, gamma, beta))
    Y, mean, rstd = psa.probsparse_layer_norm_fwd(Xd, gd, bd, EPS)
    y, _, _, e_y, _, _ = layer_norm(X, gamma, beta, EPS)
    assert_within(Y, y, e_y, "Y")
    got = psa.probsparse_layer_norm_bwd(dYd, Xd, gd, mean, rstd)
    want = layer_norm_grad(dY, X, gamma, EPS)
    for g, w, e, what in zip(got, want[:3], want[3:], ("dX", "dgamma", "dbeta")):
        assert_within(g, w, e, what)


def test_more_rows_than_one_launch_takes():
    """2^28 + 77 rows of two columns (16 rows to a work-group of 256 threads: 2^32 threads), in place; the rows repeat every 1013."""
    rows, period = (1 << 28) + 77, 1013
    X, _, gamma, beta = _inputs(period, 2, torch.bfloat16, 9)
    Xd = X.cuda().repeat((rows + period - 1) // period, 1)[:rows].contiguous()
    psa.probsparse_layer_norm_fwd(Xd, gamma.cuda(), beta.cuda(), EPS, Y=Xd, stats=False)
    y, _, _, e_y, _, _ = layer_norm(X, gamma, beta, EPS)
    assert_within(Xd[:period], y, e_y, "Y")
    whole = rows // period * period
    assert (Xd[:whole].view(-1, period, 2) == Xd[:period]).all()
    assert torch.equal(Xd[whole:], Xd[:rows - whole])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("cols", [24, 600, 9000])
def test_without_weights_and_in_place(cols, dtype):
    X, dY, gamma, beta = _inputs(11, cols, dtype, cols)
    Xd, dYd = X.cuda(), dY.cuda()
    y, _, _, e_y, _, _ = layer_norm(X, None, None, EPS)
    Y, mean, rstd = psa.probsparse_layer_norm_fwd(Xd, None, None, EPS)
    assert_within(Y, y, e_y, "Y")
    want = layer_norm_grad(dY, X, None, EPS)
    for g, w, e in zip(psa.probsparse_layer_norm_bwd(dYd, Xd, None, mean, rstd), want[:3], want[3:]):
        assert_within(g, w, e)
    y, _, _, e_y, _, _ = layer_norm(X, gamma, None, EPS)
    assert_within(psa.probsparse_layer_norm_fwd(Xd, gamma.cuda(), None, EPS, stats=False), y, e_y, "no beta")
    y, _, _, e_y, _, _ = layer_norm(X, None, beta, EPS)
    assert psa.probsparse_layer_norm_fwd(Xd, None, beta.cuda(), EPS, Y=Xd, stats=False) is Xd
    assert_within(Xd, y, e_y, "in place, no gamma")


def test_rows_far_from_zero_keep_their_spread():
    # spread 1 at 1000: the mean's own rounding (3e-5) must not reach the result
    X, dY, gamma, beta = _inputs(64, 500, torch.float32, 7, offset=1000.0)
    Xd, gd = X.cuda(), gamma.cuda()
    Y, mean, rstd = psa.probsparse_layer_norm_fwd(Xd, gd, beta.cuda(), EPS)
    y, _, _, e_y, _, _ = layer_norm(X, gamma, beta, EPS)
    assert_within(Y, y, e_y, "Y")
    got = psa.probsparse_layer_norm_bwd(dY.cuda(), Xd, gd, mean, rstd)
    want = layer_norm_grad(dY, X, gamma, EPS)
    for g, w, e in zip(got, want[:3], want[3:]):
        assert_within(g, w, e)


def test_nonfinite_rows_stay_alone():
    X, dY, gamma, beta = _inputs(50, 300, torch.bfloat16, 9)
    Xd, gd, bd = X.cuda(), gamma.cuda(), beta.cuda()
    clean = psa.probsparse_layer_norm_fwd(Xd, gd, bd, EPS, stats=False)
    Xd[7, 3], Xd[21, 299] = float("nan"), float("inf")
    Y = psa.probsparse_layer_norm_fwd(Xd, gd, bd, EPS, stats=False)
    rest = [i for i in range(50) if i not in (7, 21)]
    assert torch.equal(Y[rest], clean[rest])
    assert Y[7].isnan().all() and Y[21].isnan().any()


def test_gradient_against_differences():
    X, dY, gamma, beta = _inputs(6, 40, torch.float32, 3)
    Xd, gd, bd, w = X.cuda(), gamma.cuda(), beta.cuda(), dY.double()
    _, mean, rstd = psa.probsparse_layer_norm_fwd(Xd, gd, bd, EPS)
    grads = psa.probsparse_layer_norm_bwd(dY.cuda(), Xd, gd, mean, rstd)
    h = 2.0 ** -7
    # the loss sums 240 outputs with weights of mean size 0.8, each output off by less than 100 half steps (2^-24) of 1, over
    # 2h = 2^-6: 0.15 at the most for the two; what the third derivative adds is 6e-6 (the same differences in float64)
    for tensor, grad in ((Xd, grads[0]), (gd, grads[1]), (bd, grads[2])):
        flat = tensor.view(-1)
        for i in range(0, flat.numel(), 37):
            old = flat[i].item()
            vals = []
            for x in (old + h, old - h):
                flat[i] = x
                vals.append((psa.probsparse_layer_norm_fwd(Xd, gd, bd, EPS, stats=False).double().cpu() * w).sum().item())
            flat[i] = old
            assert abs((vals[0] - vals[1]) / (2 * h) - grad.view(-1)[i].item()) < 0.16


def test_other_stream_and_graph():
    X, dY, gamma, beta = _inputs(700, 512, torch.bfloat16, 5)
    Xd, dYd, gd, bd = (t.cuda() for t in (X, dY, gamma, beta))
    ref = psa.probsparse_layer_norm_fwd(Xd, gd, bd, EPS)
    ref_grads = psa.probsparse_layer_norm_bwd(dYd, Xd, gd, *ref[1:])
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        got = psa.probsparse_layer_norm_fwd(Xd, gd, bd, EPS)
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, ref))
    with torch.cuda.graph(graph):
        got = psa.probsparse_layer_norm_fwd(Xd, gd, bd, EPS)
        grads = psa.probsparse_layer_norm_bwd(dYd, Xd, gd, *got[1:])
    for k in range(3):
        for t in (*got, *grads):
            t.fill_(float(k))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((*got, *grads), (*ref, *ref_grads)))
