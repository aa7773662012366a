"""Rotary positions against float64."""
import math

import pytest
import torch

from paper_2106_09236_amd import binding as psa
from tests.operator_bounds import assert_within, rotary

pytestmark = pytest.mark.gpu


def _make(B, H, L, dtype, seed, by_frame):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((B, L, H, 64) if by_frame else (B, H, L, 64), generator=g).to(dtype)
    d = x.cuda()
    return (x.transpose(1, 2), d.transpose(1, 2)) if by_frame else (x, d)


def _angles(spec, positions):
    return positions.double()[..., None] * torch.tensor(psa.rotary_frequencies(spec), dtype=torch.float64)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("layout", [psa.ROTARY_HALF, psa.ROTARY_INTERLEAVED])
@pytest.mark.parametrize("B,H,H_kv,L,dim,by_frame", [(1, 1, 1, 1, 64, False), (1, 8, 2, 1, 64, True), (2, 4, 4, 17, 64, False), (3, 4, 1, 100, 32, True),
                                                     (1, 4, 2, 333, 16, False), (2, 3, 1, 15, 2, True), (2, 2, 2, 50, 62, False), (1, 5, 5, 31, 24, True)])
def test_turns_and_back(B, H, H_kv, L, dim, by_frame, layout, dtype):
    Q, Qd = _make(B, H, L, dtype, L + dim, by_frame)
    K, Kd = _make(B, H_kv, L, dtype, L + dim + 1, by_frame)
    spec = psa.make_rotary(dim, layout=layout, magnitude=1.25)
    positions = torch.randint(0, 1 << 20, (B, L), generator=torch.Generator().manual_seed(L), dtype=torch.int32)
    cases = [(None, 0, torch.arange(L).expand(B, L)), (None, 777777, (777777 + torch.arange(L)).expand(B, L)),
             (positions, 0, positions), (positions[0].contiguous(), 0, positions[:1].expand(B, L))]
    for given, first, where in cases:
        pd = None if given is None else given.cuda()
        for back in (False, True):
            f = psa.probsparse_rotary_bwd if back else psa.probsparse_rotary_fwd
            outs = f(Qd, Kd, spec, positions=pd, first=first)
            for got, x in zip(outs, (Q, K)):
                want, bound = rotary(x, _angles(spec, where) * (-1 if back else 1), 1.25, dim, layout == psa.ROTARY_INTERLEAVED)
                assert_within(got, want, bound, f"first {first} back {back}")
                assert torch.equal(got[..., dim:].cpu(), x[..., dim:])
            assert torch.equal(f(Qd, None, spec, positions=pd, first=first), outs[0])
    # in place
    qo, ko = psa.probsparse_rotary_fwd(Qd, Kd, spec, first=3)
    q2, k2 = Qd.clone(), Kd.clone()
    assert psa.probsparse_rotary_fwd(q2, k2, spec, first=3, Q_out=q2, K_out=k2)[0] is q2
    assert torch.equal(q2, qo) and torch.equal(k2, ko)


@pytest.mark.parametrize("layout", [psa.ROTARY_HALF, psa.ROTARY_INTERLEAVED])
def test_inside_a_larger_array(layout):
    # Q, K, V of a fused projection [T, 3, H, 64], turned in place; V is not touched
    T, H = 77, 4
    fused = torch.randn(T, 3, H, 64, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    d = fused.cuda()
    spec = psa.make_rotary(48, layout=layout)
    q, k = d[:, 0].transpose(0, 1), d[:, 1].transpose(0, 1)
    psa.probsparse_rotary_fwd(q, k, spec, Q_out=q, K_out=k)
    for i in range(2):
        want, bound = rotary(fused[:, i].transpose(0, 1)[None], _angles(spec, torch.arange(T)[None]), 1.0, 48, layout == psa.ROTARY_INTERLEAVED)
        assert_within(d[:, i].transpose(0, 1)[None], want, bound)
    assert torch.equal(d[:, 2].cpu(), fused[:, 2])


def test_gradient_is_the_transpose():
    # <R x, y> = <x, R' y>; 64 products a head, each off by 12 half steps of its factors, over 2 * 20 * 64 elements
    spec = psa.make_rotary(64, base=500.0)
    x, y = (torch.randn(1, 2, 20, 64, generator=torch.Generator().manual_seed(i)).cuda() for i in (1, 2))
    a = (psa.probsparse_rotary_fwd(x, None, spec).double() * y.double()).sum().item()
    b = (x.double() * psa.probsparse_rotary_bwd(y, None, spec).double()).sum().item()
    assert abs(a - b) <= 2 * 2 * 13 * 2.0 ** -24 * (x.abs().double().sum() * y.abs().max().double()).item()


def test_graph_replays():
    spec = psa.make_rotary(64)
    q, k = (torch.randn(2, 4, 50, 64, device="cuda") for _ in range(2))
    pos = torch.arange(50, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = psa.probsparse_rotary_fwd(q, k, spec, positions=pos)
    for step in range(3):
        pos += 50
        graph.replay()
        ref = psa.probsparse_rotary_fwd(q, k, spec, first=50 * (step + 1))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, ref))
