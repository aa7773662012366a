"""How exact packed attention is, by the root mean square of its errors: what bounds of single elements, which add up the worst of all
terms, do not show.

float32: a product of three parts is off by 2^-23 of its factors at the most (2^-25 as a rule) where float32 arithmetic rounds it and each
partial sum by 2^-24; scores, weights and sums are float32 in both.  At most twice as much in every step, and up to 3 roundings of the
exponent (2 in the plain form): within 6 times the error of the same formulas in plain float32.  The emulation below shows that a product
of two parts is far beyond."""
import math

import pytest
import torch

from paper_2106_09236_amd import binding as psa

NAMES = ("out", "lse", "dQ", "dK", "dV")


def _rms(x):
    return x.double().square().mean().sqrt().item()


def _offsets(lens):
    off = [0]
    for n in lens:
        off.append(off[-1] + n)
    return off


def _case(H, H_kv, q_lens, k_lens, dtype, seed=0, wide=0.1):
    """Q, K, V, dOut by head; a tenth of the queries (`wide`) is four times as long."""
    g = torch.Generator().manual_seed(seed + 31 * sum(q_lens) + sum(k_lens))
    Q, K, V, G = (torch.randn(h, n, 64, generator=g) for h, n in ((H, sum(q_lens)), (H_kv, sum(k_lens)), (H_kv, sum(k_lens)), (H, sum(q_lens))))
    Q *= 1 + 3 * (torch.rand(Q.shape[:-1], generator=g) < wide).unsqueeze(-1)
    return [t.to(dtype) for t in (Q, K, V, G)], _offsets(q_lens), _offsets(k_lens)


def formulas(tensors, q_off, k_off, causal, product=torch.matmul, dtype=torch.float64, scale=0.125):
    """out, lse, dQ, dK, dV in `dtype`, every product of two tensors by `product`."""
    Q, K, V, G = (t.to(dtype) for t in tensors)
    H, H_kv = Q.shape[0], K.shape[0]
    out, lse, dQ = torch.zeros_like(Q), torch.full(Q.shape[:2], -math.inf, dtype=dtype), torch.zeros_like(Q)
    dK, dV = torch.zeros_like(K), torch.zeros_like(V)
    for b in range(len(q_off) - 1):
        q, k = slice(q_off[b], q_off[b + 1]), slice(k_off[b], k_off[b + 1])
        n_q, n_k = q_off[b + 1] - q_off[b], k_off[b + 1] - k_off[b]
        if not n_q or not n_k:
            continue
        for h in range(H):
            hk = h // (H // H_kv)
            s = product(Q[h, q], K[hk, k].T.contiguous()) * scale
            if causal:
                s = s.masked_fill(torch.arange(n_k)[None, :] > torch.arange(n_q)[:, None] + (n_k - n_q), -math.inf)
            m = s.amax(1, keepdim=True)
            w = torch.exp(s - m)
            l = w.sum(1, keepdim=True)
            p = w / l
            out[h, q] = product(p, V[hk, k])
            lse[h, q] = (m + torch.log(l))[:, 0]
            dp = product(G[h, q], V[hk, k].T.contiguous())
            ds = p * (dp - (G[h, q] * out[h, q]).sum(1, keepdim=True))
            dQ[h, q] = product(ds, K[hk, k]) * scale
            dK[hk, k] += product(ds.T.contiguous(), Q[h, q]) * scale
            dV[hk, k] += product(p.T.contiguous(), G[h, q])
    return out, lse, dQ, dK, dV


def _run(tensors, q_off, k_off, causal):
    Q, K, V, G = (t.cuda() for t in tensors)
    qo, ko = (torch.tensor(o, dtype=torch.int32, device="cuda") for o in (q_off, k_off))
    out, lse = psa.dense_attn_packed_fwd(Q, K, V, qo, ko, causal=causal, lse=True)
    return [t.cpu() for t in (out, lse, *psa.dense_attn_packed_bwd(Q, K, V, out, lse, G, qo, ko, causal=causal))]


# ------------------------------------------------------------------------------------------------------------ float32
F32_CASES = [(4, 4, [30, 60, 1, 44], [30, 60, 1, 44]), (4, 2, [90, 140], [90, 140]), (8, 2, [3, 1, 2], [400, 700, 129]),
             (64, 32, [200, 290], [200, 290]), (16, 16, [500, 401], [500, 401]), (8, 1, [700, 33], [700, 33])]
F32_TIMES = 6


def _parts_product(n):
    """A float32 product as sums of the products of bfloat16 parts: three parts, those whose indices add up to less than n."""
    def split(x):
        parts = []
        for _ in range(3):
            parts.append(x.to(torch.bfloat16).float())
            x = x - parts[-1]
        return parts

    def product(a, b):
        return sum(x.double() @ y.double() for i, x in enumerate(split(a)) for j, y in enumerate(split(b)) if i + j < n).float()
    return product


def test_plain_float32_tells_products_of_two_parts_apart():
    """On the CPU, what the GPU test below can see: six products of three parts pass, three products of two parts do not."""
    tensors, q_off, k_off = _case(2, 2, [90, 61], [90, 61], torch.float32)
    want = formulas(tensors, q_off, k_off, True)
    plain, six, three = (formulas(tensors, q_off, k_off, True, product, torch.float32) for product in (torch.matmul, _parts_product(3), _parts_product(2)))
    for w, x, a, b, what in zip(want, plain, six, three, NAMES):
        own = _rms(x - w)
        assert _rms(a - w) <= F32_TIMES / 2 * own, what
        assert _rms(b - w) > F32_TIMES * own, what


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("H,H_kv,q_lens,k_lens", F32_CASES)
def test_float32_is_as_exact_as_float32(H, H_kv, q_lens, k_lens, causal):
    tensors, q_off, k_off = _case(H, H_kv, q_lens, k_lens, torch.float32)
    want = formulas(tensors, q_off, k_off, causal)
    plain = formulas(tensors, q_off, k_off, causal, dtype=torch.float32)
    got = _run(tensors, q_off, k_off, causal)
    for g, x, w, what in zip(got, plain, want, NAMES):
        assert _rms(g - w) <= F32_TIMES * _rms(x - w), (what, _rms(g - w) / _rms(x - w))
