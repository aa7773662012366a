"""Plain float64 forms of layer norm, rotary positions and packed attention on the CPU, with what a correct implementation in
float32 (and bfloat16 where it rounds) may be off by, element by element.

A rounding is off by at most half a step, HALF[dtype] of the value.  Sums of n terms in float32 are off by at most n half
steps of the sum of the terms' sizes, whatever their order.  Everything below follows from these two."""
import math

import torch

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
U = 2.0 ** -24
TINY = 2.0 ** -126


def assert_within(got, want, bound, what=""):
    got, want = got.detach().double().cpu(), want.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    bad = ~((got - want).abs() <= bound)          # (a NaN is bad)
    if bad.any():
        i = tuple(bad.nonzero()[0].tolist())
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} elements off, first at {i}: {got[i].item()!r} "
                             f"for {want[i].item()!r}, bound {bound[i].item() if bound.dim() else bound.item():.3g}")


# ---------------------------------------------------------------------------------------------------------- layer norm
def layer_norm(X, gamma, beta, eps):
    """Y, mean, rstd and the bounds of Y, mean, rstd.  A thread adds up to 32 elements, then the sums of up to 256 threads
    are joined in 8 steps: 40 half steps for a mean over a row that is kept (rows beyond 8192: cols / 256 + 8)."""
    x = X.double()
    n = x.shape[-1]
    chain = max(40, n / 256 + 16)
    mean = x.mean(-1, keepdim=True)
    d = x - mean
    var = (d * d).mean(-1, keepdim=True)
    rstd = 1 / torch.sqrt(var + eps)
    xhat = d * rstd
    g = torch.ones(n, dtype=torch.float64) if gamma is None else gamma.double()
    b = torch.zeros(n, dtype=torch.float64) if beta is None else beta.double()
    y = xhat * g + b
    # the deviations are taken from a rounded mean and corrected by their own mean: relative to the spread
    e_mean = chain * U * d.abs().mean(-1, keepdim=True) + U * mean.abs() + 2 * U * (x.abs().mean(-1, keepdim=True) * chain * U)
    e_rstd = (chain + 4) * U * rstd
    e_xhat = U * ((chain + 8) * xhat.abs() + (chain + 2) * (d.abs().mean(-1, keepdim=True) * rstd))
    e_y = e_xhat * g.abs() + 2 * U * (y.abs() + (xhat * g).abs()) + HALF[X.dtype] * y.abs()
    return y, mean[..., 0], rstd[..., 0], e_y * 1.01, (e_mean * 1.01)[..., 0], (e_rstd * 1.01)[..., 0]


def layer_norm_grad(dY, X, gamma, eps):
    """dX, dgamma, dbeta and their bounds."""
    x, dy = X.double(), dY.double()
    n, rows = x.shape[-1], x.numel() // x.shape[-1]
    chain = max(40, n / 256 + 16)
    x, dy = x.reshape(rows, n), dy.reshape(rows, n)
    mean = x.mean(-1, keepdim=True)
    d = x - mean
    rstd = 1 / torch.sqrt((d * d).mean(-1, keepdim=True) + eps)
    xhat = d * rstd
    g = dy if gamma is None else dy * gamma.double()
    c1, c2 = g.mean(-1, keepdim=True), (g * xhat).mean(-1, keepdim=True)
    dx = rstd * (g - c1 - xhat * c2)
    # rstd is itself off by (chain + 4) half steps where it was saved
    e_xhat = U * ((chain + 8) * xhat.abs() + (chain + 2))
    a1, a2 = g.abs().mean(-1, keepdim=True), (g * xhat).abs().mean(-1, keepdim=True)
    e_c1 = (chain + 2) * U * a1
    e_c2 = (2 * chain + 8) * U * a2 + a1 * U * (chain + 2)
    e = rstd * (2 * U * g.abs() + e_c1 + e_xhat * c2.abs() + xhat.abs() * e_c2 + 4 * U * (g.abs() + c1.abs() + (xhat * c2).abs()))
    e = e + (chain + 5) * U * dx.abs() + HALF[X.dtype] * dx.abs()
    # column sums: at most rows / 256 + 16 rows in a row to a thread, 4 halvings, 1024 partial rows in eight parts
    steps = rows / 256 + 16 + 4 + 128 + 8
    e_g = (dy.abs() * e_xhat).sum(0) + steps * U * (dy * xhat).abs().sum(0)
    e_b = steps * U * dy.abs().sum(0)
    return dx.reshape(X.shape), (dy * xhat).sum(0), dy.sum(0), e.reshape(X.shape) * 1.01, e_g * 1.01, e_b * 1.01


# ------------------------------------------------------------------------------------------------------------- rotary
def rotary(X, angle, magnitude, dim, interleaved):
    """X [B, H, L, 64] turned by angle [B, L, dim / 2] (float64), and its bound: the angle in float32 turns is off by
    pi half steps, sine and cosine by 4 each, then two products and a sum."""
    x = X.double()
    half = dim // 2
    i = torch.arange(half)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
    c, s = (f(angle).unsqueeze(1) * magnitude for f in (torch.cos, torch.sin))
    out = x.clone()
    out[..., a] = x[..., a] * c - x[..., b] * s
    out[..., b] = x[..., a] * s + x[..., b] * c
    bound = torch.zeros_like(out)
    size = (x[..., a].abs() + x[..., b].abs()) * (magnitude * 12 * U)
    bound[..., a] = size + HALF[X.dtype] * out[..., a].abs()
    bound[..., b] = size + HALF[X.dtype] * out[..., b].abs()
    return out, bound * 1.01


# --------------------------------------------------------------------------------------------------- packed attention
class Attention:
    """Rows of one query head of one sequence: weights, output, gradients' parts and bounds, all float64."""

    def __init__(self, Q, K, V, causal, scale, dtype):
        self.q, self.k, self.v, self.scale, self.dtype = Q.double(), K.double(), V.double(), scale, dtype
        n_q, n_k = Q.shape[0], K.shape[0]
        s = scale * self.q @ self.k.T
        self.seen = torch.ones(n_q, n_k, dtype=torch.bool)
        if causal:
            self.seen = torch.arange(n_k)[None, :] <= torch.arange(n_q)[:, None] + (n_k - n_q)
        s = s.masked_fill(~self.seen, -math.inf)
        self.lse = torch.logsumexp(s, 1) if n_k else torch.full((n_q,), -math.inf, dtype=torch.float64)
        self.p = torch.where(self.seen, torch.exp(s - torch.where(torch.isfinite(self.lse), self.lse, 0.0)[:, None]), 0.0)
        # a score is a sum of 64 products and is scaled; its exponential rounds its argument and itself
        size = scale * self.q.abs() @ self.k.abs().T
        self.e_s = 66 * U * size + 4 * U * size + 4 * U * s.abs().masked_fill(~self.seen, 0.0) + 8 * U
        top = torch.where(self.seen, self.e_s, 0.0)
        self.e_p = top + (top.amax(1, keepdim=True) if n_k else 0)        # relative error of a weight (its own, the sum's)
        self.round_p = HALF[dtype] if dtype == torch.bfloat16 else 0.0
        self.out = self.p @ self.v
        pv = self.p @ self.v.abs()
        # a sum over n_k keys, rescaled when the maximum moves (at most once for every tile of 32)
        self.chain = (2 * n_k + 16) * U
        self.e_out = (self.p * self.e_p + TINY * self.seen) @ self.v.abs() + TINY + (self.chain + self.round_p) * pv + HALF[dtype] * self.out.abs()
        self.e_lse = (top.amax(1) if n_k else torch.zeros(n_q)) + self.chain + 8 * U + 2 * U * torch.where(torch.isfinite(self.lse), self.lse, 0.0).abs()

    def gradients(self, dOut):
        """Contributions (dQ, dK, dV) and their bounds before the last rounding, which is of the sum over heads."""
        G = dOut.double()
        w = G @ self.v.T
        d = (G * self.out).sum(1, keepdim=True)
        ds = self.p * (w - d)
        e_d = (G.abs() * self.e_out).sum(1, keepdim=True) + 66 * U * (G * self.out).abs().sum(1, keepdim=True)
        e_w = 66 * U * G.abs() @ self.v.abs().T
        e_p = self.p * (self.e_p + self.e_lse[:, None].masked_fill(~torch.isfinite(self.e_lse[:, None]), 0.0) + 8 * U)
        e_p = e_p + TINY * self.seen
        e_ds = self.p * (e_d + e_w) + e_p * (w - d).abs() + 4 * U * ds.abs() + TINY * self.seen
        r = self.round_p
        e_ds = e_ds * (1 + r) + r * ds.abs()
        e_p = e_p * (1 + r) + r * self.p
        n_q, n_k = ds.shape
        dQ, dK, dV = self.scale * ds @ self.k, self.scale * ds.T @ self.q, self.p.T @ G
        e_q = self.scale * ((e_ds + (n_k + 8) * U * ds.abs()) @ self.k.abs())
        e_k = self.scale * ((e_ds + (n_q + 8) * U * ds.abs()).T @ self.q.abs())
        e_v = (e_p + (n_q + 8) * U * self.p).T @ G.abs()
        return (dQ, dK, dV), (e_q, e_k, e_v)


def packed_attention(Q, K, V, q_off, k_off, causal, scale, dOut=None):
    """out and lse (and dQ, dK, dV) of CPU tensors, and the bound of each."""
    H, T_q, _ = Q.shape
    H_kv, T_k, _ = K.shape
    group = H // H_kv
    zero = lambda *s: torch.zeros(*s, dtype=torch.float64)
    out, e_out, lse, e_lse = zero(H, T_q, 64), zero(H, T_q, 64), torch.full((H, T_q), -math.inf, dtype=torch.float64), zero(H, T_q)
    grads, e_grads = [zero(H, T_q, 64), zero(H_kv, T_k, 64), zero(H_kv, T_k, 64)], [zero(H, T_q, 64), zero(H_kv, T_k, 64), zero(H_kv, T_k, 64)]
    for b in range(len(q_off) - 1):
        q, k = slice(q_off[b], q_off[b + 1]), slice(k_off[b], k_off[b + 1])
        for h in range(H):
            a = Attention(Q[h, q], K[h // group, k], V[h // group, k], causal, scale, Q.dtype)
            out[h, q], e_out[h, q], lse[h, q], e_lse[h, q] = a.out, a.e_out, a.lse, a.e_lse
            if dOut is not None:
                g, e = a.gradients(dOut[h, q])
                for i, (where, head) in enumerate(((q, h), (k, h // group), (k, h // group))):
                    grads[i][head, where] += g[i]
                    e_grads[i][head, where] += e[i]
    result = [(out, e_out * 1.01), (lse, e_lse * 1.01)]
    if dOut is not None:
        result += [(g, (e + HALF[Q.dtype] * (g.abs() + e) + group * U * g.abs() + TINY) * 1.01) for g, e in zip(grads, e_grads)]
    return result
