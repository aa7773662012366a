"""Operators around the prob-sparse path that are worth timing: layer norm, rotary positions and dense attention over
packed sequences, forward and backward, as a speech or language model built on this library has them.

A case is one call (or, for "train", a forward call and its backward) of `paper_2106_09236_amd.binding` on inputs that
are on the GPU, on the current stream:

    op "norm"    what "serve"   probsparse_layer_norm_fwd                    rows of `cols` elements
                 what "train"   probsparse_layer_norm_fwd and _bwd
    op "rotary"  what "fwd"     probsparse_rotary_fwd on Q and K             Q [B, H, L, 64], K [B, H_kv, L, 64]
                 what "bwd"     probsparse_rotary_bwd on dQ and dK
    op "attn"    what "serve"   dense_attn_packed_fwd                        Q [H, T_q, 64], K and V [H_kv, T_k, 64]
                 what "train"   dense_attn_packed_fwd and _bwd

The sequences of an attention case have `len_lo` to `len_hi` keys each, drawn from `lens`; `new` > 0 says that only the
last `new` frames of each are queries (frames that arrive while the earlier ones are kept), 0 that all are.  Q, K, V and
their gradients are row-major either by head ([H, T, 64], what the projections of this library write) or by frame
([T, H, 64], what a fused projection writes).
"""
import math
import random

import torch

own = False

D = 64
EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------------------------------------- the cases
def _norm(what, dtype, rows, cols, affine=True, **name):
    return dict(name, op="norm", what=what, dtype=dtype, rows=rows, cols=cols, affine=affine)


def _rotary(what, dtype, B, H, H_kv, L, dim, layout, scaling="plain", factor=1.0, start=0, by_frame=False, given=False, **name):
    return dict(name, op="rotary", what=what, dtype=dtype, B=B, H=H, H_kv=H_kv, L=L, dim=dim, layout=layout,
                scaling=scaling, factor=factor, start=start, by_frame=by_frame, given=given)


def _attn(what, dtype, B, H, H_kv, len_lo, len_hi, causal, new=0, by_frame=False, values="normal", lens=1, **name):
    return dict(name, op="attn", what=what, dtype=dtype, B=B, H=H, H_kv=H_kv, len_lo=len_lo, len_hi=len_hi,
                causal=causal, new=new, by_frame=by_frame, values=values, lens=lens)


def listed():
    return [
        # the norm before a layer of the 8-head model for one frame that has just arrived: latency alone
        _norm("serve", "bf16", 1, 512, name="norm_frame_bf16"),
        # training of the 4-head model on a padded batch of 24 clips of up to 30 s
        _norm("train", "f32", 18000, 256, name="norm_train_f32"),
        # training of the 8-head model: 64 segments of 80 s
        _norm("train", "bf16", 131072, 512, name="norm_train_bf16"),
        # filter-bank features with their first and second differences, appended to an odd number of channels
        _norm("serve", "f32", 12345, 1001, name="norm_odd_f32"),
        # Q and K of an 8-head layer on a batch of 80-second segments
        _rotary("fwd", "bf16", 8, 8, 8, 2048, 64, "half", name="rotary_batch_bf16"),
        # gradients of an odd utterance in the 4-head model, half of each head rotated, far into a recording
        _rotary("bwd", "f32", 1, 4, 2, 333, 32, "interleaved", "parts", 8.0, start=60000, by_frame=True, given=True,
                name="rotary_utterance_f32"),
        # corpus clips of 40 to 500 frames packed without padding, all frames see each other
        _attn("serve", "bf16", 32, 4, 4, 40, 500, False, name="attn_clips_bf16"),
        # eleven minutes of audio in one sequence, each frame sees those before it
        _attn("serve", "bf16", 1, 8, 8, 16384, 16384, True, values="peaky", name="attn_longform_bf16"),
        # a batch of 20-second clips in float32
        _attn("serve", "f32", 16, 4, 4, 512, 512, False, values="peaky", name="attn_batch_f32"),
        # one new frame in each of 32 running streams, query heads share keys in fours
        _attn("serve", "bf16", 32, 8, 2, 1, 4096, True, new=1, name="attn_streams_bf16"),
        # a training step of the 8-head layer on a batch of 80-second segments, tensors as a fused projection leaves them
        _attn("train", "bf16", 8, 8, 8, 2048, 2048, True, by_frame=True, name="attn_train_bf16"),
        # a training step of the 4-head layer on packed clips of up to 30 s, two query heads to a key head
        _attn("train", "f32", 24, 4, 2, 120, 750, True, values="peaky", name="attn_train_f32"),
    ]


def _cost(case):
    """Seconds the case takes at a nominal card's rates."""
    w = work(case)
    return w["bytes"] / 8e12 + w["flops"] / (157e12 if case["dtype"] == "f32" else 2.5e15)


def draw(rng):
    def log_uniform(lo, hi):
        return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))
    op = rng.choice(["norm", "rotary", "attn", "attn"])
    what = rng.choice(["fwd", "bwd"] if op == "rotary" else ["serve", "train"])
    most = max(_cost(c) for c in listed() if c["op"] == op)
    while True:
        dtype = rng.choice(["f32", "bf16"])
        if op == "norm":
            case = _norm(what, dtype, log_uniform(1, 131072), rng.choice([256, 512, log_uniform(16, 4096)]), rng.random() < 0.9)
        elif op == "rotary":
            H = rng.choice([4, 8])
            case = _rotary(what, dtype, log_uniform(1, 32), H, H // rng.choice([1, 1, 2, 4]), log_uniform(1, 16384),
                           rng.choice([64, 64, 32, 2 * rng.randint(1, 32)]), rng.choice(["half", "interleaved"]),
                           *rng.choice([("plain", 1.0), ("linear", 4.0), ("base", 8.0), ("parts", 16.0)]),
                           rng.choice([0, rng.randint(0, 1000000)]), rng.random() < 0.5, rng.random() < 0.5)
        else:
            H = rng.choice([4, 8])
            hi = log_uniform(1, 16384)
            lo = hi if rng.random() < 0.3 else max(1, hi // rng.choice([2, 8, 64]))
            case = _attn(what, dtype, log_uniform(1, 64), H, H // rng.choice([1, 1, 2, 4]), lo, hi, rng.random() < 0.6,
                         0 if what == "train" or rng.random() < 0.6 else log_uniform(1, 64), rng.random() < 0.5,
                         rng.choice(["normal", "peaky"]), rng.randint(1, 1 << 30))
            if case["B"] * hi > 131072:
                continue
        if _cost(case) <= most:
            return case


def _lengths(case):
    """Queries and keys of each sequence of an attention case."""
    r = random.Random(case["lens"])
    keys = [r.randint(case["len_lo"], case["len_hi"]) for _ in range(case["B"])]
    return [min(n, case["new"]) if case["new"] else n for n in keys], keys


def _pairs(case):
    """Query-key pairs of an attention case that are not masked, for one head."""
    return sum(q * (k - q) + q * (q + 1) // 2 if case["causal"] else q * k for q, k in zip(*_lengths(case)))


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    train = case["what"] == "train"
    if case["op"] == "norm":
        n, c = case["rows"] * case["cols"], case["cols"] * case["affine"]
        if train:      # reads X and dY, writes Y and dX, and the weights' gradients in 32 bits
            return {"bytes": 4 * n * size + 2 * c * size + 8 * case["cols"], "flops": 18 * n}
        return {"bytes": 2 * n * size + 2 * c * size, "flops": 7 * n}
    if case["op"] == "rotary":
        rows = case["B"] * case["L"]
        heads = case["H"] + case["H_kv"]
        return {"bytes": 2 * rows * heads * D * size + (4 * rows if case["given"] else 0), "flops": 3 * rows * heads * case["dim"]}
    q, k = (sum(n) for n in _lengths(case))
    q, k = q * case["H"] * D * size, k * case["H_kv"] * D * size
    offsets = 8 * (case["B"] + 1)
    if train:          # two products forward, five backward; Q, K, V, dOut in, out, dQ, dK, dV out
        return {"bytes": 4 * q + 4 * k + offsets, "flops": 14 * D * _pairs(case) * case["H"]}
    return {"bytes": 2 * q + 2 * k + offsets, "flops": 4 * D * _pairs(case) * case["H"]}


# --------------------------------------------------------------------------------------------------------- the inputs


class State:
    """What a user's program has in hand before a call."""


def _heads(g, case, B, H, T, values="normal"):
    """Random [B, H, T, 64], by head or by frame in memory."""
    x = torch.randn((B, T, H, D) if case["by_frame"] else (B, H, T, D), generator=g, device="cuda")
    if values == "peaky":      # a tenth of the rows has scores several times as wide as the others
        x *= 1 + 3 * (torch.rand(x.shape[:-1], generator=g, device="cuda") < 0.1).unsqueeze(-1)
    x = x.to(TYPES[case["dtype"]])
    return x.transpose(1, 2) if case["by_frame"] else x


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = State()
    s.case = case
    t = TYPES[case["dtype"]]
    if case["op"] == "norm":
        rows, cols = case["rows"], case["cols"]
        x = torch.randn((rows, cols), generator=g, device="cuda")
        s.X = (x * (0.5 + torch.rand((rows, 1), generator=g, device="cuda")) + torch.randn((rows, 1), generator=g, device="cuda")).to(t)
        s.gamma = s.beta = None
        if case["affine"]:
            s.gamma = (1 + 0.2 * torch.randn(cols, generator=g, device="cuda")).to(t)
            s.beta = (0.2 * torch.randn(cols, generator=g, device="cuda")).to(t)
        if case["what"] == "train":
            s.dY = torch.randn((rows, cols), generator=g, device="cuda").to(t)
    elif case["op"] == "rotary":
        s.Q = _heads(g, case, case["B"], case["H"], case["L"])
        s.K = _heads(g, case, case["B"], case["H_kv"], case["L"])
        s.positions = None
        if case["given"]:
            gaps = torch.randint(1, 3, (case["B"], case["L"]), generator=g, device="cuda", dtype=torch.int32)
            s.positions = (case["start"] + gaps.cumsum(1)).to(torch.int32)
    else:
        q, k = _lengths(case)
        s.q_offsets, s.k_offsets = [0], [0]
        for a, b in zip(q, k):
            s.q_offsets.append(s.q_offsets[-1] + a)
            s.k_offsets.append(s.k_offsets[-1] + b)
        s.q_off = torch.tensor(s.q_offsets, dtype=torch.int32, device="cuda")
        s.k_off = torch.tensor(s.k_offsets, dtype=torch.int32, device="cuda")
        s.Q = _heads(g, case, 1, case["H"], s.q_offsets[-1], case["values"])[0]
        s.K = _heads(g, case, 1, case["H_kv"], s.k_offsets[-1])[0]
        s.V = _heads(g, case, 1, case["H_kv"], s.k_offsets[-1])[0]
        if case["what"] == "train":
            s.dOut = _heads(g, case, 1, case["H"], s.q_offsets[-1])[0]
    if own:
        from paper_2106_09236_amd import binding as psa
        s.psa = psa
        if case["op"] == "rotary":
            s.rotary = psa.make_rotary(case["dim"], layout=psa.ROTARY_HALF if case["layout"] == "half" else psa.ROTARY_INTERLEAVED,
                                       scaling={"plain": psa.ROTARY_PLAIN, "linear": psa.ROTARY_LINEAR, "base": psa.ROTARY_BASE,
                                                "parts": psa.ROTARY_PARTS}[case["scaling"]], **_scaling(case))
    return s


def _scaling(case):
    return dict(base=10000.0, factor=case["factor"], original_length=2048.0, fast_turns=32.0, slow_turns=1.0,
                magnitude=1 + 0.1 * math.log(case["factor"]) if case["scaling"] == "parts" else 1.0)


def run(s):
    case = s.case
    return (_own if own else _plain)[case["op"], case["what"]](s)


# ------------------------------------------------------------------------------------------------- the library's calls
def _own_norm(s):
    return s.psa.probsparse_layer_norm_fwd(s.X, s.gamma, s.beta, EPS, stats=False)


def _own_norm_train(s):
    Y, mean, rstd = s.psa.probsparse_layer_norm_fwd(s.X, s.gamma, s.beta, EPS)
    return (Y, *s.psa.probsparse_layer_norm_bwd(s.dY, s.X, s.gamma, mean, rstd))


def _own_rotary(s):
    return s.psa.probsparse_rotary_fwd(s.Q, s.K, s.rotary, positions=s.positions, first=s.case["start"])


def _own_rotary_bwd(s):
    return s.psa.probsparse_rotary_bwd(s.Q, s.K, s.rotary, positions=s.positions, first=s.case["start"])


def _own_attn(s):
    return s.psa.dense_attn_packed_fwd(s.Q, s.K, s.V, s.q_off, s.k_off, causal=s.case["causal"])


def _own_attn_train(s):
    out, lse = s.psa.dense_attn_packed_fwd(s.Q, s.K, s.V, s.q_off, s.k_off, causal=s.case["causal"], lse=True)
    return (out, *s.psa.dense_attn_packed_bwd(s.Q, s.K, s.V, out, lse, s.dOut, s.q_off, s.k_off, causal=s.case["causal"]))


_own = {("norm", "serve"): _own_norm, ("norm", "train"): _own_norm_train, ("rotary", "fwd"): _own_rotary,
        ("rotary", "bwd"): _own_rotary_bwd, ("attn", "serve"): _own_attn, ("attn", "train"): _own_attn_train}


# ----------------------------------------------------------------------------------------------------- the plain forms
def _plain_norm_parts(s):
    x = s.X.float()
    d = x - x.mean(1, keepdim=True)
    rstd = torch.rsqrt((d * d).mean(1, keepdim=True) + EPS)
    xhat = d * rstd
    y = xhat
    if s.gamma is not None:
        y = y * s.gamma.float() + s.beta.float()
    return y.to(s.X.dtype), xhat, rstd


def _plain_norm(s):
    return _plain_norm_parts(s)[0]


def _plain_norm_train(s):
    Y, xhat, rstd = _plain_norm_parts(s)
    dY = s.dY.float()
    g = dY if s.gamma is None else dY * s.gamma.float()
    dX = rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    return Y, dX.to(s.X.dtype), (dY * xhat).sum(0), dY.sum(0)


def _frequencies(case):
    """Radians per position of each rotated pair, float64 on the CPU."""
    o = _scaling(case)
    dim, base = case["dim"], o["base"]
    if case["scaling"] == "base" and dim > 2:
        base = base * o["factor"] ** (dim / (dim - 2))
    f = torch.tensor([base ** (-2.0 * i / dim) for i in range(dim // 2)], dtype=torch.float64)
    if case["scaling"] == "linear":
        f = f / o["factor"]
    if case["scaling"] == "parts":
        turns = o["original_length"] * f / (2 * math.pi)
        keep = ((turns - o["slow_turns"]) / (o["fast_turns"] - o["slow_turns"])).clamp(0, 1)
        f = f * keep + f / o["factor"] * (1 - keep)
    return f


def _angles(s):
    case = s.case
    if s.positions is None:
        p = torch.arange(case["start"], case["start"] + case["L"], device="cuda", dtype=torch.float64).expand(case["B"], -1)
    else:
        p = s.positions.double()
    return p[:, None, :, None] * _frequencies(case).cuda()       # [B, 1, L, dim / 2]


def _plain_rotary_with(s, sign):
    case = s.case
    angle = _angles(s)
    m = _scaling(case)["magnitude"]
    c, n = (torch.cos(angle) * m).float(), (sign * torch.sin(angle) * m).float()
    outs = []
    for X in (s.Q, s.K):
        y = X.float()
        r = y[..., :case["dim"]]
        if case["layout"] == "half":
            a, b = r.chunk(2, -1)
            r = torch.cat((a * c - b * n, a * n + b * c), -1)
        else:
            a, b = r[..., 0::2], r[..., 1::2]
            r = torch.stack((a * c - b * n, a * n + b * c), -1).flatten(-2)
        outs.append(torch.cat((r, y[..., case["dim"]:]), -1).to(X.dtype))
    return tuple(outs)


def _plain_rotary(s):
    return _plain_rotary_with(s, 1.0)


def _plain_rotary_bwd(s):
    return _plain_rotary_with(s, -1.0)


_CHUNK = 2048      # queries of a sequence whose weights are held at a time


def _plain_weights(s, Q, K, rows, n_q, n_k):
    """Weights of some queries of one sequence: [H_kv, group * rows, keys], float32."""
    case = s.case
    group = case["H"] // case["H_kv"]
    scores = Q.reshape(case["H_kv"], -1, D) @ K.transpose(1, 2) / math.sqrt(D)
    if case["causal"]:
        last = torch.arange(rows.start, rows.stop, device="cuda").repeat(group) + (n_k - n_q)
        scores = scores.masked_fill(torch.arange(n_k, device="cuda")[None, :] > last[:, None], float("-inf"))
    p = torch.exp(scores - scores.amax(2, keepdim=True))
    return p / p.sum(2, keepdim=True)


def _plain_sequences(s):
    case = s.case
    for b in range(case["B"]):
        q0, q1, k0, k1 = s.q_offsets[b], s.q_offsets[b + 1], s.k_offsets[b], s.k_offsets[b + 1]
        K, V = s.K[:, k0:k1].float(), s.V[:, k0:k1].float()
        for r0 in range(0, q1 - q0, _CHUNK):
            rows = range(r0, min(q1 - q0, r0 + _CHUNK))
            Q = s.Q[:, q0 + rows.start:q0 + rows.stop].float()
            yield slice(q0 + rows.start, q0 + rows.stop), slice(k0, k1), Q, K, V, _plain_weights(s, Q, K, rows, q1 - q0, k1 - k0)


def _plain_attn(s):
    out = torch.empty_like(s.Q)
    for q, _, Q, _, V, p in _plain_sequences(s):
        out[:, q] = (p @ V).reshape(Q.shape).to(out.dtype)
    return out


def _plain_attn_train(s):
    out, dQ = torch.empty_like(s.Q), torch.empty_like(s.Q)
    dK, dV = (torch.zeros(s.K.shape, dtype=torch.float32, device="cuda") for _ in range(2))
    for q, k, Q, K, V, p in _plain_sequences(s):
        o = p @ V
        G = s.dOut[:, q].float().reshape(o.shape)
        dp = G @ V.transpose(1, 2)
        ds = p * (dp - (p * dp).sum(2, keepdim=True)) / math.sqrt(D)
        out[:, q] = o.reshape(Q.shape).to(out.dtype)
        dQ[:, q] = (ds @ K).reshape(Q.shape).to(dQ.dtype)
        dK[:, k] += ds.transpose(1, 2) @ Q.reshape(o.shape)
        dV[:, k] += p.transpose(1, 2) @ G
    return out, dQ, dK.to(s.K.dtype), dV.to(s.V.dtype)


_plain = {("norm", "serve"): _plain_norm, ("norm", "train"): _plain_norm_train, ("rotary", "fwd"): _plain_rotary,
          ("rotary", "bwd"): _plain_rotary_bwd, ("attn", "serve"): _plain_attn, ("attn", "train"): _plain_attn_train}


# ------------------------------------------------------------------------------------------------ the values in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"norm": _exact_norm, "rotary": _exact_rotary, "attn": _exact_attn}[case["op"]](s)


def _exact_norm(s):
    x = s.X.double()
    n = x.shape[1]
    mean = x.sum(1, keepdim=True) / n
    sigma = (((x - mean) ** 2).sum(1, keepdim=True) / n + EPS).sqrt()
    gamma = torch.ones(n, dtype=torch.float64, device="cuda") if s.gamma is None else s.gamma.double()
    beta = torch.zeros_like(gamma) if s.beta is None else s.beta.double()
    xhat = (x - mean) / sigma
    y = gamma * xhat + beta
    if s.case["what"] == "serve":
        return y
    dxhat = s.dY.double() * gamma
    # through xhat = (x - mean) / sigma: what is left of dxhat beside its parts along 1 and along xhat
    dx = (n * dxhat - dxhat.sum(1, keepdim=True) - xhat * (dxhat * xhat).sum(1, keepdim=True)) / (n * sigma)
    return y, dx, (s.dY.double() * xhat).sum(0), s.dY.double().sum(0)


def _exact_rotary(s):
    """Each pair (a, b) as the complex number a + ib, times m e^(i angle), or e^(-i angle) for the gradient."""
    case = s.case
    o = _scaling(case)
    half = case["dim"] // 2
    index = torch.arange(half, dtype=torch.float64, device="cuda")
    log_base = math.log(o["base"])
    if case["scaling"] == "base" and case["dim"] > 2:
        log_base += math.log(o["factor"]) * case["dim"] / (case["dim"] - 2)
    freq = torch.exp(-log_base * index / half)
    if case["scaling"] == "linear":
        freq = freq / o["factor"]
    elif case["scaling"] == "parts":
        share = (freq * (o["original_length"] / (2 * math.pi)) - o["slow_turns"]) / (o["fast_turns"] - o["slow_turns"])
        share = torch.clamp(share, 0.0, 1.0)
        freq = (1 - share) * (freq / o["factor"]) + share * freq
    steps = torch.arange(case["L"], device="cuda").double()[None] + case["start"] if s.positions is None else s.positions.double()
    angle = steps[:, None, :, None] * freq
    turn = torch.polar(torch.full_like(angle, o["magnitude"]), angle if case["what"] == "fwd" else -angle)
    even = (torch.arange(half) if case["layout"] == "half" else 2 * torch.arange(half)).cuda()
    odd = even + (half if case["layout"] == "half" else 1)
    outs = []
    for X in (s.Q, s.K):
        y = X.double().clone()
        z = torch.complex(y[..., even], y[..., odd]) * turn
        y[..., even], y[..., odd] = z.real, z.imag
        outs.append(y)
    return tuple(outs)


def _exact_attn(s):
    """One query head and one block of queries at a time."""
    case = s.case
    train = case["what"] == "train"
    if _pairs(case) * case["H"] * (7 if train else 2) > 1.5e10:      # 128 flops for each, well under 20 s
        return None
    group = case["H"] // case["H_kv"]
    out = torch.zeros(s.Q.shape, dtype=torch.float64, device="cuda")
    if train:
        dQ, dK, dV = (torch.zeros(x.shape, dtype=torch.float64, device="cuda") for x in (s.Q, s.K, s.V))
    for b in range(case["B"]):
        q0, q1, k0, k1 = s.q_offsets[b], s.q_offsets[b + 1], s.k_offsets[b], s.k_offsets[b + 1]
        for h in range(case["H"]):
            K, V = s.K[h // group, k0:k1].double(), s.V[h // group, k0:k1].double()
            for i in range(q0, q1, 4096):
                j = min(q1, i + 4096)
                Q = s.Q[h, i:j].double()
                e = torch.mm(Q, K.t().contiguous()).mul_(0.125)
                if case["causal"]:     # the last query of a sequence sees its last key
                    behind = torch.arange(k1 - k0, device="cuda")[None, :] - (torch.arange(i, j, device="cuda")[:, None] - q1 + (k1 - k0))
                    e[behind > 0] = float("-inf")
                p = torch.softmax(e, 1)
                out[h, i:j] = torch.mm(p, V)
                if train:
                    G = s.dOut[h, i:j].double()
                    w = torch.mm(G, V.t().contiguous())
                    w = p * (w - (G * out[h, i:j]).sum(1, keepdim=True)) * 0.125
                    dQ[h, i:j] = torch.mm(w, K)
                    dK[h // group, k0:k1] += torch.mm(w.t().contiguous(), Q)
                    dV[h // group, k0:k1] += torch.mm(p.t().contiguous(), G)
    return (out, dQ, dK, dV) if train else out
