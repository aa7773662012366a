"""Refusals of layer norm, rotary positions and packed attention: argument checks run before anything touches the GPU."""
import ctypes
import math

import pytest
import torch

from paper_2106_09236_amd import binding as psa

NULL, SHAPE, DTYPE, ARG, WORKSPACE, ALIGN = -1, -2, -3, -4, -5, -7
BF16, F32 = psa.PSA_BF16, psa.PSA_F32


def _ref(x):
    return None if x is None else ctypes.byref(x)


def test_layer_norm_refusals():
    lib = psa.load()

    def fwd(X=0x1000, gamma=0x2000, beta=0x3000, eps=1e-5, Y=0x4000, mean=0x5000, rstd=0x6000, rows=4, cols=8, dtype=F32):
        return lib.probsparse_layer_norm_fwd(X, gamma, beta, eps, Y, mean, rstd, rows, cols, dtype, None)

    def bwd(dY=0x1000, X=0x2000, gamma=0x3000, mean=0x4000, rstd=0x5000, dX=0x6000, dg=0x7000, db=0x8000, rows=4, cols=8, dtype=F32,
            ws=0x10000, n=1 << 40):
        return lib.probsparse_layer_norm_bwd(dY, X, gamma, mean, rstd, dX, dg, db, rows, cols, dtype, ws, n, None)
    for f in (fwd, bwd):
        assert f(X=None) == NULL
        assert f(rows=0) == f(rows=-1) == f(cols=0) == f(cols=(1 << 24) + 1) == f(rows=1 << 31) == SHAPE
        assert f(dtype=2) == f(dtype=-1) == DTYPE
        assert f(X=0x1008) == f(gamma=0x2004) == f(mean=0x5002) == ALIGN
    assert fwd(Y=None) == fwd(mean=None) == fwd(rstd=None) == NULL
    assert fwd(eps=-1e-9) == fwd(eps=math.nan) == fwd(eps=math.inf) == fwd(eps=1e300) == ARG
    assert fwd(Y=0x4001) == fwd(beta=0x3008) == ALIGN
    assert bwd(dY=None) == bwd(mean=None) == bwd(rstd=None) == bwd(dX=None) == bwd(dg=None) == bwd(db=None) == bwd(ws=None) == NULL
    assert bwd(n=16) == WORKSPACE
    assert bwd(ws=0x10010) == bwd(dX=0x6008) == bwd(dg=0x7002) == ALIGN
    size = lib.probsparse_layer_norm_bwd_workspace_bytes
    assert size(4, 8, F32) > 0 and size(4, 8, F32) % 256 == 0
    assert size(0, 8, F32) == size(4, 0, F32) == size(4, 8, 5) == 0
    assert size(1 << 20, 512, BF16) < 1 << 24        # partial rows, not rows


def test_rotary_options():
    bad = [dict(dim=0), dict(dim=3), dict(dim=66), dict(layout=2), dict(scaling=4), dict(base=0.5), dict(base=math.inf), dict(factor=0.0),
           dict(factor=-1.0), dict(factor=math.nan), dict(magnitude=0.0), dict(magnitude=math.inf), dict(magnitude=1e39), dict(magnitude=1e-50), dict(factor=1e-310),
           dict(scaling=psa.ROTARY_PARTS), dict(scaling=psa.ROTARY_PARTS, original_length=100.0, fast_turns=1.0, slow_turns=1.0),
           dict(scaling=psa.ROTARY_BASE, dim=4, base=1e200, factor=1e100)]
    for kw in bad:
        with pytest.raises(psa.ProbSparseError) as e:
            psa.make_rotary(**{"dim": 64, **kw})
        assert e.value.code == ARG, kw


def test_rotary_frequencies():
    f = psa.rotary_frequencies(psa.make_rotary(32, base=100.0))
    assert len(f) == 16 and f[0] == 1.0
    assert all(abs(x - 100.0 ** (-2 * i / 32)) <= 1e-15 * x for i, x in enumerate(f))
    linear = psa.rotary_frequencies(psa.make_rotary(32, base=100.0, scaling=psa.ROTARY_LINEAR, factor=4.0))
    assert all(a == b / 4 for a, b in zip(linear, f))
    base = psa.rotary_frequencies(psa.make_rotary(32, base=100.0, scaling=psa.ROTARY_BASE, factor=4.0))
    assert base[0] == 1.0 and abs(base[-1] * 4 / f[-1] - 1) < 1e-13      # the slowest turns 4 times slower
    assert psa.rotary_frequencies(psa.make_rotary(2, scaling=psa.ROTARY_BASE, factor=4.0)) == [1.0]
    parts = psa.rotary_frequencies(psa.make_rotary(64, scaling=psa.ROTARY_PARTS, factor=8.0, original_length=2048.0))
    plain = psa.rotary_frequencies(psa.make_rotary(64))
    for a, b in zip(parts, plain):
        turns = 2048 * b / (2 * math.pi)
        keep = min(1.0, max(0.0, (turns - 1) / 31))
        assert abs(a - (b * keep + b / 8 * (1 - keep))) <= 1e-15 * b
    assert parts[0] == plain[0] and parts[-1] == plain[-1] / 8


def test_rotary_refusals():
    lib = psa.load()
    spec = psa.make_rotary(64)
    heads = lambda data=0x1000, b=64 * 8 * 10, h=640, r=64: psa.PsaHeads(data, b, h, r)
    shape = lambda **kw: psa.make_shape(**{**dict(B=2, H=8, L=10, U=1, dtype=F32), **kw})

    def call(Q=heads(), K=heads(), H_kv=8, rotary=spec, positions=None, stride=0, first=0, Qo=heads(), Ko=heads(), s=shape(), f=lib.probsparse_rotary_fwd):
        return f(_ref(Q), _ref(K), H_kv, _ref(rotary), positions, stride, first, _ref(Qo), _ref(Ko), _ref(s), None)
    for f in (lib.probsparse_rotary_fwd, lib.probsparse_rotary_bwd):
        assert call(Q=None, f=f) == call(Qo=None, f=f) == call(rotary=None, f=f) == call(s=None, f=f) == call(Ko=None, f=f) == NULL
        assert call(Q=heads(data=None), f=f) == call(K=heads(data=None), f=f) == NULL
        assert call(s=shape(D=32), f=f) == call(s=shape(B=0), f=f) == call(s=shape(L=0), f=f) == call(H_kv=0, f=f) == call(s=shape(L_Q=3), f=f) == SHAPE
        assert call(s=shape(B=65536), f=f) == SHAPE
        assert call(s=shape(dtype=3), f=f) == DTYPE
        assert call(rotary=psa.PsaRotary(7), f=f) == ARG
        assert call(first=2 ** 31 - 5, f=f) == ARG
        assert call(positions=0x100, stride=9, f=f) == ARG
        assert call(positions=0x102, stride=0, f=f) == ALIGN
        assert call(Qo=heads(r=0), f=f) == call(Qo=heads(h=32), f=f) == call(Q=heads(r=-64), f=f) == ARG
        assert call(Q=heads(data=0x1008), f=f) == call(Q=heads(h=642), f=f) == call(Ko=heads(r=66), f=f) == ALIGN


def _packed(B=2, H=4, H_kv=2, T_q=10, T_k=20, D=64, dtype=F32, causal=1, scale=0.125):
    return psa.PsaPackedShape(B, H, H_kv, T_q, T_k, D, dtype, causal, scale)


@pytest.mark.parametrize("backward", [False, True])
def test_packed_attention_refusals(backward):
    lib = psa.load()
    names = ["Q", "K", "V", "out"] + (["dOut", "dQ", "dK", "dV"] if backward else [])
    outputs = ["dQ", "dK", "dV"] if backward else ["out"]

    def call(shape=_packed(), qo=0x100, ko=0x200, lse=0x300, ws=0x10000, n=1 << 40, **heads):
        t = {name: heads.get(name, psa.PsaHeads(0x1000, 0, 64 * 20, 64)) for name in names}
        if backward:
            return lib.dense_attn_packed_bwd(*(_ref(t[x]) for x in "QKV"), qo, ko, _ref(t["out"]), lse, *(_ref(t[x]) for x in names[4:]),
                                             _ref(shape), ws, n, None)
        return lib.dense_attn_packed_fwd(*(_ref(t[x]) for x in "QKV"), qo, ko, _ref(t["out"]), lse, _ref(shape), ws, n, None)
    for name in names:
        assert call(**{name: None}) == call(**{name: psa.PsaHeads(None, 0, 1280, 64)}) == NULL
        assert call(**{name: psa.PsaHeads(0x1004, 0, 1280, 64)}) == call(**{name: psa.PsaHeads(0x1000, 0, 1282, 64)}) == ALIGN
        assert call(**{name: psa.PsaHeads(0x1000, 0, 1280, -64)}) == call(**{name: psa.PsaHeads(0x1000, 0, 1280, 1 << 23)}) == ARG
    for name in outputs:
        assert call(**{name: psa.PsaHeads(0x1000, 0, 1280, 0)}) == call(**{name: psa.PsaHeads(0x1000, 0, 0, 64)}) == ARG
    assert call(shape=None) == call(ws=None) == call(qo=None) == call(ko=None) == call(qo=None, ko=None) == NULL
    for kw in (dict(B=0), dict(H=0), dict(H_kv=0), dict(H=3), dict(T_q=0), dict(T_k=0), dict(D=128), dict(H=70000, H_kv=1), dict(T_q=1 << 29)):
        assert call(shape=_packed(**kw)) == SHAPE, kw
    assert call(shape=_packed(H=64, H_kv=1, T_q=1 << 26)) == SHAPE           # rows of a key head beyond 31 bits
    assert call(shape=_packed(B=1 << 20, H=64, H_kv=64, T_q=1 << 20, T_k=1 << 20)) == SHAPE      # 2^32 threads and more
    assert call(shape=_packed(B=1 << 20, H=16, H_kv=4, T_q=1 << 20, T_k=1 << 20), n=0) == WORKSPACE
    assert call(shape=_packed(dtype=9)) == DTYPE
    for kw in (dict(causal=2), dict(causal=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan), dict(scale=math.inf), dict(scale=1e-40), dict(scale=1e40)):
        assert call(shape=_packed(**kw)) == ARG, kw
    assert call(qo=0x101) == call(lse=0x302) == call(ws=0x10080) == ALIGN
    assert call(n=0) == WORKSPACE
    if backward:
        assert call(lse=None) == NULL
    for f in (lib.dense_attn_packed_workspace_bytes, lib.dense_attn_packed_bwd_workspace_bytes):
        assert f(ctypes.byref(_packed())) > 0 and f(ctypes.byref(_packed())) % 256 == 0
        assert f(ctypes.byref(_packed(D=32))) == f(ctypes.byref(_packed(scale=0.0))) == 0


def test_binding_refuses_before_a_call():
    cpu = torch.zeros(4, 10, 64)
    with pytest.raises(ValueError):
        psa.probsparse_layer_norm_fwd(cpu)
    with pytest.raises(ValueError):
        psa.dense_attn_packed_fwd(cpu, cpu, cpu)
    with pytest.raises(ValueError):
        psa.probsparse_rotary_fwd(cpu, cpu, psa.make_rotary(64))


@pytest.mark.gpu
def test_binding_refuses_wrong_tensors():
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(*s, dtype=dtype, device="cuda")
    q, k = z(4, 10, 64), z(2, 10, 64)
    off = torch.tensor([0, 10], dtype=torch.int32, device="cuda")
    for args in ((q, k, z(2, 11, 64)), (z(3, 10, 64), k, k), (z(4, 10, 32), k, k), (q, k, k, off[:1]), (q, z(2, 9, 64), z(2, 9, 64), off),
                 (q, k, k, None, off), (q, k, k, off, torch.tensor([0, 3, 10], dtype=torch.int32, device="cuda")),
                 (q, z(2, 64, 10).transpose(1, 2), k), (q, k, k, off.cpu())):
        with pytest.raises(ValueError):
            psa.dense_attn_packed_fwd(*args)
    with pytest.raises(TypeError):
        psa.dense_attn_packed_fwd(q, k, k.float())
    with pytest.raises(TypeError):
        psa.dense_attn_packed_fwd(q, k, k, off.long())
    with pytest.raises(TypeError):
        psa.dense_attn_packed_fwd(q.half(), k.half(), k.half())
    with pytest.raises(psa.ProbSparseError):
        psa.dense_attn_packed_fwd(q, k, k, off, scale=-1.0)
    with pytest.raises(psa.ProbSparseError):
        psa.dense_attn_packed_fwd(q, k, k, off, out=z(10, 64)[None].expand(4, 10, 64))
    with pytest.raises(ValueError):
        psa.dense_attn_packed_bwd(q, k, k, q, z(4, 9, dtype=torch.float32), q, off)
    x = z(6, 32)
    for kw in (dict(gamma=z(31)), dict(Y=z(6, 31)), dict(beta=z(64)[::2])):
        with pytest.raises(ValueError):
            psa.probsparse_layer_norm_fwd(x, **kw)
    with pytest.raises(TypeError):
        psa.probsparse_layer_norm_fwd(x, z(32, dtype=torch.float32))
    with pytest.raises(ValueError):
        psa.probsparse_layer_norm_fwd(z(32, 6).t())
    spec = psa.make_rotary(64)
    for args, kw in (((q, z(2, 9, 64), spec), {}), ((q[..., :32], None, spec), {}), ((q, None, spec), dict(positions=z(9, dtype=torch.int32)))):
        with pytest.raises(ValueError):
            psa.probsparse_rotary_fwd(*args, **kw)
    with pytest.raises(TypeError):
        psa.probsparse_rotary_fwd(q, None, spec, positions=z(10, dtype=torch.int64))


@pytest.mark.gpu
def test_ctypes_path_gives_the_same(monkeypatch):
    g = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)
    q, k, v, d, x, w = rand(4, 50, 64), rand(2, 50, 64), rand(2, 50, 64), rand(4, 50, 64), rand(9, 5, 96), rand(96)
    off = torch.tensor([0, 20, 50], dtype=torch.int32, device="cuda")
    pos = torch.arange(50, dtype=torch.int32, device="cuda")
    spec = psa.make_rotary(64)

    def calls():
        y, mean, rstd = psa.probsparse_layer_norm_fwd(x, w, w, 1e-5)
        out, lse = psa.dense_attn_packed_fwd(q, k, v, off, causal=True, scale=0.2, lse=True)
        return [y, mean, rstd, psa.probsparse_layer_norm_fwd(x, w, None, stats=False), *psa.probsparse_layer_norm_bwd(x, x, w, mean, rstd),
                *psa.probsparse_rotary_fwd(q, k, spec, positions=pos), psa.probsparse_rotary_bwd(q, None, spec, first=7), out, lse,
                psa.dense_attn_packed_fwd(q, k, v), *psa.dense_attn_packed_bwd(q, k, v, out, lse, d, off, causal=True, scale=0.2)]
    native = calls()
    assert psa._native is not psa._CtypesOnly
    monkeypatch.setattr(psa, "_native", psa._CtypesOnly)
    other = calls()
    assert all(a.shape == b.shape and a.dtype == b.dtype and torch.equal(a, b) for a, b in zip(native, other))
