"""Dense attention over packed sequences, forward and backward, against float64."""
import math

import pytest
import torch

from paper_2106_09236_amd import binding as psa
from tests.operator_bounds import HALF, assert_within, packed_attention

pytestmark = pytest.mark.gpu


def _offsets(lens, front=0):
    off = [front]
    for n in lens:
        off.append(off[-1] + n)
    return off


def _tensor(heads, rows, dtype, g, by_frame, wide=False):
    x = torch.randn((rows, heads, 64) if by_frame else (heads, rows, 64), generator=g)
    if wide:
        x = x * (1 + 5 * (torch.rand(x.shape[:-1], generator=g) < 0.1).unsqueeze(-1))
    x = x.to(dtype)
    d = x.cuda()
    return (x.transpose(0, 1), d.transpose(0, 1)) if by_frame else (x, d)


def _case(H, H_kv, q_lens, k_lens, dtype, by_frame=False, front=0, behind=0, wide=True, seed=0):
    g = torch.Generator().manual_seed(seed + 17 * sum(q_lens) + sum(k_lens))
    q_off, k_off = _offsets(q_lens, front), _offsets(k_lens, front)
    Q, Qd = _tensor(H, q_off[-1] + behind, dtype, g, by_frame, wide)
    K, Kd = _tensor(H_kv, k_off[-1] + behind, dtype, g, by_frame)
    V, Vd = _tensor(H_kv, k_off[-1] + behind, dtype, g, by_frame)
    G, Gd = _tensor(H, q_off[-1] + behind, dtype, g, by_frame)
    return (Q, K, V, G), (Qd, Kd, Vd, Gd), q_off, k_off


def _check(host, dev, q_off, k_off, causal, scale=0.125, backward=True):
    Q, K, V, G = host
    Qd, Kd, Vd, Gd = dev
    qo, ko = (torch.tensor(o, dtype=torch.int32, device="cuda") for o in (q_off, k_off))
    out = torch.full_like(Qd, float("nan"))
    _, lse = psa.dense_attn_packed_fwd(Qd, Kd, Vd, qo, ko, causal=causal, scale=scale, out=out, lse=True)
    want = packed_attention(Q, K, V, q_off, k_off, causal, scale, G if backward else None)
    assert_within(out, want[0][0], want[0][1], "out")
    empty = want[1][0].isinf()
    assert torch.equal(lse.cpu().isinf(), empty) and not (lse.cpu()[empty] > 0).any()
    assert_within(lse.cpu().masked_fill(empty, 0.0), want[1][0].masked_fill(empty, 0.0), want[1][1].masked_fill(empty, 1.0), "lse")
    assert torch.equal(psa.dense_attn_packed_fwd(Qd, Kd, Vd, qo, ko, causal=causal, scale=scale), out)
    if not backward:
        return
    grads = [torch.full_like(t, float("nan")) for t in (Qd, Kd, Vd)]
    psa.dense_attn_packed_bwd(Qd, Kd, Vd, out, lse, Gd, qo, ko, causal=causal, scale=scale, dQ=grads[0], dK=grads[1], dV=grads[2])
    for g, (w, e), what in zip(grads, want[2:], ("dQ", "dK", "dV")):
        assert_within(g, w, e, what)
    again = psa.dense_attn_packed_bwd(Qd, Kd, Vd, out, lse, Gd, qo, ko, causal=causal, scale=scale)
    assert all(torch.equal(a, b) for a, b in zip(again, grads))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("H,H_kv,lens,by_frame", [
    (1, 1, [1], False), (2, 2, [2, 1, 3], True), (4, 4, [31, 32, 33], False), (4, 2, [63, 64, 65, 1], True), (8, 2, [127, 5, 128, 129], False),
    (4, 1, [0, 17, 0, 0, 100, 0], False), (3, 3, [255, 257], True), (6, 2, [333], False), (2, 1, [700], True),
    (4, 4, [3] * 70, False), (2, 2, [1] * 130, True)])
def test_whole_sequences(H, H_kv, lens, by_frame, causal, dtype):
    _check(*_case(H, H_kv, lens, lens, dtype, by_frame), causal)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("H,H_kv,q_lens,k_lens", [
    (128, 64, [127, 0, 5, 128, 129, 65, 300], [127, 0, 5, 128, 129, 65, 300]), (96, 32, [111, 222, 1, 90], [70, 222, 150, 0]),
    (64, 64, [260, 255, 256, 1], [257, 300, 256, 33]), (32, 16, [500, 401, 390], [500, 401, 390]), (32, 32, [300, 1, 400], [700, 300, 401])])
def test_many_heads(H, H_kv, q_lens, k_lens, causal, dtype):
    """Enough heads for work-groups of 128 rows (fewer leave the card idle, and rows are taken 32 at a time)."""
    _check(*_case(H, H_kv, q_lens, k_lens, dtype, by_frame=causal, front=3, behind=200), causal)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("H,H_kv,q_lens,k_lens", [
    (8, 2, [1] * 5, [1, 40, 129, 600, 0]),              # single tokens; one stream without keys
    (4, 4, [1], [5000]), (8, 1, [3, 1], [2047, 2049]),  # long caches
    (4, 2, [20, 5, 64, 7], [10, 5, 300, 0]),            # more queries than keys: the first see none under the mask
    (4, 2, [0, 9, 0], [30, 0, 12]),                     # keys that no query reads: zero gradients
    (2, 2, [130], [67])])
def test_queries_and_keys_of_other_lengths(H, H_kv, q_lens, k_lens, causal, dtype):
    _check(*_case(H, H_kv, q_lens, k_lens, dtype), causal)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("H,H_kv,B,longest", [(2, 1, 256, 5), (2, 1, 257, 5), (2, 2, 700, 9), (1, 1, 5000, 3), (32, 32, 300, 70)])
def test_many_sequences(H, H_kv, B, longest, causal, dtype):
    """Hundreds of sequences, empty ones and a long one among them, the last group of 64 not full."""
    g = torch.Generator().manual_seed(B)
    q_lens = torch.randint(0, longest + 1, (B,), generator=g).tolist()
    k_lens = [n + int(e) for n, e in zip(q_lens, torch.randint(0, 3, (B,), generator=g))]
    q_lens[B // 3] = k_lens[B // 3] = 300 if H < 32 else 100
    k_lens[2] = 0
    _check(*_case(H, H_kv, q_lens, k_lens, dtype, behind=7), causal)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_few_queries_of_many_keys_with_gradients(dtype):
    """Rows taken 32 at a time, keys 128 at a time."""
    _check(*_case(16, 16, [40], [2500], dtype), True)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("H,H_kv,q_lens,k_lens", [
    (8, 1, [700, 0, 1, 333], [700, 5, 1, 333]), (4, 1, [1500], [1500]), (6, 2, [1900, 260], [300, 40]), (64, 2, [1, 40, 511], [130, 300, 511]),
    (2, 2, [2100], [2100])])
def test_keys_of_many_rows(H, H_kv, q_lens, k_lens, causal, dtype):
    """Few keys that many rows read, those of a group's heads together: the rows are divided among work-groups.  Sequences of one
    key, without rows or without keys among them, and rows of no sequence before and behind."""
    _check(*_case(H, H_kv, q_lens, k_lens, dtype, by_frame=causal, front=5, behind=40), causal)


def test_offsets_beyond_31_bits():
    """K and V as columns of a cache whose rows are 8 MB apart: element offsets up to 2^32."""
    n, wide = 1024, 1 << 22
    cache = torch.empty(n, wide, dtype=torch.bfloat16, device="cuda")
    (Q, K, V, G), (Qd, Kd, Vd, Gd), q_off, k_off = _case(2, 1, [3, 70], [600, n - 600], torch.bfloat16)
    kv = cache[:, wide - 128:].unflatten(1, (2, 64))
    kv[:, 0], kv[:, 1] = Kd[0], Vd[0]
    Kc, Vc = kv[:, :1].transpose(0, 1), kv[:, 1:].transpose(0, 1)
    qo, ko = (torch.tensor(o, dtype=torch.int32, device="cuda") for o in (q_off, k_off))
    out, lse = psa.dense_attn_packed_fwd(Qd, Kc, Vc, qo, ko, causal=True, lse=True)
    want = packed_attention(Q, K, V, q_off, k_off, True, 0.125, G)
    grads = psa.dense_attn_packed_bwd(Qd, Kc, Vc, out, lse, Gd, qo, ko, causal=True)
    for g, (w, e) in zip((out, lse, *grads), want):
        assert_within(g, w, e)
    with pytest.raises(psa.ProbSparseError):          # a wider row would pass the limit of offsets within a tile
        psa.dense_attn_packed_fwd(Qd, cache.view(-1)[:64 * 2].view(1, 2, 64).as_strided((1, 2, 64), (0, wide + 8, 1)), Vc[:, :2], torch.tensor([0, 73], dtype=torch.int32, device="cuda"),
                                  torch.tensor([0, 2], dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("lens", [[270], [40, 130]])
def test_rows_far_apart_float32(lens):
    """K and V with rows 16 MB apart: 270 rows are beyond 32 bits of bytes, 129 beyond 31."""
    wide = 1 << 22
    (Q, K, V, G), (Qd, Kd, Vd, Gd), q_off, k_off = _case(2, 1, lens, lens, torch.float32)
    cache = torch.empty(k_off[-1], wide, device="cuda")
    kv = cache[:, wide - 128:].unflatten(1, (2, 64))
    kv[:, 0], kv[:, 1] = Kd[0], Vd[0]
    _check((Q, K, V, G), (Qd, kv[:, :1].transpose(0, 1), kv[:, 1:].transpose(0, 1), Gd), q_off, k_off, True)


def test_two_streams_at_once():
    """Calls on two streams, each with a workspace of its own, give what they give alone."""
    a = _case(8, 2, [1] * 9, [2000] * 9, torch.bfloat16)
    b = _case(4, 4, [300, 500], [300, 500], torch.float32)
    def run(case, causal=True):
        _, (Qd, Kd, Vd, Gd), q_off, k_off = case
        qo, ko = case_offsets[id(case)]
        out, lse = psa.dense_attn_packed_fwd(Qd, Kd, Vd, qo, ko, causal=causal, lse=True)
        return (out, lse, *psa.dense_attn_packed_bwd(Qd, Kd, Vd, out, lse, Gd, qo, ko, causal=causal))
    case_offsets = {id(c): [torch.tensor(o, dtype=torch.int32, device="cuda") for o in c[2:]] for c in (a, b)}
    ref = [run(a), run(b)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for s, c in zip(streams, (a, b)):
            with torch.cuda.stream(s):
                got.append(run(c))
    torch.cuda.synchronize()
    for i, g in enumerate(got):
        assert all(torch.equal(x, y) for x, y in zip(g, ref[i % 2]))


def test_one_key_has_no_gradient_but_its_value():
    for dtype in (torch.float32, torch.bfloat16):
        for H, H_kv, lens in ((4, 2, [1] * 7), (64, 64, [1] * 300)):
            host, (Qd, Kd, Vd, Gd), q_off, k_off = _case(H, H_kv, lens, lens, dtype)
            off = torch.tensor(q_off, dtype=torch.int32, device="cuda")
            out, lse = psa.dense_attn_packed_fwd(Qd, Kd, Vd, off, causal=True, lse=True)
            dQ, dK, dV = psa.dense_attn_packed_bwd(Qd, Kd, Vd, out, lse, Gd, off, causal=True)
            assert not dQ.any() and not dK.any()
            # p is 1 but for the rounding of the score that is subtracted, and its sum is p: p V and 1 / p are left.  In half steps
            # of float32: 2 for the parts of a product, 1 for their sum, 1 for the reciprocal, 1 for the product with it; then the tensor's own
            v = Vd.repeat_interleave(H // H_kv, 0).cpu().double()
            assert_within(out, v, (5 * 2.0 ** -24 + HALF[dtype]) * v.abs())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_in_no_sequence(dtype):
    _check(*_case(4, 2, [40, 9], [60, 30], dtype, by_frame=True, front=150, behind=300), True)
    _check(*_case(2, 2, [0, 0], [0, 0], dtype, behind=5), False)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_one_sequence_without_offsets(dtype):
    (Q, K, V, G), dev, q_off, k_off = _case(4, 2, [100], [150], dtype)
    Qd, Kd, Vd, Gd = dev
    out, lse = psa.dense_attn_packed_fwd(Qd, Kd, Vd, causal=True, scale=0.3, lse=True)
    want = packed_attention(Q, K, V, q_off, k_off, True, 0.3, G)
    got = (out, lse, *psa.dense_attn_packed_bwd(Qd, Kd, Vd, out, lse, Gd, causal=True, scale=0.3))
    for g, (w, e) in zip(got, want):
        assert_within(g, w, e)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("H,H_kv,q_lens,k_lens", [(4, 2, [200, 90], [200, 90]), (4, 2, [4, 2], [300, 90]), (64, 32, [200, 290], [200, 290])])
def test_what_is_not_seen_has_no_part(H, H_kv, q_lens, k_lens, dtype):
    """Infinities and NaN in later keys and values, in other sequences and between them leave a row's output as it is."""
    host, dev, q_off, k_off = _case(H, H_kv, q_lens, k_lens, dtype, front=20, behind=30)
    Qd, Kd, Vd, _ = dev
    qo, ko = (torch.tensor(o, dtype=torch.int32, device="cuda") for o in (q_off, k_off))
    clean, clean_lse = psa.dense_attn_packed_fwd(Qd, Kd, Vd, qo, ko, causal=True, lse=True)
    for value in (float("nan"), float("inf"), -float("inf")):
        bad = k_off[1] - 1                       # the last key of the first sequence: its last query alone sees it
        K2, V2 = Kd.clone(), Vd.clone()
        for t in (K2, V2):
            t[:, :k_off[0]] = value
            t[:, k_off[-1]:] = value
        V2[:, bad, 5] = value
        out, lse = psa.dense_attn_packed_fwd(Qd, K2, V2, qo, ko, causal=True, lse=True)
        rows = [i for i in range(Qd.shape[1]) if i != q_off[1] - 1]
        assert torch.equal(out[:, rows], clean[:, rows]) and torch.equal(lse, clean_lse)
        hit = out[:, q_off[1] - 1].float().cpu()
        assert (hit[:, 5].isnan().all() if value != value else (hit[:, 5] == value).all()) and hit[:, [0, 4, 6, 63]].isfinite().all()
        K2[:, bad, 3] = float("nan")
        out = psa.dense_attn_packed_fwd(Qd, K2, V2, qo, ko, causal=True)
        assert torch.equal(out[:, rows], clean[:, rows]) and out[:, q_off[1] - 1].isnan().all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradients_of_one_sequence_do_not_reach_another(dtype):
    host, dev, q_off, k_off = _case(4, 2, [50, 90, 40], [50, 90, 40], dtype)
    Qd, Kd, Vd, Gd = dev
    off = torch.tensor(q_off, dtype=torch.int32, device="cuda")
    grads = lambda Q, V, G: psa.dense_attn_packed_bwd(Q, Kd, V, *psa.dense_attn_packed_fwd(Q, Kd, V, off, causal=True, lse=True), G, off, causal=True)
    clean = grads(Qd, Vd, Gd)
    Q2, V2, G2 = Qd.clone(), Vd.clone(), Gd.clone()
    for t in (Q2, V2, G2):
        t[:, 60:70] = float("nan")
    for a, b in zip(grads(Q2, V2, G2), clean):
        assert torch.equal(a[:, :50], b[:, :50]) and torch.equal(a[:, 140:], b[:, 140:])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_large_scores(dtype):
    """Scores of some hundreds: one key has all the weight, and no exponential overflows."""
    host, dev, q_off, k_off = _case(2, 2, [70], [200], dtype, wide=False)
    host[0].mul_(40.0)
    dev[0].mul_(40.0)
    _check(host, dev, q_off, k_off, False)
    _check(host, dev, q_off, k_off, True)


def test_offsets_out_of_range_are_clamped():
    """What the header says of bad offsets; nothing outside the tensors is read or written (rows of other sequences are as ever)."""
    host, dev, _, _ = _case(2, 1, [64], [64], torch.bfloat16)
    Qd, Kd, Vd, _ = dev
    bad = torch.tensor([-7, 30, 1 << 30], dtype=torch.int32, device="cuda")
    good = torch.tensor([0, 30, 64], dtype=torch.int32, device="cuda")
    a = psa.dense_attn_packed_fwd(Qd, Kd, Vd, bad, causal=True, lse=True)
    b = psa.dense_attn_packed_fwd(Qd, Kd, Vd, good, causal=True, lse=True)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    # decreasing offsets: the first sequence's rows that no other claims
    back = torch.tensor([0, 30, 20, 64], dtype=torch.int32, device="cuda")
    out = psa.dense_attn_packed_fwd(Qd, Kd, Vd, back, causal=True)
    assert torch.equal(out[:, :20], b[0][:, :20])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_decreasing_offsets_of_many_sequences(dtype):
    """600 sequences of which every other claims all rows: together more tiles than there are work-groups.  The tensors are parts of
    larger ones, and what lies around them stays as it was; the next call is as ever."""
    T, B = 500, 600
    host, dev, q_off, _ = _case(4, 2, [T], [T], dtype)
    off = torch.tensor([0, T] * (B // 2) + [0], dtype=torch.int32, device="cuda")

    def around(heads):
        whole = torch.full((heads, T + 64, 64), 7.0, dtype=dtype, device="cuda")
        return whole, whole[:, 32:32 + T]
    (o_all, out), *grads = around(4), around(4), around(2), around(2)
    _, lse = psa.dense_attn_packed_fwd(*dev[:3], off, causal=True, out=out, lse=True)
    psa.dense_attn_packed_bwd(*dev[:3], out, lse, dev[3], off, causal=True, **{n: g[1] for n, g in zip(("dQ", "dK", "dV"), grads)})
    for whole in (o_all, *(g[0] for g in grads)):
        assert (whole[:, :32] == 7).all() and (whole[:, 32 + T:] == 7).all()
    _check(host, dev, q_off, q_off, True)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_repeated_keys_and_fused_layout(dtype):
    """K and V of one head repeated by a stride of 0, and Q, K, V and their gradients inside [T, 3, H, 64] arrays."""
    T, H = 90, 4
    g = torch.Generator().manual_seed(5)
    fused = torch.randn(T, 3, H, 64, generator=g).to(dtype)
    G = torch.randn(H, T, 64, generator=g).to(dtype)
    d = fused.cuda()
    q, k, v = (d[:, i].transpose(0, 1) for i in range(3))
    out, lse = psa.dense_attn_packed_fwd(q, k, v, causal=True, lse=True)
    grad = torch.zeros_like(d)
    psa.dense_attn_packed_bwd(q, k, v, out, lse, G.cuda(), causal=True, **{n: grad[:, i].transpose(0, 1) for i, n in enumerate(("dQ", "dK", "dV"))})
    hq, hk, hv = (fused[:, i].transpose(0, 1) for i in range(3))
    want = packed_attention(hq, hk, hv, [0, T], [0, T], True, 0.125, G)
    for x, (w, e) in zip((out, lse, *(grad[:, i].transpose(0, 1) for i in range(3))), want):
        assert_within(x, w, e)
    one = [t[:1] for t in (k, v)]
    shared = psa.dense_attn_packed_fwd(q, *(t.expand(H, T, 64) for t in one), causal=True)
    want = packed_attention(hq, hk[:1], hv[:1], [0, T], [0, T], True, 0.125)
    assert_within(shared, *want[0])


def test_gradient_against_differences():
    """float32, h = 2^-5: the loss sums 1536 outputs, each off by less than 2^-20, with weights of mean size 0.8, over 2h = 2^-4:
    0.038 at the most for the two; what the third derivative adds is 5e-6 (the same differences of the float64 form)."""
    host, dev, q_off, k_off = _case(2, 1, [5, 7], [5, 9], torch.float32, wide=False)
    Qd, Kd, Vd, Gd = dev
    qo, ko = (torch.tensor(o, dtype=torch.int32, device="cuda") for o in (q_off, k_off))
    run = lambda **kw: psa.dense_attn_packed_fwd(Qd, Kd, Vd, qo, ko, causal=True, **kw)
    out, lse = run(lse=True)
    grads = psa.dense_attn_packed_bwd(Qd, Kd, Vd, out, lse, Gd, qo, ko, causal=True)
    h = 2.0 ** -5
    for tensor, grad in zip((Qd, Kd, Vd), grads):
        flat = tensor.view(-1)
        for i in range(3, flat.numel(), 101):
            old = flat[i].item()
            vals = []
            for x in (old + h, old - h):
                flat[i] = x
                vals.append((run().double() * Gd.double()).sum().item())
            flat[i] = old
            assert abs((vals[0] - vals[1]) / (2 * h) - grad.view(-1)[i].item()) < 0.04


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("q_lens,k_lens", [([150, 40], [150, 40]), ([1, 1], [900, 30])])
def test_graph_replays_with_new_lengths(q_lens, k_lens, dtype):
    """A captured forward and backward: offsets are read by the kernels, so a replay takes the lengths it finds."""
    host, dev, q_off, k_off = _case(4, 2, q_lens, k_lens, dtype)
    Qd, Kd, Vd, Gd = dev
    qo, ko = (torch.tensor(o, dtype=torch.int32, device="cuda") for o in (q_off, k_off))

    def step():
        out, lse = psa.dense_attn_packed_fwd(Qd, Kd, Vd, qo, ko, causal=True, lse=True)
        return (out, lse, *psa.dense_attn_packed_bwd(Qd, Kd, Vd, out, lse, Gd, qo, ko, causal=True))
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for move in (0, 1, 0, -1):
        qo[1] = q_off[1] + (move if q_lens[0] > 1 else 0)
        ko[1] = k_off[1] + move * 7
        graph.replay()
        ref = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, ref))


def test_run_of_a_layer():
    """Layer norm, the projections, rotary positions, attention over packed clips and the output matrix, one after the other on one
    frame-packed batch as a layer would have them; the last step's input against float64 from the tensors as they were rounded."""
    lens, H = [37, 1, 120, 64], 4
    T, dm = sum(lens), 64 * H
    g = torch.Generator().manual_seed(11)
    dt = torch.bfloat16
    X = torch.randn(T, dm, generator=g).to(dt)
    gamma, beta = (1 + 0.1 * torch.randn(dm, generator=g)).to(dt), (0.1 * torch.randn(dm, generator=g)).to(dt)
    W = [(torch.randn(dm, dm, generator=g) / math.sqrt(dm)).to(dt) for _ in range(4)]
    Wd = [w.cuda() for w in W]
    weights = psa.make_weights(*Wd)
    off = torch.tensor(_offsets(lens), dtype=torch.int32, device="cuda")
    pos = torch.cat([torch.arange(n) for n in lens]).to(torch.int32)
    spec = psa.make_rotary(64)
    Y = psa.probsparse_layer_norm_fwd(X.cuda(), gamma.cuda(), beta.cuda(), stats=False)
    Q, K, V = psa.probsparse_qkv_project(Y[None], weights)
    psa.probsparse_rotary_fwd(Q, K, spec, positions=pos.cuda(), Q_out=Q, K_out=K)
    A = torch.empty_like(Q)
    psa.dense_attn_packed_fwd(Q[0], K[0], V[0], off, causal=True, out=A[0])
    out = psa.probsparse_out_project(A, weights)
    # from the float64 layer on the same weights: every tensor in between is rounded to bfloat16 once (2^-8 of it), so compare
    # each step with float64 from its own rounded input
    want = packed_attention(Q[0].cpu(), K[0].cpu(), V[0].cpu(), _offsets(lens), _offsets(lens), True, 0.125)
    assert_within(A[0], *want[0], "attention")
    a = A[0].cpu().double().transpose(0, 1).reshape(T, dm)
    y, size = a @ W[3].double().T, a.abs() @ W[3].double().abs().T
    assert_within(out[0], y, HALF[dt] * y.abs() + dm * 2.0 ** -24 * size, "output matrix")
