"""Packed attention at the ends of the number range: the largest float32 numbers, and infinities of V wherever they stand."""
import pytest
import torch

from paper_2106_09236_amd import binding as psa
from tests.operator_bounds import assert_within, packed_attention

pytestmark = pytest.mark.gpu

# Beyond (2 - 2^-8) 2^127 a float32 number rounds to an infinity in bfloat16.  3.4e38 is one of them; times a weight of 1 that is off by some
# half steps it still is a float32 number (the largest is 3.4028e38).
HUGE = 3.4e38
MAX = torch.finfo(torch.float32).max


def _offsets(lens, front=0):
    off = [front]
    for n in lens:
        off.append(off[-1] + n)
    return off


def _tensors(H, H_kv, q_rows, k_rows, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(h, n, 64, generator=g).to(dtype) for h, n in ((H, q_rows), (H_kv, k_rows), (H_kv, k_rows), (H, q_rows))]


def _device_offsets(*offs):
    return [torch.tensor(o, dtype=torch.int32, device="cuda") for o in offs]


# Few rows with long sequences, many rows, and few work-groups with long sequences: each takes a kernel of its own.
SHAPES = [(4, 2, [90, 40], [90, 40]), (4, 2, [4, 2], [300, 90]), (64, 32, [200, 290], [200, 290]), (32, 32, [500, 401, 390], [500, 401, 390])]


@pytest.mark.parametrize("H,H_kv,q_lens,k_lens", SHAPES)
def test_largest_numbers_that_are_not_seen(H, H_kv, q_lens, k_lens):
    front, behind = 20, 30
    q_off, k_off = _offsets(q_lens, front), _offsets(k_lens, front)
    Q, K, V, _ = (t.cuda() for t in _tensors(H, H_kv, q_off[-1] + behind, k_off[-1] + behind, torch.float32, 3))
    qo, ko = _device_offsets(q_off, k_off)
    clean, clean_lse = psa.dense_attn_packed_fwd(Q, K, V, qo, ko, causal=True, lse=True)
    bad = k_off[1] - 1                       # the last key of the first sequence: its last query alone sees it
    rows = [i for i in range(Q.shape[1]) if i != q_off[1] - 1]
    for value in (MAX, -MAX, HUGE):
        K2, V2 = K.clone(), V.clone()
        for t in (K2, V2):
            t[:, :k_off[0]] = value
            t[:, k_off[-1]:] = value
            t[:, bad] = value
        out, lse = psa.dense_attn_packed_fwd(Q, K2, V2, qo, ko, causal=True, lse=True)
        assert torch.equal(out[:, rows], clean[:, rows]) and torch.equal(lse[:, rows], clean_lse[:, rows])


@pytest.mark.parametrize("H,H_kv,q_lens,k_lens", SHAPES)
@pytest.mark.parametrize("which", ["Q", "K", "V", "dOut"])
def test_largest_numbers_that_are_seen(H, H_kv, q_lens, k_lens, which):
    """One element of a row of one head at 3.4e38, against a column of powers of two so small that the product with it is
    ordinary.  (Not compared: the gradient in that column, which is of numbers near the smallest.)"""
    q_off, k_off = _offsets(q_lens), _offsets(k_lens)
    tensors = dict(zip(("Q", "K", "V", "dOut"), _tensors(H, H_kv, q_off[-1], k_off[-1], torch.float32, 4)))
    other, small = {"Q": ("K", 2.0 ** -126), "K": ("Q", 2.0 ** -126), "V": ("dOut", 2.0 ** -60), "dOut": ("V", 2.0 ** -60)}[which]
    e = 7
    tensors[other][..., e] = torch.where(tensors[other][..., e] < 0, -small, small)
    tensors[which][0, 1, e] = HUGE
    if which in "QK":
        tensors["dOut"] *= 2.0 ** -20
    host = [tensors[n] for n in ("Q", "K", "V", "dOut")]
    dev = [t.cuda() for t in host]
    qo, ko = _device_offsets(q_off, k_off)
    out, lse = psa.dense_attn_packed_fwd(*dev[:3], qo, ko, causal=True, lse=True)
    grads = psa.dense_attn_packed_bwd(*dev[:3], out, lse, dev[3], qo, ko, causal=True)
    want = packed_attention(*host[:3], q_off, k_off, True, 0.125, host[3])
    keep = [i for i in range(64) if i != e]
    for got, (w, bound), what in zip((out, lse, *grads), want, ("out", "lse", "dQ", "dK", "dV")):
        got = got.cpu()
        empty = w.isinf()
        assert torch.equal(got.isinf(), empty), what
        if which in "QK" and what == "d" + which:
            got, w, bound = (t[..., keep] for t in (got, w, bound))
        elif empty.any():
            got, w, bound = got.masked_fill(empty, 0.0), w.masked_fill(empty, 0.0), bound.masked_fill(empty, 1.0)
        assert_within(got, w, bound, what)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("H,H_kv,q_lens,k_lens", [(4, 2, [3, 2], [300, 200]), (4, 2, [1], [3000]), (4, 2, [20, 6], [40, 6]),
                                                  (32, 32, [500, 401, 390], [500, 401, 390])])
def test_infinite_value_wherever_it_stands(H, H_kv, q_lens, k_lens, causal, dtype):
    """An infinity in one element of the first key, which every query of its sequence sees, is that element of their outputs; the other
    elements and the other sequences stay as they are."""
    q_off, k_off = _offsets(q_lens), _offsets(k_lens)
    Q, K, V, _ = (t.cuda() for t in _tensors(H, H_kv, q_off[-1], k_off[-1], dtype, 5))
    qo, ko = _device_offsets(q_off, k_off)
    clean = psa.dense_attn_packed_fwd(Q, K, V, qo, ko, causal=causal)
    for value in (float("inf"), -float("inf"), float("nan")):
        V2 = V.clone()
        V2[:, 0, 5] = value
        out = psa.dense_attn_packed_fwd(Q, K, V2, qo, ko, causal=causal)
        hit = out[:, :q_off[1], 5].float()
        assert (hit.isnan() if value != value else hit == value).all()
        out[:, :q_off[1], 5] = clean[:, :q_off[1], 5]
        assert torch.equal(out, clean)
