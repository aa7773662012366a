"""Attention of more than 256 sequences, whose parts are counted by a kernel of its own: several of them divided, in different groups
of 64, in each kernel; and rows of an append that are in no sequence."""
import pytest
import torch

from paper_2106_09236_amd import binding as psa
from tests import cache_oracle as O
from tests.operator_bounds import assert_within
from tests.test_cache_gpu import BF16, F32, FORMATS, Cache, _check, _offsets, _queries

pytestmark = pytest.mark.gpu


class OnHost(Cache):
    """A cache whose rows are brought to the host once, since every sequence asks for some."""

    def keep(self):
        (K, V), self._kept = super().rows(torch.arange(self.n_pages).repeat_interleave(self.P), torch.arange(self.P).repeat(self.n_pages)), None
        self._kept = [x.unflatten(1, (self.n_pages, self.P)) for x in (K, V)]

    def rows(self, page, slot):
        return [x[:, page, slot] for x in self._kept]


def _many(B, longest, long, width, dtype, mx, H_kv=1, page_rows=16):
    """Short sequences, some of them empty, and long ones at the places and of the lengths in `long`."""
    g = torch.Generator().manual_seed(B + longest)
    lengths = torch.randint(0, longest + 1, (B,), generator=g).tolist()
    for s, n in long.items():
        lengths[s] = n
    cache = OnHost(H_kv, page_rows, lengths, dtype, mx, width=width)
    cache.fill()
    cache.keep()
    return cache


@pytest.mark.parametrize("dtype,mx", FORMATS)
@pytest.mark.parametrize("B,long", [(300, {3: 5000, 70: 700, 133: 9000, 200: 2500, 299: 3000}), (700, {0: 6000, 64: 5000, 65: 3000, 400: 9000, 699: 4500}),
                                    (1300, {10: 9000, 650: 8000, 1100: 9000, 1298: 4000, 1299: 7000})])
def test_single_tokens_of_many_sequences(B, long, dtype, mx):
    cache = _many(B, 40, long, 600, dtype, mx)
    _check(cache, 2, [min(n, 1) for n in cache.lengths_host], True)
    _check(cache, 2, [1] * B, True, uniform=True)


@pytest.mark.parametrize("dtype,mx", FORMATS)
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("B,new,long", [(280, 21, {2: 3000, 66: 2200, 140: 700, 279: 4000}), (270, 45, {0: 2500, 100: 3000, 128: 1700, 269: 2200}),
                                        (1090, 18, {9: 3500, 500: 4000, 1030: 2500, 1089: 3600})])
def test_chunks_of_many_sequences(B, new, long, causal, dtype, mx):
    """Work-groups of 64 and 128 rows, sequences in several splits and undivided ones of several tiles."""
    cache = _many(B, 60, long, 300, dtype, mx)
    new = [new + (s % 3 - 1) * (new // 2) for s in range(B)]
    for s in long:
        new[s] += 100
    _check(cache, 2, new, causal)


@pytest.mark.parametrize("dtype,mx", FORMATS)
@pytest.mark.parametrize("new", [21, 45])
def test_undivided_chunks_of_many_sequences(new, dtype, mx):
    """Tables of few rows: nothing is divided, and tiles are taken by their index."""
    B = 900
    cache = _many(B, 50, {7: 800, 300: 500, 899: 900}, 60, dtype, mx)
    new = [new + (s % 3 - 1) * (new // 2) + (300 if s in (7, 300, 640, 899) else 0) for s in range(B)]
    _check(cache, 2, new, True)


@pytest.mark.parametrize("dtype,mx", FORMATS)
@pytest.mark.parametrize("front,lens,T", [(5, [2, 0, 1], 30), (3, [1], 5), (0, [4, 4], 9), (70, [9, 0, 40, 2], 200), (1, [1, 1, 1, 1, 1, 1], 8), (60, [0, 0], 64)])
def test_append_of_rows_in_no_sequence(front, lens, T, dtype, mx):
    """Rows before the first offset and behind the last are left out, also where one wave has both, and sequences between them."""
    H_kv, P = 3, 4
    cache = Cache(H_kv, P, [n + 3 for n in lens], dtype, mx)
    before = [x.contiguous().view(torch.uint8).cpu() for x in (cache.K, cache.V)]
    _, K = _queries(H_kv, T, dtype)
    _, V = _queries(H_kv, T, dtype, seed=9)
    cache.append(K, V, _offsets(lens, front=front))
    for x, was, source, scales in zip((cache.K, cache.V), before, (K.cpu(), V.cpu()), cache.scales):
        got = x.contiguous().view(torch.uint8).cpu()
        at = front
        for s, a in enumerate(lens):
            j = torch.arange(3, 3 + a)
            page, slot = cache.table_host[s].long()[j // P], j % P
            rows = source[:, at:at + a].transpose(0, 1)
            if mx:
                codes, e = O.mx_encode(rows)
                assert torch.equal(got[page, :, slot].view(torch.float8_e4m3fn).double(), codes)
                assert torch.equal(scales.contiguous().cpu()[page, :, slot].long(), e + 127)
            else:
                assert torch.equal(got[page, :, slot], rows.contiguous().view(torch.uint8))
            got[page, :, slot] = was[page, :, slot]
            at += a
        assert torch.equal(got, was)
