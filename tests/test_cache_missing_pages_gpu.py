"""Sequences that grow inside a page that they do not have: their rows are left out, and every call that grows them there says so."""
import math

import pytest
import torch

from paper_2106_09236_amd import binding as psa
from tests import cache_oracle as O
from tests.operator_bounds import assert_within
from tests.test_cache_gpu import BF16, F32, _ints

pytestmark = pytest.mark.gpu

# (up to 8192 pages a call is one launch, beyond them three)
SIZES = [12, 600, 9000]


def _inside(table, lengths, n_pages, page_rows, parents, grow):
    """How many of the new sequences get rows that lie on their last page, which the table does not name."""
    n = 0
    for i, p in enumerate(range(len(table)) if parents is None else parents):
        if not 0 <= p < len(table):
            continue
        rows = min(lengths[p], len(table[0]) * page_rows)
        grown = min(rows + max(grow[i], 0), len(table[0]) * page_rows)
        n += grown > rows and rows % page_rows != 0 and not 0 <= table[p][rows // page_rows] < n_pages
    return n


def _step(table, lengths, refs, page_rows, parents, grow):
    """The call and what lists say of it; its outputs on lists."""
    got = psa.probsparse_cache_update(_ints(table), _ints(lengths), _ints(refs), page_rows, None if parents is None else _ints(parents), _ints(grow))
    rows, grown, counts, pairs, missing = O.update(table, lengths, refs, page_rows, parents, grow)
    assert got[0].tolist() == rows and got[1].tolist() == grown and got[2].tolist() == counts
    assert got[3].tolist() == [list(p) for p in pairs] + [[-1, -1]] * (len(rows) - len(pairs))
    assert got[4].tolist() == [len(pairs), missing or _inside(table, lengths, len(refs), page_rows, parents, grow)]
    return rows, grown, counts, got[4].tolist()


@pytest.mark.parametrize("n_pages", SIZES)
def test_a_page_that_was_missing_is_said_again(n_pages):
    """Pages run out, some are freed, and the sequences go on growing inside the pages that they were refused, then beyond them."""
    table, lengths, refs = [[0, -1, -1], [1, -1, -1], [2, -1, -1]], [3, 4, 1], [1] * n_pages
    table, lengths, refs, said = _step(table, lengths, refs, 4, None, [4, 2, 1])
    assert said == [0, 2] and table == [[0, -1, -1], [1, -1, -1], [2, -1, -1]] and lengths == [7, 6, 2]
    refs[5] = refs[6] = refs[7] = 0                     # another table lets go
    table, lengths, refs, said = _step(table, lengths, refs, 4, None, [1, 1, 1])
    assert said == [0, 2] and table == [[0, -1, -1], [1, -1, -1], [2, -1, -1]]          # (rows 4 .. of these pages were never written: none is given)
    table, lengths, refs, said = _step(table, lengths, refs, 4, None, [0, 0, 1])
    assert said == [0, 0]                               # nobody grows there
    table, lengths, refs, said = _step(table, lengths, refs, 4, [1, 0, 1, -1], [2, 1, 0, 1])
    assert said == [0, 1] and table == [[1, -1, 2], [0, -1, 5], [1, -1, -1], [6, -1, -1]] and lengths == [9, 9, 7, 1]          # (nobody continues 2)
    table, lengths, refs, said = _step(table, lengths, refs, 4, None, [1, 1, 0, 1])
    assert said == [0, 0]                               # every new row has a page


@pytest.mark.parametrize("n_pages", SIZES)
def test_a_copy_that_was_given_up_is_said_again(n_pages):
    refs = [1] * n_pages
    refs[0] = 2
    table, lengths, refs, said = _step([[0, -1], [0, -1]], [2, 2], refs, 4, None, [1, 1])
    assert said == [0, 1] and table == [[0, -1], [-1, -1]] and refs[0] == 1
    refs[3] = 0
    table, lengths, refs, said = _step(table, lengths, refs, 4, None, [1, 1])
    assert said == [0, 1] and table == [[0, -1], [-1, -1]]
    table, lengths, refs, said = _step(table, lengths, refs, 4, [1], [1])
    assert said == [0, 0] and table == [[-1, 0]]        # (page 0 is free by then)


@pytest.mark.parametrize("n_pages", SIZES)
def test_entries_without_pages_anywhere(n_pages):
    """Tables with missing entries in front, in the middle and at the end, -1 or out of range, over several steps."""
    for seed in range(8):
        g = torch.Generator().manual_seed(seed)
        draw = lambda lo, hi, n: torch.randint(lo, hi, (n,), generator=g).tolist()
        B, width, P = 3 if n_pages < 100 else 40, 6, 4
        lengths, free = draw(0, width * P - 8, B), torch.randperm(n_pages, generator=g).tolist()
        refs, table = [int(x) for x in torch.rand(n_pages, generator=g) < 0.5], []
        for n in lengths:
            row = []
            for _ in range(-(-n // P)):
                row.append(free.pop() if free and float(torch.rand(1, generator=g)) < 0.7 else [-1, n_pages, 1 << 30][len(free) % 3])
            table.append(row + [-1] * (width - len(row)))
        for row in table:
            for x in row:
                if 0 <= x < n_pages:
                    refs[x] = 1
        for step in range(3):
            table, lengths, refs, _ = _step(table, lengths, refs, P, None if step == 1 else draw(-1, B, B), draw(0, 4, B))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_on_a_page_that_is_missing(dtype):
    """They are not written and not seen; rows behind the page's end are."""
    P, H_kv, n_pages, width = 4, 2, 6, 4
    g = torch.Generator().manual_seed(3)
    pool = torch.full((n_pages, 2, H_kv, P, 64), math.nan, dtype=dtype, device="cuda")
    K_pages, V_pages = pool[:, 0], pool[:, 1]
    table, lengths, refs = _ints([[-1] * width]), _ints([0]), _ints([0, 1, 1, 1, 1, 1])
    history = [torch.zeros(H_kv, 0, 64, dtype=dtype)] * 2
    lost = []
    for i, (new, missing) in enumerate([(3, 0), (3, 1), (1, 1), (3, 1), (2, 0)]):
        if i == 2:
            refs[4] = 0
        table, lengths, refs, _, counts = psa.probsparse_cache_update(table, lengths, refs, P, None, _ints([new]))
        assert counts.tolist() == [0, missing], i
        K, V = (torch.randn((H_kv, new, 64), generator=g).to(dtype) for _ in range(2))
        Q = torch.randn((2 * H_kv, new, 64), generator=g).to(dtype)
        psa.probsparse_cache_append(K.cuda(), V.cuda(), K_pages, V_pages, table, lengths)
        history = [torch.cat(x, 1) for x in zip(history, (K, V))]
        n = lengths.item()
        lost = [j for j in range(n) if table[0, j // P] < 0]
        seen = torch.arange(n)[None, :] <= torch.arange(new)[:, None] + (n - new)
        seen[:, lost] = False
        out = psa.dense_attn_paged_fwd(Q.cuda(), K_pages, V_pages, table, lengths, causal=True)
        for h in range(2 * H_kv):
            want, e, _, _ = O.attend(Q[h], history[0][h // 2], history[1][h // 2], seen, 0.125, dtype, 0.0 if dtype == F32 else 2.0 ** -15)
            assert_within(out[h], want, e, str(i))
    assert lost == [4, 5, 6, 7] and table.tolist() == [[0, -1, 4, -1]]
