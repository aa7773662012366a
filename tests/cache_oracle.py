"""A cache in pages on the CPU, in float64 and in plain lists: rows by position, attention over them with what a correct
implementation may be off by, the 8-bit form, and who holds which page."""
import math

import torch

from tests.operator_bounds import HALF, TINY, U

LOW, HIGH = -117, 119


# ------------------------------------------------------------------------------------------------------- 8-bit elements
def mx_encode(x):
    """Rows [.., 64] (float64) as the values of their codes before the power (float64; NaN for what is not finite) and the exponents of
    their powers [.., 2]: the least that brings the largest finite magnitude to 448, and the step between codes around a value."""
    y = x.double().unflatten(-1, (2, 32))
    size = torch.where(y.isfinite(), y.abs(), 0.0)
    most = size.amax(-1)
    e = torch.full(most.shape, LOW, dtype=torch.int64)
    some = most > 0
    e[some] = torch.ceil(torch.log2(most[some] / 448)).long()
    e = e.clamp(LOW, HIGH)
    z = torch.ldexp(y, -e.unsqueeze(-1)).clamp(-448, 448)
    step = torch.ldexp(torch.ones_like(z), torch.floor(torch.log2(z.abs().clamp(min=2.0 ** -6))).nan_to_num().int() - 3)
    return torch.where(y.isfinite(), torch.round(z / step) * step, math.nan).flatten(-2), e


def mx_decode(codes, bytes_):
    """The values of 8-bit rows, float64."""
    return (codes.double().unflatten(-1, (2, 32)) * torch.ldexp(torch.ones(bytes_.shape, dtype=torch.float64), bytes_.int() - 127).unsqueeze(-1)).flatten(-2)


# ------------------------------------------------------------------------------------------------------------ attention
def fine(T, H, H_kv, B, causal):
    """Whether bfloat16 weights are kept to 16 bits."""
    rows = T * (H // H_kv)
    return rows <= 32 * B or (rows // 16 + B) * H_kv <= 192 or (rows // 128 + B) * H_kv < (224 if causal else 152)


def attend(Q, K, V, seen, scale, dtype, round_p):
    """out, its bound, lse, its bound of rows Q [n, 64] that see the keys `seen` [n, n_k] of K and V [n_k, 64]: as for packed
    attention.  Keys that nobody sees may hold anything."""
    q, any_ = Q.double(), seen.any(0)
    k, v = torch.where(any_[:, None], K.double(), 0.0), torch.where(any_[:, None], V.double(), 0.0)
    n, n_k = seen.shape
    if n_k == 0:
        return torch.zeros(n, 64).double(), torch.full((n, 64), TINY).double(), torch.full((n,), -math.inf).double(), torch.ones(n).double()
    s = (scale * q @ k.T).masked_fill(~seen, -math.inf)
    lse = torch.logsumexp(s, 1)
    p = torch.where(seen, torch.exp(s - torch.where(torch.isfinite(lse), lse, 0.0)[:, None]), 0.0)
    # a score is a sum of 64 products and is scaled; its exponential rounds its argument and itself
    size = scale * q.abs() @ k.abs().T
    e_s = torch.where(seen, 70 * U * size + 4 * U * s.abs().masked_fill(~seen, 0.0) + 8 * U, 0.0)
    e_p = e_s + e_s.amax(1, keepdim=True)
    out, pv = p @ v, p @ v.abs()
    chain = (2 * n_k + 16) * U            # a sum over n_k keys, rescaled once for every tile of 32 at most, and where splits are joined
    e_out = (p * e_p + TINY * seen) @ v.abs() + TINY + (chain + round_p) * pv + HALF[dtype] * out.abs()
    e_lse = e_s.amax(1) + chain + 8 * U + 2 * U * torch.where(torch.isfinite(lse), lse, 0.0).abs()
    return out, e_out * 1.01, lse, e_lse * 1.01


def attention(Q, rows, table, lengths, new, page_rows, causal, scale, dtype, n_pages):
    """Of Q [H, T, 64] (new[s] rows of each sequence) over rows(page, slot) -> K, V [H_kv, n, 64] float64: out, lse and their bounds."""
    H, T, _ = Q.shape
    out, e_out = torch.zeros(H, T, 64).double(), torch.full((H, T, 64), TINY).double()
    lse, e_lse = torch.full((H, T), -math.inf).double(), torch.ones(H, T).double()
    at = 0
    for s, (n, a) in enumerate(zip(lengths, new)):
        n = min(max(n, 0), table.shape[1] * page_rows)
        j = torch.arange(n)
        page = table[s].long()[j // page_rows] if n else j
        held = (page >= 0) & (page < n_pages)
        j, page = j[held], page[held]
        K, V = rows(page, j % page_rows)
        H_kv = K.shape[0]
        round_p = 0.0 if dtype == torch.float32 else 2.0 ** -15 if fine(T, H, H_kv, len(lengths), causal) else HALF[dtype]
        seen = torch.ones(a, j.numel(), dtype=torch.bool)
        if causal:
            seen = j[None, :] <= torch.arange(a)[:, None] + (n - a)
        for h in range(H):
            g = h // (H // H_kv)
            out[h, at:at + a], e_out[h, at:at + a], lse[h, at:at + a], e_lse[h, at:at + a] = attend(Q[h, at:at + a], K[g], V[g], seen, scale, dtype, round_p)
        at += a
    return out, e_out, lse, e_lse


# ----------------------------------------------------------------------------------------------------------- the holders
def update(table, lengths, refs, page_rows, parents, grow):
    """The next step's sequences, on lists: (table, lengths, refs, pairs, missing)."""
    width = len(table[0])
    B, n_pages = len(table), len(refs)
    parents = list(range(B)) if parents is None else parents
    grow = [0] * len(parents) if grow is None else [max(g, 0) for g in grow]
    pages = lambda n: -(-n // page_rows)
    good = lambda x: x if 0 <= x < n_pages else -1
    refs = list(refs)
    held = [[good(x) for x in row[:pages(n)]] for row, n in zip(table, lengths)]
    for row in held:
        for x in row:
            if x >= 0:
                refs[x] -= 1
    rows = [list(held[p]) if 0 <= p < B else [] for p in parents]
    had = [lengths[p] if 0 <= p < B else 0 for p in parents]
    for row in rows:
        for x in row:
            if x >= 0:
                refs[x] += 1
    grown = [min(n + g, width * page_rows) for n, g in zip(had, grow)]
    writers = {}
    for i, row in enumerate(rows):
        if grown[i] > had[i] and had[i] % page_rows and row[-1] >= 0:
            writers.setdefault(row[-1], []).append(i)
    copies = [i for x, who in writers.items() for i in who if not (refs[x] == len(who) and who[0] == i)]
    free = [x for x in range(n_pages) if refs[x] == 0]
    pairs, missing = [], 0
    for i, row in enumerate(rows):
        if i in copies:
            old = row.pop()
            refs[old] -= 1
            if free:
                pairs.append((old, free[0]))
        while len(row) < pages(grown[i]):
            if free:
                refs[free[0]] = 1
            else:
                missing += 1
            row.append(free.pop(0) if free else -1)
        missing += pages(had[i] + grow[i]) - pages(grown[i])
        row += [-1] * (width - len(row))
    return rows, grown, refs, pairs, missing


def compact(table, refs):
    """(table, refs, pairs, pages in use), on lists."""
    used = sum(r != 0 for r in refs)
    moves = list(zip([x for x in range(used, len(refs)) if refs[x]], [x for x in range(used) if not refs[x]]))
    to = dict(moves)
    refs = list(refs)
    for old, new in moves:
        refs[new], refs[old] = refs[old], 0
    return [[to.get(x, x) for x in row] for row in table], refs, moves, used
