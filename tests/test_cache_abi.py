"""Refusals of the cache in pages: argument checks run before anything touches the GPU."""
import ctypes
import math

import pytest
import torch

from paper_2106_09236_amd import binding as psa

NULL, SHAPE, DTYPE, ARG, WORKSPACE, ALIGN = -1, -2, -3, -4, -5, -7
BF16, F32 = psa.PSA_BF16, psa.PSA_F32


def _ref(x):
    return None if x is None else ctypes.byref(x)


def _heads(data=0x1000, page=64 * 2 * 16, head=64 * 16, row=64):
    return psa.PsaHeads(data, page, head, row)


def _scales(data=0x1000, page=2 * 2 * 16, head=2 * 16, row=2):
    return psa.PsaHeads(data, page, head, row)


def _cache(mx=False, n_pages=9, page_rows=16, max_pages=4, table=0x100, lengths=0x200, format=None, **t):
    none = psa.PsaHeads(None, 0, 0, 0)
    parts = [t.get("K", _heads()), t.get("V", _heads()), t.get("K_scales", _scales() if mx else none), t.get("V_scales", _scales() if mx else none)]
    return psa.PsaCache(*parts, table, lengths, n_pages, page_rows, max_pages, int(mx) if format is None else format)


def _shape(B=2, H=4, H_kv=2, T=10, D=64, dtype=F32, causal=1, scale=0.125):
    return psa.PsaPagedShape(B, H, H_kv, T, D, dtype, causal, scale)


def _append(K=_heads(), V=_heads(), offsets=0x300, cache=_cache(), shape=_shape()):
    return psa.load().probsparse_cache_append(_ref(K), _ref(V), offsets, _ref(cache), _ref(shape), None)


def _attend(Q=_heads(), offsets=0x300, cache=_cache(), out=_heads(), lse=0x400, shape=_shape(), ws=0x10000, n=1 << 40):
    return psa.load().dense_attn_paged_fwd(_ref(Q), offsets, _ref(cache), _ref(out), lse, _ref(shape), ws, n, None)


@pytest.mark.parametrize("call", [_append, _attend])
def test_cache_refusals(call):
    bad = _heads(data=None)
    assert call(cache=None) == call(shape=None) == call(cache=_cache(K=bad)) == call(cache=_cache(V=bad)) == NULL
    assert call(cache=_cache(table=None)) == call(cache=_cache(lengths=None)) == NULL
    assert call(cache=_cache(mx=True, K_scales=bad)) == call(cache=_cache(mx=True, V_scales=bad)) == NULL
    for kw in (dict(n_pages=0), dict(n_pages=(1 << 28) + 1), dict(page_rows=0), dict(page_rows=24), dict(page_rows=1 << 17), dict(max_pages=0), dict(max_pages=1 << 25)):
        assert call(cache=_cache(**kw)) == SHAPE, kw
    for kw in (dict(B=0), dict(B=(1 << 20) + 1), dict(H_kv=0), dict(T=0), dict(T=(1 << 28) + 1), dict(D=32)):
        assert call(shape=_shape(**kw)) == SHAPE, kw
    assert call(shape=_shape(B=3), offsets=None) == SHAPE                    # 10 rows are not the same number each
    assert call(shape=_shape(B=1 << 20), cache=_cache(max_pages=1 << 11)) == SHAPE
    assert call(shape=_shape(dtype=2)) == DTYPE
    assert call(cache=_cache(format=2)) == call(cache=_cache(format=-1)) == ARG
    assert call(cache=_cache(K=_heads(row=-64))) == call(cache=_cache(V=_heads(row=1 << 23))) == ARG
    assert call(cache=_cache(K=_heads(data=0x1008))) == call(cache=_cache(V=_heads(head=1026))) == call(cache=_cache(K=_heads(page=2050))) == ALIGN
    assert call(cache=_cache(mx=True, K=_heads(row=72))) == ALIGN             # 16 bytes are 16 elements there
    assert call(cache=_cache(mx=True, K_scales=_scales(data=0x1001))) == call(cache=_cache(mx=True, V_scales=_scales(row=3))) == ALIGN
    assert call(cache=_cache(table=0x102)) == call(cache=_cache(lengths=0x201)) == call(offsets=0x302) == ALIGN


def test_append_refusals():
    assert _append(shape=_shape(T=1 << 28)) == _append(shape=_shape(T=1 << 25, H_kv=64, dtype=BF16)) == SHAPE        # too many work-groups
    assert _append(K=None) == _append(V=None) == _append(K=_heads(data=None)) == NULL
    assert _append(K=_heads(data=0x1004)) == _append(V=_heads(head=1026)) == ALIGN
    # rows of the cache must not overlap: they are written
    assert _append(cache=_cache(K=_heads(row=0))) == _append(cache=_cache(V=_heads(head=32))) == _append(cache=_cache(K=_heads(page=0))) == ARG
    assert _append(cache=_cache(mx=True, K_scales=_scales(row=0))) == ARG


def test_attention_refusals():
    assert _attend(Q=None) == _attend(out=None) == _attend(ws=None) == _attend(out=_heads(data=None)) == NULL
    for kw in (dict(H=0), dict(H=3), dict(H=70000, H_kv=1), dict(H=64, H_kv=1, T=1 << 26)):
        assert _attend(shape=_shape(**kw)) == SHAPE, kw
    assert _attend(shape=_shape(H=65535, H_kv=65535, B=1 << 12, T=1 << 12)) == SHAPE          # too many work-groups
    for kw in (dict(causal=2), dict(scale=0.0), dict(scale=math.nan), dict(scale=1e31), dict(scale=-1.0)):
        assert _attend(shape=_shape(**kw)) == ARG, kw
    assert _attend(out=_heads(row=0)) == _attend(out=_heads(head=0)) == ARG
    assert _attend(Q=_heads(data=0x1008)) == _attend(lse=0x402) == _attend(ws=0x10080) == ALIGN
    assert _attend(n=128) == WORKSPACE
    size = psa.load().dense_attn_paged_workspace_bytes
    c = _cache()
    assert 0 < size(_ref(c), _ref(_shape())) < 1 << 28
    assert size(_ref(c), _ref(_shape(H=3))) == size(_ref(_cache(page_rows=3)), _ref(_shape())) == size(None, _ref(_shape())) == size(_ref(c), None) == 0


def test_workspace_does_not_grow_with_the_cache():
    """What long sequences need does not depend on how long they may be."""
    size = psa.load().dense_attn_paged_workspace_bytes
    shape = _shape(B=64, H=8, H_kv=8, T=64, dtype=BF16)
    sizes = {size(_ref(_cache(n_pages=1 << 16, page_rows=64, max_pages=m)), _ref(shape)) for m in (65, 512, 4096, 1 << 16)}
    assert len(sizes) == 1 and sizes.pop() < 1 << 28


def test_update_refusals():
    lib = psa.load()

    def call(table=0x100, lengths=0x200, refs=0x300, B=4, parents=0x400, grow=0x500, B_out=6, n_pages=10, page_rows=8, max_pages=3, table_out=0x600,
             lengths_out=0x700, refs_out=0x800, pairs=0x900, counts=0xA00, ws=0x10000, n=1 << 30):
        return lib.probsparse_cache_update(table, lengths, refs, B, parents, grow, B_out, n_pages, page_rows, max_pages, table_out, lengths_out, refs_out, pairs, counts, ws, n, None)
    for name in ("table", "lengths", "refs", "table_out", "lengths_out", "refs_out", "pairs", "counts", "ws"):
        assert call(**{name: None}) == NULL, name
    for kw in (dict(B=0), dict(B_out=0), dict(B=(1 << 20) + 1), dict(n_pages=0), dict(page_rows=12), dict(page_rows=0), dict(max_pages=0), dict(max_pages=1 << 27),
               dict(parents=None), dict(B_out=1 << 20, max_pages=1 << 11)):
        assert call(**kw) == SHAPE, kw
    for name in ("table", "lengths", "refs", "parents", "grow", "table_out", "lengths_out", "refs_out", "pairs", "counts"):
        assert call(**{name: 0x1002}) == ALIGN, name
    assert call(ws=0x10010) == ALIGN
    assert call(table_out=0x100) == call(lengths_out=0x200) == call(refs_out=0x300) == ARG
    size = lib.probsparse_cache_update_workspace_bytes
    assert call(n=size(4, 6, 10) - 1) == WORKSPACE
    assert size(4, 6, 10) % 256 == 0 and size(0, 6, 10) == size(4, 0, 10) == size(4, 6, 0) == size(4, 6, (1 << 28) + 1) == 0


def test_compact_refusals():
    lib = psa.load()

    def call(table=0x100, refs=0x200, B=4, n_pages=10, max_pages=3, table_out=0x300, refs_out=0x400, pairs=0x500, counts=0x600, ws=0x10000, n=1 << 30):
        return lib.probsparse_cache_compact(table, refs, B, n_pages, max_pages, table_out, refs_out, pairs, counts, ws, n, None)
    for name in ("table", "refs", "table_out", "refs_out", "pairs", "counts", "ws"):
        assert call(**{name: None}) == NULL, name
    for kw in (dict(B=0), dict(n_pages=0), dict(max_pages=0), dict(B=1 << 20, max_pages=1 << 11)):
        assert call(**kw) == SHAPE, kw
    for name in ("table", "refs", "table_out", "refs_out", "pairs", "counts"):
        assert call(**{name: 0x1002}) == ALIGN, name
    assert call(refs_out=0x200) == ARG
    assert call(n=16) == WORKSPACE and call(ws=0x10010) == ALIGN
    assert lib.probsparse_cache_compact_workspace_bytes(0) == 0


def test_copy_refusals():
    lib = psa.load()

    def call(pools=((0x1000, 256, 256),), n_pages=4, pairs=0x100, counts=0x200, n_pairs=2, n=None):
        array = (psa.PsaPool * max(1, len(pools)))(*[psa.PsaPool(*p) for p in pools])
        return lib.probsparse_cache_copy(array, len(pools) if n is None else n, n_pages, pairs, counts, n_pairs, None)
    assert call(pools=((None, 256, 256),)) == call(pairs=None) == lib.probsparse_cache_copy(None, 1, 4, 0x100, None, 2, None) == NULL
    assert call(n=0) == call(n_pages=0) == call(n_pairs=-1) == call(pools=((0x1000, 256, 0),)) == call(pools=((0x1000, 1 << 62, 256),)) == SHAPE
    assert call(pools=((0x1000, 128, 256),)) == ARG                          # pages that overlap
    assert call(pairs=0x102) == call(counts=0x201) == ALIGN
    assert call(n_pairs=0) == 0 and call(pairs=None, n_pairs=0) == 0          # nothing to do


def test_binding_checks_tensors():
    """Tensors that are not on a GPU never reach the library."""
    x = torch.zeros(2, 4, 64)
    pages = torch.zeros(3, 2, 16, 64)
    table, n = torch.zeros(4, 2, dtype=torch.int32), torch.zeros(4, dtype=torch.int32)
    for call in (lambda: psa.probsparse_cache_append(x, x, pages, pages, table, n), lambda: psa.dense_attn_paged_fwd(x, pages, pages, table, n),
                 lambda: psa.probsparse_cache_update(table, n, n, 16), lambda: psa.probsparse_cache_compact(table, n),
                 lambda: psa.probsparse_cache_copy([pages], torch.zeros(1, 2, dtype=torch.int32))):
        with pytest.raises(ValueError):
            call()
