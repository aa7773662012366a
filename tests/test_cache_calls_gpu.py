"""How the calls of a cache in pages may be made: captured and replayed while sequences grow, on another stream, through either
binding, with far offsets, odd strides and values out of range; and what is refused."""
import math

import pytest
import torch

from paper_2106_09236_amd import binding as psa
from tests import cache_oracle as O
from tests.operator_bounds import assert_within
from tests.test_cache_gpu import BF16, F32, FORMATS, Cache, _check, _holders, _ints, _offsets, _queries

pytestmark = pytest.mark.gpu


class Streams:
    """A cache, its tables, and one step of a program on it."""

    def __init__(self, dtype, mx, beams, H=4, H_kv=2, P=8, width=20, n_pages=300):
        self.H, self.P, self.beams = H, P, beams
        kind = torch.float8_e4m3fn if mx else dtype
        self.pool = torch.zeros((n_pages, 2, H_kv, P, 64), dtype=torch.float32, device="cuda").to(kind)
        self.scales = torch.full((n_pages, 2, H_kv, P, 2), 127, dtype=torch.uint8, device="cuda") if mx else None
        self.kw = dict(K_scales=self.scales[:, 0], V_scales=self.scales[:, 1]) if mx else {}
        self.table = torch.full((beams, width), -1, dtype=torch.int32, device="cuda")
        self.lengths = torch.zeros(beams, dtype=torch.int32, device="cuda")
        self.refs = torch.zeros(n_pages, dtype=torch.int32, device="cuda")
        self.parents = torch.arange(beams, dtype=torch.int32, device="cuda")
        self.grow = torch.ones(beams, dtype=torch.int32, device="cuda")
        self.Q = torch.zeros((H, beams, 64), dtype=dtype, device="cuda")
        self.K, self.V = (torch.zeros((H_kv, beams, 64), dtype=dtype, device="cuda") for _ in range(2))

    def step(self, causal=True):
        table, lengths, refs, pairs, counts = psa.probsparse_cache_update(self.table, self.lengths, self.refs, self.P, self.parents, self.grow)
        psa.probsparse_cache_copy([self.pool] if self.scales is None else [self.pool, self.scales], pairs, counts)
        psa.probsparse_cache_append(self.K, self.V, self.pool[:, 0], self.pool[:, 1], table, lengths, **self.kw)
        out, lse = psa.dense_attn_paged_fwd(self.Q, self.pool[:, 0], self.pool[:, 1], table, lengths, causal=causal, lse=True, **self.kw)
        for mine, new in ((self.table, table), (self.lengths, lengths), (self.refs, refs)):
            torch.add(new, 0, out=mine)
        return out, lse, counts

    def draw(self, g):
        for x in (self.Q, self.K, self.V):
            x.copy_(torch.randn(x.shape, generator=g))
        self.parents.copy_(torch.randint(0, self.beams, (self.beams,), generator=g))


@pytest.mark.parametrize("dtype,mx", FORMATS)
def test_graph_of_a_step(dtype, mx):
    """A step captured once serves while sequences fork and grow from nothing over many pages, with eager steps in between: every replay says
    what an eager program says."""
    a, b = Streams(dtype, mx, 5), Streams(dtype, mx, 5)
    psa.probsparse_init()
    a.step()                                            # (warm; then from the start again)
    for x in (a.lengths, a.refs):
        x.zero_()
    a.table.fill_(-1)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            captured = a.step()
    torch.cuda.synchronize()
    ga, gb = torch.Generator().manual_seed(3), torch.Generator().manual_seed(3)
    for i in range(60):
        a.draw(ga)
        b.draw(gb)
        if i % 10 == 9:
            got = a.step()
        else:
            graph.replay()
            got = captured
        want = b.step()
        torch.cuda.synchronize()
        for x, y in zip(got, want):
            assert torch.equal(x, y), i
        for name in ("table", "lengths", "refs"):
            assert torch.equal(getattr(a, name), getattr(b, name)), (i, name)
    assert a.lengths.tolist() == [60] * 5


def test_graph_of_long_sequences():
    """Sequences that grow from one split to many between replays, in one captured call; two graphs share a workspace."""
    cache = Cache(2, 64, [9000, 700, 64], BF16)
    cache.fill()
    ws = torch.empty(1 << 27, dtype=torch.uint8, device="cuda")
    Q, Qd = _queries(8, 3, BF16)
    Q2, Qd2 = _queries(8, 3 * 50, BF16)
    psa.probsparse_init()
    outs, graphs = [], []
    for q in (Qd, Qd2):
        cache.attend(q, causal=True, workspace=ws)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(cache.attend(q, causal=True, workspace=ws))
        graphs.append(graph)
    for lengths in ([9000, 700, 64], [50, 1, 64], [5000, 0, 3], [9000, 699, 60]):
        cache.lengths.copy_(torch.tensor(lengths, dtype=torch.int32))
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for q, qd, out in ((Q, Qd, outs[0]), (Q2, Qd2, outs[1])):
            new = [q.shape[1] // 3] * 3
            want, e, _, _ = O.attention(q, cache.rows, cache.table_host, lengths, new, 64, True, 0.125, BF16, cache.n_pages)
            assert_within(out, want, e, str(lengths))
            assert torch.equal(out, cache.attend(qd, causal=True))


def test_other_stream():
    cache = Cache(2, 16, [300, 50], F32)
    cache.fill()
    Q, Qd = _queries(4, 40, F32)
    want = cache.attend(Qd, causal=True)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        busy = torch.randn(2048, 2048, device="cuda")
        for _ in range(10):
            busy = busy @ busy * 1e-3
        late = Qd * 1.0
        out = cache.attend(late, causal=True)
        update = psa.probsparse_cache_update(cache.table, cache.lengths, torch.ones(cache.n_pages, dtype=torch.int32, device="cuda"), 16)
    stream.synchronize()
    assert torch.equal(out, want) and torch.equal(update[0], cache.table)


@pytest.mark.parametrize("dtype,mx", FORMATS)
def test_without_the_extension_module(dtype, mx, monkeypatch):
    """The ctypes path makes the same calls."""
    def program():
        s = Streams(dtype, mx, 4)
        g = torch.Generator().manual_seed(1)
        results = []
        for _ in range(12):
            s.draw(g)
            results += s.step(causal=False)
        table, refs, pairs, counts = psa.probsparse_cache_compact(s.table, s.refs)
        psa.probsparse_cache_copy([s.pool], pairs, counts)
        return [x.clone() for x in (*results, table, refs, pairs, counts, s.pool.view(torch.uint8))]
    native = program()
    monkeypatch.setattr(psa, "_native", psa._CtypesOnly)
    for x, y in zip(native, program()):
        assert torch.equal(x, y)


def test_the_extension_module_takes_the_calls(monkeypatch):
    """None of the ordinary calls falls back to ctypes."""
    s = Streams(BF16, True, 4)
    s.step()
    monkeypatch.setattr(psa, "_launch", None)
    s.step()
    psa.probsparse_cache_compact(s.table, s.refs)


def test_pools_beyond_4_gib():
    """Pages whose offsets pass 32 bits, in elements and bytes."""
    n_pages, P = 48000, 64
    pool = torch.empty((n_pages, 2, 8, P, 64), dtype=BF16, device="cuda")        # 6.3 GB
    cache = Cache(8, P, [200, 130], BF16)
    used = torch.tensor([n_pages - 1, 3, n_pages - 7, 40000, 33000, 20000, 47000], dtype=torch.int32)
    cache.n_pages = n_pages
    cache.K, cache.V = pool[:, 0], pool[:, 1]
    cache.table_host[0, :4], cache.table_host[1, :3] = used[:4], used[4:]
    cache.table = cache.table_host.cuda()
    K, V = cache.fill()
    at = [0, 200]
    Q, Qd = _queries(8, 2, BF16)
    Q2, Qd2 = _queries(8, 160, BF16)
    rows = lambda s, n: (lambda page, slot: (K[:, at[s]:at[s] + n].double(), V[:, at[s]:at[s] + n].double()))
    for q, qd, new in ((Q, Qd, 1), (Q2, Qd2, 80)):
        out = cache.attend(qd, causal=True)
        for s, n in enumerate((200, 130)):
            part = slice(s * new, (s + 1) * new)
            want, e, _, _ = O.attention(q[:, part], rows(s, n), cache.table_host[s:s + 1], [n], [new], P, True, 0.125, BF16, n_pages)
            # (weights are rounded by a rule on the whole call)
            assert_within(out[:, part], want, e + 2.0 ** -8 * (want.abs() + V.double().abs().amax()))
    pairs = _ints([[n_pages - 1, 1], [3, n_pages - 2]])
    psa.probsparse_cache_copy([pool], pairs)
    assert torch.equal(pool[1, 0, :, 5], pool[n_pages - 1, 0, :, 5]) and torch.equal(pool[n_pages - 2], pool[3])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_far_apart(dtype):
    """Rows 8 MB apart, heads and pages inside them."""
    wide, P, n_pages = 8 * 2 ** 20 // (4 if dtype == F32 else 2), 16, 6
    room = torch.empty((P, wide), dtype=dtype, device="cuda")
    view = room[:, -n_pages * 2 * 2 * 64:].unflatten(1, (n_pages, 2, 2, 64))      # [P, n_pages, K or V, H_kv, 64]
    cache = Cache(2, P, [40, 20], dtype, spare=1)
    assert cache.n_pages == n_pages
    cache.K, cache.V = view[:, :, 0].permute(1, 2, 0, 3), view[:, :, 1].permute(1, 2, 0, 3)
    cache.fill()
    _check(cache, 4, [1, 1], True, uniform=True)
    _check(cache, 4, [35, 20], True)


@pytest.mark.parametrize("dtype,mx", FORMATS)
def test_long_sequence(dtype, mx):
    """One new row over 150000 keys, and 33 of them."""
    cache = Cache(1, 64, [150000], dtype, mx)
    cache.fill()
    _check(cache, 4, [1], True)
    _check(cache, 1, [33], True)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", [1e-3, 30.0, 1e4])
def test_scores_of_other_sizes(size, dtype):
    """Scores near zero, and so far apart that one key has all the weight and the running maximum moves often."""
    cache = Cache(2, 16, [900, 300], dtype)
    cache.fill()
    for new in (1, 40):
        Q, Qd = _queries(4, 2 * new, dtype)
        out = cache.attend(Qd, causal=True, scale=0.125 * size)
        want, e, _, _ = O.attention(Q, cache.rows, cache.table_host, cache.lengths_host, [new, new], 16, True, 0.125 * size, dtype, cache.n_pages)
        # (two keys whose scores are closer than what scores may be off by share the weight in another way: bounded by the values)
        assert_within(out, want, torch.minimum(e, torch.full_like(e, 12.0)))


def test_lengths_out_of_range():
    """Clamped to the table's rows, and to 0."""
    cache = Cache(1, 16, [40, 48], F32, width=3)
    cache.fill()
    Q, Qd = _queries(2, 2, F32)
    full = Cache(1, 16, [40, 48], F32, width=3)
    want = cache.attend(Qd, causal=False)
    cache.lengths.copy_(torch.tensor([-5, 2 ** 31 - 1], dtype=torch.int32))
    out, lse = cache.attend(Qd, causal=False, lse=True)
    assert (out[:, 0] == 0).all() and (lse[:, 0] == -math.inf).all() and torch.equal(out[:, 1], want[:, 1])
    before = cache.K.clone()
    cache.append(torch.ones(1, 2, 64, device="cuda"), torch.ones(1, 2, 64, device="cuda"))
    page = cache.table_host[1, 2].item()
    assert (cache.K[page, 0, 15] == 1).all()
    cache.K[page, 0, 15] = before[page, 0, 15]
    assert torch.equal(cache.K.view(torch.int32), before.view(torch.int32))
    table, lengths, refs = [[0, 1], [2, -1]], [2 ** 31 - 1, -3], [1, 1, 0, 0]
    got = psa.probsparse_cache_update(_ints(table), _ints(lengths), _ints(refs), 4, _ints([0, 1]), _ints([2 ** 31 - 1, -2 ** 31]))
    assert got[0].tolist() == [[0, 1], [-1, -1]] and got[1].tolist() == [8, 0] and got[2].tolist() == [1, 1, 0, 0]
    assert got[4].tolist() == [0, (8 + 2 ** 31 - 1 + 3) // 4 - 2]


@pytest.mark.parametrize("n_pages", [100, 20000])
def test_update_into_given_outputs(n_pages):
    g = torch.Generator().manual_seed(4)
    table, lengths, refs = _holders(6, 8, 4, n_pages, g)
    parents, grow = [0, 0, 3, 9, 2], [3, 1, 0, 5, 2]
    args = (_ints(table), _ints(lengths), _ints(refs), 4, _ints(parents), _ints(grow))
    want = psa.probsparse_cache_update(*args)
    given = [torch.full_like(x, 77) for x in want]
    got = psa.probsparse_cache_update(*args, *given)
    assert all(a is b and torch.equal(a, c) for a, b, c in zip(got, given, want))
    assert args[0].tolist() == table and args[2].tolist() == refs              # inputs stay
    want = psa.probsparse_cache_compact(want[0], want[2])
    again = psa.probsparse_cache_compact(got[0], got[2], refs_out=torch.full_like(got[2], 5))
    assert all(torch.equal(a, b) for a, b in zip(again, want))


def test_refusals_of_tensors():
    """Both bindings say what is wrong before anything is enqueued."""
    cache = Cache(2, 16, [40, 20], BF16)
    Q, K = torch.zeros(4, 6, 64, dtype=BF16, device="cuda"), torch.zeros(2, 6, 64, dtype=BF16, device="cuda")
    off = _ints([0, 3, 6])
    scales = torch.zeros((*cache.K.shape[:3], 2), dtype=torch.uint8, device="cuda")

    def attend(Q=Q, K_pages=cache.K, V_pages=cache.V, table=cache.table, lengths=cache.lengths, off=off, **kw):
        psa.dense_attn_paged_fwd(Q, K_pages, V_pages, table, lengths, off, **kw)

    def append(K=K, V=K, K_pages=cache.K, V_pages=cache.V, table=cache.table, lengths=cache.lengths, off=off, **kw):
        psa.probsparse_cache_append(K, V, K_pages, V_pages, table, lengths, off, **kw)
    for call in (attend, append):
        call()
        for kw in (dict(table=cache.table.long()), dict(lengths=cache.lengths.float()), dict(off=off.long())):
            with pytest.raises(TypeError):
                call(**kw)
        for kw in (dict(table=cache.table[0]), dict(table=cache.table[:, ::2]), dict(lengths=cache.lengths[:1]), dict(off=off[:2]), dict(K_pages=cache.K[0]),
                   dict(K_scales=scales), dict(K_scales=scales, V_scales=scales), dict(V_pages=cache.V[:, :, :8]), dict(K_pages=cache.K.cpu()),
                   dict(off=None, table=cache.table[:1].expand(4, -1).contiguous(), lengths=_ints([1] * 4))):
            with pytest.raises(ValueError):
                call(**kw)
        with pytest.raises(psa.ProbSparseError):
            call(K_pages=cache.K[:, :, :12], V_pages=cache.V[:, :, :12])           # pages of 12 rows
    for kw in (dict(Q=Q[:3]), dict(Q=Q[..., :32]), dict(Q=Q[0]), dict(out=Q[:, :5])):
        with pytest.raises(ValueError):
            attend(**kw)
    with pytest.raises(TypeError):
        attend(Q=Q.half())
    with pytest.raises(TypeError):
        attend(Q=Q.float())                                                        # a cache of another type
    with pytest.raises(psa.ProbSparseError):
        attend(workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    with pytest.raises(psa.ProbSparseError):
        attend(scale=math.nan)
    with pytest.raises(ValueError):
        append(V=K[:, :5])
    with pytest.raises(ValueError):
        append(K=torch.zeros(3, 6, 64, dtype=BF16, device="cuda"), V=torch.zeros(3, 6, 64, dtype=BF16, device="cuda"))
    n = torch.zeros(cache.n_pages, dtype=torch.int32, device="cuda")
    with pytest.raises(psa.ProbSparseError):
        psa.probsparse_cache_update(cache.table, cache.lengths, n, 12)
    with pytest.raises(psa.ProbSparseError):
        psa.probsparse_cache_update(cache.table, cache.lengths, n, 16, refs_out=n)
    with pytest.raises(ValueError):
        psa.probsparse_cache_update(cache.table, cache.lengths, n, 16, grow=_ints([1]))
    with pytest.raises(TypeError):
        psa.probsparse_cache_update(cache.table, cache.lengths, n.long(), 16)
    with pytest.raises(psa.ProbSparseError):
        psa.probsparse_cache_compact(cache.table, n, refs_out=n)
    with pytest.raises(ValueError):
        psa.probsparse_cache_compact(cache.table, n, pairs=_ints([[0, 0]]))
    pool = torch.zeros(5, 4, 8, device="cuda")
    for pools, pairs in (([], _ints([[0, 1]])), ([pool.transpose(1, 2)], _ints([[0, 1]])), ([pool, pool[:4]], _ints([[0, 1]])), ([pool], _ints([0, 1]))):
        with pytest.raises(ValueError):
            psa.probsparse_cache_copy(pools, pairs)
