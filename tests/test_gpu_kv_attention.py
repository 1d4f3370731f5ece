"""Attention over the paged key-value cache, whole prompts and single tokens, against a plain implementation in
64 bits, with bounds that follow from the roundings (tests/kv_util.py)."""
import pytest
import torch

from tests.kv_util import BF16, E4M3, FP16, Made, check

pytestmark = pytest.mark.gpu

HEADS = [(4, 4, 64), (8, 2, 128), (7, 1, 128), (6, 2, 64), (16, 1, 64), (24, 1, 128), (40, 2, 64)]


@pytest.mark.parametrize("dtype,store", [(BF16, BF16), (FP16, FP16), (BF16, E4M3), (FP16, E4M3)])
@pytest.mark.parametrize("heads,kv_heads,dim", HEADS)
def test_decode(dtype, store, heads, kv_heads, dim):
    kv = [0, 1, 15, 16, 17, 63, 64, 65, 0, 127, 128, 129, 200, 511, 700, 1, 33]
    for page in (16, 64, 512):
        m = Made(11 + page, [1] * len(kv), kv, heads=heads, kv_heads=kv_heads, dim=dim, dtype=dtype, store=store, page=page)
        lse = torch.empty((len(kv), heads), device="cuda")
        out = m.cache.decode(m.batch, m.q, lse=lse)
        m.batch.check()
        check(out, lse, m.expected(m.q, dim ** -0.5, True), dtype)


@pytest.mark.parametrize("dtype,store", [(BF16, BF16), (FP16, FP16), (BF16, E4M3), (FP16, E4M3)])
@pytest.mark.parametrize("heads,kv_heads,dim", HEADS)
def test_prefill(dtype, store, heads, kv_heads, dim):
    new = [1, 0, 5, 130, 1, 64, 33, 257, 2, 7]
    kv = [1, 9, 5, 130, 300, 65, 161, 257, 128, 3]           # the last has more new tokens than tokens: rows that see nothing
    for page in (16, 128, 1024):
        m = Made(23 + page, new, kv, heads=heads, kv_heads=kv_heads, dim=dim, dtype=dtype, store=store, page=page)
        lse = torch.empty((sum(new), heads), device="cuda")
        out = m.cache.prefill(m.batch, m.q, lse=lse)
        m.batch.check()
        check(out, lse, m.expected(m.q, dim ** -0.5, False), dtype)


@pytest.mark.parametrize("dtype", [BF16, FP16])
def test_long_sequences_and_sharp_scores(dtype):
    """Scores far apart (one key dominates, then another): the running maximum moves by much."""
    m = Made(31, [1, 1, 3], [5000, 9001, 2049], heads=8, kv_heads=2, dim=128, dtype=dtype, page=256, q_scale=8.0)
    out = m.cache.decode(m.batch, m.q[:3])
    check(out, None, m.expected(m.q[:3], 128 ** -0.5, True), dtype)
    out = m.cache.prefill(m.batch, m.q)
    check(out, None, m.expected(m.q, 128 ** -0.5, False), dtype)


@pytest.mark.parametrize("scale", [0.0, -0.2, 3e-6])
def test_other_scales(scale):
    m = Made(37, [3, 40], [70, 40], heads=4, kv_heads=2, dim=64, page=32)
    check(m.cache.prefill(m.batch, m.q, scale), None, m.expected(m.q, scale, False), BF16)
    check(m.cache.decode(m.batch, m.q[:2], scale), None, m.expected(m.q[:2], scale, True), BF16)


@pytest.mark.parametrize("decode", [False, True])
def test_rows_with_strides_and_rows_behind_the_last(decode):
    m = Made(41, [3, 9, 1], [90, 9, 33], heads=6, kv_heads=3, dim=64, page=16)
    n = 3 if decode else 13
    wide = torch.full((n + 5, 6 + 4, 64), float("nan"), dtype=BF16, device="cuda")
    wide[:n, :6] = m.q[:n]
    out = torch.full((n + 5, 8, 64), 7.0, dtype=BF16, device="cuda")
    lse = torch.full((n + 5, 6), 7.0, device="cuda")
    (m.cache.decode if decode else m.cache.prefill)(m.batch, wide[:, :6], out=out[:, 1:7], lse=lse)
    check(out[:n, 1:7], lse[:n], m.expected(m.q, 64 ** -0.5, decode), BF16)
    assert bool((out[:, 0] == 7).all()) and bool((out[:, 7] == 7).all()) and bool((out[n:] == 7).all()) and bool((lse[n:] == 7).all())


def test_a_value_that_is_not_finite_stays_where_it_is_seen():
    """A NaN or infinity among the values reaches the rows that see its key and no others, in its own column."""
    for bad in (float("nan"), float("inf")):
        for at in (0, 40, 69, 128, 199):
            m = Made(43, [200, 30], [200, 64], heads=4, kv_heads=2, dim=64, page=64)
            pg, slot = m.where(0, torch.tensor([at], device="cuda"))
            want = m.expected(m.q, 0.125, False)
            m.cache.v[pg, 1, slot, 5] = bad
            out = m.cache.prefill(m.batch, m.q)
            hit = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
            hit[at:200, 2:4, 5] = True
            assert not bool(torch.isfinite(out[hit]).any())
            out[hit] = want[0][hit].to(BF16)
            check(out, None, want, BF16)


def test_a_key_that_is_not_finite_stays_where_it_is_seen():
    m = Made(47, [200, 30], [200, 64], heads=4, kv_heads=2, dim=64, page=64)
    pg, slot = m.where(0, torch.tensor([100], device="cuda"))
    want = m.expected(m.q, 0.125, False)
    m.cache.k[pg, 0, slot, 3] = float("nan")
    out = m.cache.prefill(m.batch, m.q)
    hit = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
    hit[100:200, :2] = True
    assert bool(torch.isnan(out[hit]).all())
    out[hit] = want[0][hit].to(BF16)
    check(out, None, want, BF16)


@pytest.mark.parametrize("decode", [False, True])
def test_wrong_pages_and_lengths_are_reported(decode):
    from paper_2602_11688_b200 import binding as gb
    for fault, bit in (("page", gb.GORGO_KV_BAD_PAGE), ("kv", gb.GORGO_KV_BAD_LENGTH), ("low", gb.GORGO_KV_BAD_LENGTH)):
        m = Made(53, [3, 4, 2], [30, 70, 40], page=16)
        want = m.expected(m.q, 0.125, decode)
        if fault == "page":
            m.batch.table[1, 2] = m.cache.n_pages
        else:
            m.batch.kv_len[1] = 71 if fault == "kv" else -1
        out = (m.cache.decode if decode else m.cache.prefill)(m.batch, m.q)
        with pytest.raises(gb.GorgoError):
            m.batch.check()
        assert int(m.batch.status.item()) == bit
        lo, hi = (1, 2) if decode else (3, 7)
        assert bool(torch.isnan(out[lo:hi]).all())
        n = out.shape[0] if not decode else 3
        keep = [i for i in range(n) if not lo <= i < hi]
        check(out[keep], None, [w[keep] for w in want], BF16)


@pytest.mark.parametrize("decode", [False, True])
def test_a_row_that_is_in_no_place_is_reported_and_left(decode):
    from paper_2602_11688_b200 import binding as gb
    m = Made(71, [3, 4, 2], [30, 70, 40], page=16)
    m.batch.cu_new[1:3] = torch.tensor([5, 4], dtype=torch.int32, device="cuda")      # decreasing: the second has no rows
    if decode:                                               # which does not use them
        check(m.cache.decode(m.batch, m.q[:3]), None, m.expected(m.q[:3], 0.125, True), BF16)
        m.batch.check()
        return
    m.cache.prefill(m.batch, m.q)
    assert int(m.batch.status.item()) == gb.GORGO_KV_BAD_LENGTH


@pytest.mark.parametrize("heads,kv_heads,dim", [(128, 1, 64), (130, 2, 128), (99, 3, 64)])
@pytest.mark.parametrize("store", [BF16, E4M3])
def test_large_groups(heads, kv_heads, dim, store):
    m = Made(73, [1, 5, 2], [140, 5, 300], heads=heads, kv_heads=kv_heads, dim=dim, store=store, page=32)
    lse = torch.empty((8, heads), device="cuda")
    check(m.cache.prefill(m.batch, m.q, lse=lse), lse, m.expected(m.q, dim ** -0.5, False), BF16)
    lse = torch.empty((3, heads), device="cuda")
    check(m.cache.decode(m.batch, m.q[:3], lse=lse), lse, m.expected(m.q[:3], dim ** -0.5, True), BF16)


@pytest.mark.parametrize("dtype,store", [(BF16, BF16), (FP16, FP16), (BF16, E4M3), (FP16, E4M3)])
def test_decode_with_what_is_not_finite(dtype, store):
    """In a value: that element of the heads that read it; in a key or a query: those rows.  Nothing else."""
    for what in ("value", "key", "query"):
        m = Made(79, [1, 1, 1], [200, 700, 64], heads=6, kv_heads=2, dim=64, dtype=dtype, store=store, page=64)
        want = m.expected(m.q, 0.125, True)
        hit = torch.zeros((3, 6, 64), dtype=torch.bool, device="cuda")
        pg, slot = m.where(1, torch.tensor([333], device="cuda"))
        if what == "query":
            m.q[1, 4, 7] = float("inf")
            hit[1, 4] = True
        else:
            pool = m.cache.v if what == "value" else m.cache.k
            if store == E4M3:
                pool.view(torch.uint8)[pg, 0, slot, 11] = 0x7f
            else:
                pool[pg, 0, slot, 11] = float("nan")
            hit[1, :3, slice(11, 12) if what == "value" else slice(None)] = True
        out = m.cache.decode(m.batch, m.q)
        assert not bool(torch.isfinite(out[hit]).any())
        out[hit] = want[0][hit].to(dtype)
        check(out, None, want, dtype)


@pytest.mark.parametrize("store", [BF16, E4M3])
def test_many_short_sequences(store):
    """More sequences than a warp looks at at once, some without new tokens, some without any."""
    import numpy as np
    rng = np.random.default_rng(97)
    new = [int(x) for x in rng.integers(0, 4, 333)]
    kv = [n + int(x) if x else n for n, x in zip(new, rng.integers(0, 40, 333))]
    kv[7] = new[7] = kv[200] = new[200] = 0
    m = Made(97, new, kv, heads=4, kv_heads=2, dim=64, page=16, store=store)
    check(m.cache.prefill(m.batch, m.q), None, m.expected(m.q, 0.125, False), BF16)
    q = m.q[:333]
    check(m.cache.decode(m.batch, q), None, m.expected(q, 0.125, True), BF16)
    m.batch.check()


def test_lengths_that_cut_the_line_everywhere():
    """Prompts whose units and parts begin at every kind of place: short last units, tiles before the first one seen."""
    for seed, heads, kv_heads in ((101, 7, 1), (103, 4, 4), (107, 24, 1)):
        new = [1000, 3, 517, 129, 64, 1]
        kv = [1000, 4000, 516, 2000, 63, 9000]
        m = Made(seed, new, kv, heads=heads, kv_heads=kv_heads, dim=128, page=128)
        check(m.cache.prefill(m.batch, m.q), None, m.expected(m.q, 128 ** -0.5, False), BF16)


def test_sequences_without_tokens():
    from paper_2602_11688_b200 import binding as gb
    m = Made(83, [2], [2], heads=4, kv_heads=2, dim=64)
    none = torch.zeros((2, 0), dtype=torch.int32, device="cuda")
    batch = gb.GorgoKvBatch([0, 0], [0, 0], none)
    assert m.cache.prefill(batch, m.q[:0]).shape == (0, 4, 64)
    lse = torch.empty((2, 4), device="cuda")
    out = m.cache.decode(batch, m.q, lse=lse)
    assert bool((out == 0).all()) and bool((lse == -torch.inf).all())
    batch = gb.GorgoKvBatch([2, 0], [0, 0], none)            # new rows of a sequence without tokens
    lse = torch.empty((2, 4), device="cuda")
    out = m.cache.prefill(batch, m.q, lse=lse)
    assert bool((out == 0).all()) and bool((lse == -torch.inf).all())
    batch.check()
    assert [x.shape[0] for x in m.cache.read(gb.GorgoKvBatch([], [], none[:0]))] == [0, 0]


def test_calls_side_by_side_on_several_streams():
    """Calls that run at the same time have workspaces of their own."""
    made = [Made(89 + i, [1, 40 + i, 7], [900 + i, 300, 7 + i], heads=8, kv_heads=2, dim=128, page=64,
                 store=E4M3 if i % 2 else BF16) for i in range(4)]
    first = [(m.cache.prefill(m.batch, m.q), m.cache.decode(m.batch, m.q[:3])) for m in made]
    streams = [torch.cuda.Stream() for _ in made]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    again = [[] for _ in made]
    for _ in range(20):
        for m, s, a in zip(made, streams, again):
            with torch.cuda.stream(s):
                a.append((m.cache.prefill(m.batch, m.q), m.cache.decode(m.batch, m.q[:3])))
    torch.cuda.synchronize()
    for f, a in zip(first, again):
        assert all(torch.equal(x, y) for pair in a for x, y in zip(pair, f))


def test_the_same_call_gives_the_same_bits_and_streams_and_graphs_do_too():
    m = Made(59, [1] * 5, [3000, 17, 0, 900, 4097], heads=8, kv_heads=2, dim=128, page=128)
    n = Made(61, [300, 20], [2000, 20], heads=8, kv_heads=2, dim=128, page=128)
    calls = [lambda: m.cache.decode(m.batch, m.q), lambda: n.cache.prefill(n.batch, n.q)]
    for call in calls:
        first = call()
        assert all(torch.equal(call(), first) for _ in range(5))
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            assert torch.equal(call(), first)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = call()
        for _ in range(3):
            out.zero_()
            graph.replay()
            assert torch.equal(out, first)


def test_a_graph_replayed_with_other_lengths():
    m = Made(67, [1] * 4, [700, 64, 300, 1], heads=4, kv_heads=2, dim=64, page=64)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = m.cache.decode(m.batch, m.q)
    for kv in ([5, 64, 299, 0], [700, 0, 0, 0], [1, 1, 300, 1]):
        m.batch.kv_len.copy_(torch.tensor(kv, dtype=torch.int32))
        graph.replay()
        m.kv = kv
        check(out, None, m.expected(m.q, 0.125, True), BF16)


def test_an_offset_beyond_32_bits():
    """A pool of more than 2^32 elements: the last page's rows are found."""
    from paper_2602_11688_b200 import binding as gb
    pages, page = 4200, 1024
    cache = gb.GorgoKvCache(*[torch.empty((pages, 8, page, 128), dtype=BF16, device="cuda") for _ in "kv"])
    table = torch.tensor([[pages - 1, 0, pages - 2]], dtype=torch.int32, device="cuda")
    batch = gb.GorgoKvBatch([2100], [2100], table)
    k, v = (torch.randn((2100, 8, 128), device="cuda").to(BF16) for _ in "kv")
    cache.write(batch, k, v)
    assert all(torch.equal(a, b) for a, b in zip(cache.read(batch), (k, v)))
    q = torch.randn((2100, 8, 128), device="cuda").to(BF16)
    out, one = cache.prefill(batch, q), cache.decode(batch, q[-1:])
    z = torch.einsum("hd,khd->hk", q[-1].double(), k.double()) / 128 ** 0.5
    ref = torch.einsum("hk,khd->hd", torch.softmax(z, 1), v.double())
    batch.check()
    for o in (out[-1], one[0]):
        assert (o.double() - ref).abs().max().item() < 3e-3   # values of about 0.03, each rounded by at most 2^-8 twice
