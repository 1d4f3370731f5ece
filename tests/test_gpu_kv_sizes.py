"""The paged key-value cache at the largest sizes that the header allows, and graphs replayed with other lengths."""
import pytest
import torch

from tests.kv_util import BF16, E4M3, Made, check, power, quantise

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("store", [BF16, E4M3])
def test_graphs_replayed_with_other_lengths(store):
    m = Made(107, [70, 3, 130], [300, 64, 130], heads=4, kv_heads=2, dim=64, page=64, store=store)
    x = torch.randn((203, 2, 64), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").to(BF16)
    m.cache.prefill(m.batch, m.q)
    torch.cuda.synchronize()
    graph, put = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = m.cache.prefill(m.batch, m.q)
        k, v = m.cache.read(m.batch)
    with torch.cuda.graph(put):
        m.cache.write(m.batch, x, -x)
    for new, kv in (((70, 3, 130), (300, 64, 130)), ((1, 0, 100), (200, 0, 128)), ((0, 2, 1), (0, 64, 1)), ((130, 60, 3), (300, 64, 3))):
        m.batch.cu_new.copy_(torch.tensor([0, new[0], new[0] + new[1], sum(new)], dtype=torch.int32))
        m.batch.kv_len.copy_(torch.tensor(kv, dtype=torch.int32))
        m.new, m.kv, n = new, kv, sum(new)
        out.fill_(7.0), k.fill_(7.0), v.fill_(7.0)
        graph.replay()
        m.batch.check()
        check(out[:n], None, m.expected(m.q, 0.125, False), BF16)
        assert bool((out[n:] == 7).all()) and bool((k[n:] == 7).all()) and bool((v[n:] == 7).all())
        for got, kept in ((k, m.keys), (v, m.values)):
            assert torch.equal(got[:n], torch.cat([kept[s][kv[s] - new[s]:kv[s]] for s in range(3)]).to(BF16))
        put.replay()                                         # other tokens in their places
        at = 0
        for s in range(3):
            for kept, rows in ((m.keys, x), (m.values, -x)):
                rows = rows[at:at + new[s]].double()
                if store == E4M3 and new[s]:
                    codes, e = quantise(rows)
                    rows = codes * power(e[..., None])
                kept[s] = kept[s].clone()
                kept[s][kv[s] - new[s]:kv[s]] = rows
            at += new[s]
        m.batch.check()


@pytest.mark.parametrize("store", [BF16, E4M3])
def test_as_many_sequences_as_there_may_be(store):
    from paper_2602_11688_b200 import binding as gb
    n, page = 65535, 16
    g = torch.Generator(device="cuda").manual_seed(3)
    kv = [1 + s % 3 for s in range(n)]
    table = torch.randperm(n, generator=g, device="cuda").to(torch.int32).view(n, 1)
    cache = gb.GorgoKvCache.empty(n, 1, 64, store, page)
    k, v = (torch.randn((n, 3, 64), generator=g, device="cuda").to(BF16) for _ in "kv")
    q = torch.randn((n, 2, 64), generator=g, device="cuda").to(BF16)
    for t in range(3):                                       # token t of those that have one
        some = [int(x > t) for x in kv]
        rows = torch.tensor(some, device="cuda").bool()
        cache.write(batch := gb.GorgoKvBatch(some, [min(x, t + 1) for x in kv], table), k[rows, t:t + 1], v[rows, t:t + 1])
        batch.check()
    batch = gb.GorgoKvBatch([1] * n, kv, table)
    last = torch.tensor(kv, device="cuda") - 1
    back = cache.read(batch, BF16)
    pre, dec = cache.prefill(batch, q), cache.decode(batch, q)
    batch.check()
    if store == E4M3:
        k, v = (c * power(e[..., None]) for c, e in (quantise(x) for x in (k, v)))
    for got, x in zip(back, (k, v)):
        assert torch.equal(got[:, 0], x[torch.arange(n, device="cuda"), last].to(BF16))
    z = torch.einsum("nhd,nkd->nhk", q.double(), k.double()) / 8
    z = z.masked_fill(torch.arange(3, device="cuda") > last[:, None, None], -torch.inf)
    p = torch.softmax(z, 2)
    ref, sizes = torch.einsum("nhk,nkd->nhd", p, v.double()), torch.einsum("nhk,nkd->nhd", p, v.double().abs())
    for out in (pre, dec):                                   # P and the result rounded, 2^-10 for 32-bit sums and exponentials
        assert bool(((out.double() - ref).abs() <= sizes * (2.0 ** -8 + 2.0 ** -10) + ref.abs() * 2.0 ** -8 + 2.0 ** -20).all())


@pytest.mark.parametrize("store", [BF16, E4M3])
def test_as_long_a_sequence_as_there_may_be(store):
    from paper_2602_11688_b200 import binding as gb
    n, page = (1 << 24) - 1, 1024
    g = torch.Generator(device="cuda").manual_seed(5)
    pages = 1 << 14
    table = torch.randperm(pages, generator=g, device="cuda").to(torch.int32).view(1, pages)
    cache = gb.GorgoKvCache.empty(pages, 1, 64, store, page)
    k, v = (torch.randn((n, 1, 64), generator=g, device="cuda", dtype=BF16) for _ in "kv")
    cache.write(batch := gb.GorgoKvBatch([n], [n], table), k, v)
    batch.check()
    k, v = cache.read(batch, BF16)                           # (exact for e4m3: what the codes stand for)
    batch.check()
    q = torch.randn((5, 4, 64), generator=g, device="cuda").to(BF16)
    batch = gb.GorgoKvBatch([5], [n], table)
    pre, dec = cache.prefill(batch, q), cache.decode(batch, q[4:])
    batch.check()
    z = torch.cat([torch.einsum("nhd,kd->nhk", q.double(), c[:, 0].double()) / 8 for c in k.split(1 << 21)], 2)
    for i in range(4):
        z[i, :, n - 4 + i:] = -torch.inf
    p = torch.exp(z - torch.logsumexp(z, 2, keepdim=True))
    ref = sum(torch.einsum("nhk,kd->nhd", a, b[:, 0].double()) for a, b in zip(p.split(1 << 21, 2), v.split(1 << 21)))
    sizes = sum(torch.einsum("nhk,kd->nhd", a, b[:, 0].double().abs()) for a, b in zip(p.split(1 << 21, 2), v.split(1 << 21)))
    # P rounded, n of them with errors of either sign: their sum's is below 2^-8 of sizes / sqrt(n) by far, the accumulators' in
    # the sums (2^-24 a step, 2^17 steps of 128 keys over 148 parts: 2^10 steps a part) below 2^-13 of sizes
    for out, rows in ((pre, slice(0, 5)), (dec, slice(4, 5))):
        assert bool(((out.double() - ref[rows]).abs() <= sizes[rows] * 2.0 ** -13 + ref[rows].abs() * 2.0 ** -8).all())
