"""Writing into and reading out of the paged key-value cache against the definition in 64 bits, bit by bit."""
import pytest
import torch

from tests.kv_util import BF16, E4M3, FP16, Made, power, quantise, table_for

pytestmark = pytest.mark.gpu

LENGTHS = [(0, 0), (1, 1), (1, 17), (5, 5), (0, 9), (63, 64), (130, 131), (2, 600)]    # (new, all)


def make(seed, lengths, kv_heads, dim, store, page):
    import numpy as np
    from paper_2602_11688_b200 import binding as gb
    table, pages = table_for([b for _, b in lengths], page, np.random.default_rng(seed))
    cache = gb.GorgoKvCache.empty(pages, kv_heads, dim, store, page)
    g = torch.Generator(device="cuda").manual_seed(seed)
    for x in (cache.k, cache.v):
        x.view(torch.uint8).random_(0, 256, generator=g)
    for x in (cache.k_exp, cache.v_exp):
        if x is not None:
            x.random_(-24, 10, generator=g)
    return cache, gb.GorgoKvBatch([a for a, _ in lengths], [b for _, b in lengths], table), table


def bits(x):
    return x.contiguous().view(torch.uint8).clone()


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("quant", [False, True])
@pytest.mark.parametrize("kv_heads,dim,page", [(1, 64, 16), (3, 128, 64), (8, 128, 512), (5, 64, 1024), (20, 64, 32)])
def test_written_rows_and_everything_else(dtype, quant, kv_heads, dim, page):
    store = E4M3 if quant else dtype
    cache, batch, table = make(1, LENGTHS, kv_heads, dim, store, page)
    total = batch.total_new
    g = torch.Generator(device="cuda").manual_seed(2)
    fused = torch.randn((total + 3, 2 * kv_heads + 1, dim), generator=g, device="cuda")
    fused *= torch.exp(3 * torch.randn((total + 3, 2 * kv_heads + 1, 1), generator=g, device="cuda"))
    fused = fused.to(dtype)
    fused[0, 0] = 0                                          # rows whose largest value is 0, a border or tiny
    fused[1, 0, :] = 0
    fused[1, 0, 3] = 448.0
    fused[2, 0, :] = 0
    fused[2, 0, 5] = 449.0 if dtype == FP16 else 450.0
    fused[3, 0] = 2.0 ** -24
    fused[4, 0, :8] = torch.tensor([1.0625, 1.1875, -1.0625, 2 ** -7, 2 ** -10, 3 * 2 ** -10, 448, -432], dtype=dtype)  # ties
    k_new, v_new = fused[:, :kv_heads], fused[:, kv_heads:2 * kv_heads]      # rows with a stride of their own
    want = {x: bits(getattr(cache, x)) for x in ("k", "v") + (("k_exp", "v_exp") if quant else ())}
    for s, (n, kv) in enumerate(LENGTHS):
        at = int(batch.cu_new[s])
        j = torch.arange(kv - n, kv, device="cuda")
        pg, slot = table[s].long()[j // page], j % page
        for x, rows in (("k", k_new[at:at + n]), ("v", v_new[at:at + n])):
            if n == 0:
                continue
            view = want[x].view(cache.k.shape[:3] + (-1,))
            if quant:
                codes, e = quantise(rows)
                view[pg, :, slot] = codes.to(E4M3).view(torch.uint8)
                want[x + "_exp"].view(torch.int8).view(cache.k.shape[:3])[pg, :, slot] = e.to(torch.int8)
            else:
                view[pg, :, slot] = rows.contiguous().view(torch.uint8).view(n, kv_heads, -1)
    cache.write(batch, k_new, v_new)
    batch.check()
    for x, w in want.items():
        wrong = int((bits(getattr(cache, x)).view(-1) != w.view(-1)).sum())
        assert wrong == 0, x
    # and back: what the codes stand for, in both types where the cache has codes
    for out_type in (BF16, FP16) if quant else (dtype,):
        out = [torch.full((total + 4, kv_heads + 1, dim), 7.0, dtype=out_type, device="cuda") for _ in "kv"]
        cache.read(batch, out=tuple(o[:, :kv_heads] for o in out))
        batch.check()
        for o, rows in zip(out, (k_new, v_new)):
            ref = rows[:total]
            if quant:
                codes, e = quantise(ref)
                ref = (codes * power(e[..., None])).float().to(out_type)
            got, ref = (x.contiguous().view(torch.int16) for x in (o[:total, :kv_heads], ref))
            both = torch.isnan(got.view(out_type)) & torch.isnan(ref.view(out_type))
            wrong = int(((got != ref) & ~both).sum())
            assert wrong == 0
            assert bool((o[total:] == 7).all()) and bool((o[:, kv_heads:] == 7).all())


def test_rows_with_a_nan_or_an_infinity_are_nan_in_e4m3():
    cache, batch, _ = make(3, [(4, 4)], 2, 64, E4M3, 16)
    x = torch.ones((4, 2, 64), dtype=BF16, device="cuda")
    x[0, 0, 9], x[1, 1, 63], x[2, 0, 0] = float("nan"), float("inf"), -float("inf")
    cache.write(batch, x, x)
    k, v = cache.read(batch, BF16)
    nan = torch.zeros((4, 2), dtype=torch.bool, device="cuda")
    nan[0, 0] = nan[1, 1] = nan[2, 0] = True
    for o in (k, v):
        assert torch.equal(torch.isnan(o).all(-1), nan) and torch.equal(torch.isnan(o).any(-1), nan)
        assert bool((o[~nan] == 1).all())


def test_the_holders_refuse_what_does_not_fit():
    from paper_2602_11688_b200 import binding as gb
    cache, batch, table = make(9, [(3, 40), (2, 2)], 2, 64, BF16, 16)
    x, q = (torch.zeros((5, h, 64), dtype=BF16, device="cuda") for h in (2, 4))
    for bad in (x[:4], x[:, :1], x.to(FP16), x.float(), x.cpu(), torch.zeros((5, 2, 128), dtype=BF16, device="cuda"),
                x.transpose(0, 1).contiguous().transpose(0, 1)):
        with pytest.raises((ValueError, gb.GorgoError)):
            cache.write(batch, bad, bad)
        with pytest.raises((ValueError, gb.GorgoError)):
            cache.read(batch, out=(bad, bad))
    with pytest.raises(ValueError):
        cache.write(batch, x, x.to(FP16))
    for bad in (q[:4], q[:, :3], q.to(FP16), q[0], q.float()):
        with pytest.raises((ValueError, gb.GorgoError)):
            cache.prefill(batch, bad)
    for kw in (dict(out=q[:4]), dict(out=q.to(FP16)), dict(lse=torch.zeros((5, 4), device="cuda").half()),
               dict(lse=torch.zeros((4, 4), device="cuda")), dict(scale=float("nan"))):
        with pytest.raises((ValueError, gb.GorgoError)):
            cache.prefill(batch, q, **kw)
    # a table that ends before the longest sequence does, although the rows behind it are long enough
    wide = torch.zeros((2, 9), dtype=torch.int32, device="cuda")
    short = gb.GorgoKvBatch([3, 2], [40, 2], wide[:, :2])
    with pytest.raises(ValueError):
        cache.prefill(short, q)
    for args in (([1], [1, 2], table), ([-1, 1], [1, 2], table), ([1, 1], [1, 2], table.long()), ([1], [1], table),
                 ([1, 1], [1, 2], table.cpu())):
        with pytest.raises(ValueError):
            gb.GorgoKvBatch(*args)
    with pytest.raises(ValueError):
        gb.GorgoKvBatch([1, 1], [1, 2], table, kv_len=torch.zeros(3, dtype=torch.int32, device="cuda"))
    for args in ((cache.k, cache.v[:1]), (cache.k, cache.v.to(FP16)), (cache.k.float(), cache.v.float()), (cache.k[:, :1], cache.v[:, :1]),
                 (cache.k.to(E4M3), cache.v.to(E4M3)), (cache.k, cache.v, torch.zeros(3), None)):
        with pytest.raises(ValueError):
            gb.GorgoKvCache(*args)
    with pytest.raises(gb.GorgoError):                       # pages of a size that the kernels do not have
        gb.GorgoKvCache.empty(4, 2, 64, BF16, 48).write(gb.GorgoKvBatch([5], [5], table[:1]), x, x)


def test_many_tokens_and_many_sequences():
    lengths = [(int(n), int(n) + int(m)) for n, m in zip(torch.randint(0, 9, (700,), generator=torch.Generator().manual_seed(1)),
                                                          torch.randint(0, 40, (700,), generator=torch.Generator().manual_seed(2)))]
    cache, batch, table = make(5, lengths, 2, 64, BF16, 16)
    x = torch.randn((batch.total_new, 2, 64), device="cuda").to(BF16)
    cache.write(batch, x, -x)
    k, v = cache.read(batch)
    batch.check()
    assert torch.equal(k, x) and torch.equal(v, -x)


def test_wrong_pages_and_lengths_are_reported_and_nothing_else_is_touched():
    from paper_2602_11688_b200 import binding as gb
    for fault, bit in (("page", gb.GORGO_KV_BAD_PAGE), ("low page", gb.GORGO_KV_BAD_PAGE), ("kv", gb.GORGO_KV_BAD_LENGTH),
                       ("short", gb.GORGO_KV_BAD_LENGTH), ("cu", gb.GORGO_KV_BAD_LENGTH)):
        m = Made(7, [3, 4, 2], [30, 20, 40], page=16)
        if fault.endswith("page"):
            m.batch.table[1, 1] = m.cache.n_pages if fault == "page" else -1
        elif fault == "kv":
            m.batch.kv_len[1] = 41
        elif fault == "short":
            m.batch.kv_len[1] = 3                            # fewer tokens than new ones: the first has no position
        else:
            m.batch.cu_new[1:3] = torch.tensor([5, 4], dtype=torch.int32, device="cuda")   # decreasing
        x = torch.ones((9, 2, 64), dtype=BF16, device="cuda")
        before = m.cache.k.clone()
        m.cache.write(m.batch, x, x)
        with pytest.raises(gb.GorgoError):
            m.batch.check()
        assert int(m.batch.status.item()) == bit
        changed = (bits(m.cache.k) != bits(before)).view(*m.cache.k.shape[:3], -1).any(-1)
        own = torch.zeros_like(changed)
        for s in range(3):
            j = torch.arange(m.kv[s] - 5, m.kv[s], device="cuda")
            pg, slot = m.table[s].long()[j // 16], j % 16
            ok = (pg >= 0) & (pg < m.cache.n_pages)
            own[pg[ok], :, slot[ok]] = True
        if fault in ("page", "low page", "kv"):
            assert not bool((changed & ~own).any())
        k, v = m.cache.read(m.batch)
        if fault in ("page", "low page", "kv"):
            assert bool(torch.isnan(k[3:7]).any()) and bool((k[:3] == 1).all()) and bool((k[7:] == 1).all())
