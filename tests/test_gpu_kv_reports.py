"""What the paged key-value cache's calls do with wrong pages and lengths: what they report, which rows they spoil
and which they leave."""
import pytest
import torch

from tests.kv_util import BF16, E4M3, FP16, Made, check

pytestmark = pytest.mark.gpu

TYPES = [(BF16, BF16), (FP16, FP16), (BF16, E4M3), (FP16, E4M3)]


@pytest.mark.parametrize("dtype,store", TYPES)
@pytest.mark.parametrize("decode", [False, True])
@pytest.mark.parametrize("fault", ["page", "low page", "kv", "low kv"])
def test_a_wrong_page_or_length_in_every_type_of_cache(dtype, store, decode, fault):
    from paper_2602_11688_b200 import binding as gb
    m = Made(53, [3, 4, 2], [30, 70, 40], page=16, dtype=dtype, store=store)
    want = m.expected(m.q, 0.125, decode)
    if fault.endswith("page"):
        m.batch.table[1, 2] = m.cache.n_pages if fault == "page" else -1
    else:
        m.batch.kv_len[1] = 71 if fault == "kv" else -1
    lse = torch.zeros((9, 4), device="cuda")
    out = (m.cache.decode if decode else m.cache.prefill)(m.batch, m.q, lse=lse)
    assert int(m.batch.status.item()) == (gb.GORGO_KV_BAD_PAGE if fault.endswith("page") else gb.GORGO_KV_BAD_LENGTH)
    n = 3 if decode else 9
    lo, hi = (1, 2) if decode else (3, 7)
    assert bool(torch.isnan(out[lo:hi]).all()) and bool(torch.isnan(lse[lo:hi]).all())
    keep = [i for i in range(n) if not lo <= i < hi]
    check(out[keep], lse[keep], [w[keep] for w in want], dtype)
    k, v = m.cache.read(m.batch, dtype)                      # which needs the new tokens' pages alone
    for o, kept in ((k, m.keys), (v, m.values)):
        ref = torch.cat([x[-n:] for x, n in zip(kept, m.new)]).to(dtype)
        if fault.endswith("kv"):
            assert bool(torch.isnan(o[3:7]).all())
            o, ref = (torch.cat([x[:3], x[7:]]) for x in (o, ref))
        assert torch.equal(o, ref)


@pytest.mark.parametrize("store", [BF16, E4M3])
def test_rows_that_see_a_wrong_page_and_rows_before_it(store):
    from paper_2602_11688_b200 import binding as gb
    for at in (0, 40, 130, 200, 299):
        m = Made(57, [300, 40], [300, 200], heads=4, kv_heads=2, dim=64, page=16, store=store)
        want = m.expected(m.q, 0.125, False)
        m.batch.table[0, at // 16] = m.cache.n_pages
        for _ in range(3):
            out = m.cache.prefill(m.batch, m.q)
            assert int(m.batch.status.item()) == gb.GORGO_KV_BAD_PAGE
            first = at // 16 * 16
            assert bool(torch.isnan(out[first:300]).all())
            keep = list(range(first)) + list(range(300, 340))
            check(out[keep], None, [w[keep] for w in want], BF16)
