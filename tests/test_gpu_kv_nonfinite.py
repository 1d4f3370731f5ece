"""What is not finite in the paged key-value cache: where it reaches and where it does not."""
import pytest
import torch

from tests.kv_util import BF16, E4M3, FP16, Made, check

pytestmark = pytest.mark.gpu


def test_a_row_with_a_score_that_is_none_stays_without_a_result():
    """A key that is NaN before a value that is NaN and not seen: the rows between are NaN in every element."""
    m = Made(83, [200], [200], heads=4, kv_heads=2, dim=64, page=64)
    for j, pool, d in ((0, m.cache.k, 3), (40, m.cache.v, 5)):
        pg, slot = m.where(0, torch.tensor([j], device="cuda"))
        pool[pg, :, slot, d] = float("nan")
    out = m.cache.prefill(m.batch, m.q)
    assert bool(torch.isnan(out).all())


@pytest.mark.parametrize("dtype,store", [(BF16, BF16), (FP16, FP16), (BF16, E4M3), (FP16, E4M3)])
@pytest.mark.parametrize("heads,kv_heads,dim", [(4, 2, 64), (8, 2, 128), (7, 1, 128)])
def test_a_value_in_whole_and_in_split_units(dtype, store, heads, kv_heads, dim):
    for new, kv, at in (((200, 30), (200, 64), 69), ((300, 30), (4000, 64), 3850), ((300, 1), (20000, 64), 19990)):
        m = Made(103, new, kv, heads=heads, kv_heads=kv_heads, dim=dim, dtype=dtype, store=store, page=64)
        want = m.expected(m.q, dim ** -0.5, False)
        pg, slot = m.where(0, torch.tensor([at], device="cuda"))
        if store == E4M3:
            m.cache.v.view(torch.uint8)[pg, kv_heads - 1, slot, 5] = 0x7f
        else:
            m.cache.v[pg, kv_heads - 1, slot, 5] = float("inf")
        out = m.cache.prefill(m.batch, m.q)
        assert all(torch.equal(m.cache.prefill(m.batch, m.q).view(torch.int16), out.view(torch.int16)) for _ in range(3))
        m.batch.check()
        hit = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
        hit[at - (kv[0] - new[0]):new[0], heads - heads // kv_heads:, 5] = True
        assert not bool(torch.isfinite(out[hit]).any())
        out[hit] = want[0][hit].to(dtype)
        check(out, None, want, dtype)


def test_values_at_every_other_key():
    """Rows that see such a value have that element without a result anyway; no row is lost beside it."""
    m = Made(109, [300, 30], [400, 64], heads=4, kv_heads=2, dim=64, page=64)
    want = m.expected(m.q, 0.125, False)
    pg, slot = m.where(0, torch.arange(151, 400, 2, device="cuda"))
    m.cache.v[pg, :, slot, 9] = float("nan")
    pg, slot = m.where(0, torch.arange(310, 400, device="cuda"))
    m.cache.v[pg, 0, slot, 20] = -float("inf")
    out = m.cache.prefill(m.batch, m.q)
    m.batch.check()
    hit = torch.zeros(out.shape, dtype=torch.bool, device="cuda")
    hit[51:300, :, 9] = hit[210:300, :2, 20] = True
    assert not bool(torch.isfinite(out[hit]).any())
    out[hit] = want[0][hit].to(BF16)
    check(out, None, want, BF16)


def test_rows_of_long_prefixes_are_computed_again_in_parallel():
    """A value that is not finite under the last rows of 300 heads: their rows, 30,000 keys each, do not follow one another
    (a warp of 32 such rows in a series takes 0.6 s), and no wait runs out."""
    n, heads = 30_000, 300
    m = Made(113, [64], [n], heads=heads, kv_heads=heads, dim=64, page=512)
    pg, slot = m.where(0, torch.tensor([n - 1], device="cuda"))
    m.cache.v[pg, :, slot, 5] = float("nan")
    m.cache.prefill(m.batch, m.q)
    a, b = (torch.cuda.Event(enable_timing=True) for _ in "ab")
    a.record()
    out = m.cache.prefill(m.batch, m.q)
    b.record()
    m.batch.check()
    assert bool(torch.isnan(out[63, :, 5]).all())
    out[63, :, 5] = 0
    assert bool(torch.isfinite(out).all())
    for h in (0, 149, 299):
        for i in (0, 37, 62):
            k, v = m.keys[0][:n - 63 + i, h], m.values[0][:n - 63 + i, h]
            p = torch.softmax(k @ m.q[i, h].double() * 0.125, 0)
            ref, sizes = p @ v, p @ v.abs()
            assert bool(((out[i, h].double() - ref).abs() <= sizes * 2.0 ** -9 + ref.abs() * 2.0 ** -8 + 2.0 ** -20).all())
    assert a.elapsed_time(b) < 300
