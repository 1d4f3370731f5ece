"""The paged key-value cache's attention at the ends of its numbers' ranges."""
import pytest
import torch

from tests.kv_util import BF16, E4M3, FP16, Made, check, half_step, power, quantise

pytestmark = pytest.mark.gpu

TYPES = [(BF16, BF16), (FP16, FP16), (BF16, E4M3), (FP16, E4M3)]


def refill(m, pool, exps, kept, s, x):
    """Sequence s's keys or values become the rows of x, as the cache holds them."""
    at, slot = m.where(s, torch.arange(x.shape[0], device="cuda"))
    if m.store == E4M3:
        codes, e = quantise(x)
        pool.view(torch.uint8)[at, :, slot] = codes.to(E4M3).view(torch.uint8)
        exps[at, :, slot] = e.to(torch.int8)
        kept[s] = codes * power(e[..., None])
    else:
        pool[at, :, slot] = x.to(m.store)
        kept[s] = x.to(m.store).double()


def attend(m, decode, q, scale):
    n = len(m.kv) if decode else sum(m.new)
    l = torch.zeros((n, m.heads), device="cuda")
    out = (m.cache.decode if decode else m.cache.prefill)(m.batch, q, scale, lse=l)
    m.batch.check()
    return out, l


@pytest.mark.parametrize("dtype,store", TYPES)
@pytest.mark.parametrize("decode", [False, True])
def test_scores_beyond_32_bits(dtype, store, decode):
    m = Made(59, [1, 3, 140], [1, 200, 140], heads=4, kv_heads=2, dim=64, dtype=dtype, store=store, page=64)
    for s, n in enumerate(m.kv):
        refill(m, m.cache.k, m.cache.k_exp, m.keys, s, torch.ones((n, 2, 64), device="cuda"))
    out, lse = attend(m, decode, torch.ones_like(m.q), 1e37)                # scores of 64 * 1e37
    assert not bool(torch.isfinite(out).any()) and not bool(torch.isfinite(lse).any()) and not bool((lse == -torch.inf).any())


@pytest.mark.parametrize("decode", [False, True])
@pytest.mark.parametrize("store", [BF16, E4M3])
@pytest.mark.parametrize("scale", [0.0, 1e-38, -1e-36])
def test_scales_next_to_nothing(decode, store, scale):
    """Products of about 2^110 times a scale of about nothing."""
    m = Made(67, [1, 3, 140], [1, 200, 140], heads=4, kv_heads=2, dim=64, store=store, page=64)
    for s, n in enumerate(m.kv):
        refill(m, m.cache.k, m.cache.k_exp, m.keys, s, (m.keys[s] * 2.0 ** 55).to(BF16))
    q = (m.q.float() * 2.0 ** 55).to(BF16)
    out, lse = attend(m, decode, q, scale)
    check(out, lse, m.expected(q, scale, decode), BF16)


@pytest.mark.parametrize("dtype", [BF16, FP16])
@pytest.mark.parametrize("decode", [False, True])
def test_scores_of_minus_infinity(dtype, decode):
    for none in (1, 40, 130, 200):
        m = Made(61, [1, 3, 140], [1, 200, 140], heads=4, kv_heads=2, dim=64, dtype=dtype, page=64)
        m.q[:, :, 7] = 0.5
        for s, n in enumerate(m.kv):
            k = m.keys[s].clone()
            k[:none, :, 7] = -torch.inf
            refill(m, m.cache.k, None, m.keys, s, k)
        out, lse = attend(m, decode, m.q, 0.125)
        row = 0
        for s, (n, kv) in enumerate(zip(m.new, m.kv)):
            for i in range(1 if decode else n):
                seen = kv if decode else kv - n + i + 1
                q = m.q[s if decode else row]
                if seen <= none:
                    assert bool((out[row] == 0).all()) and bool((lse[row] == -torch.inf).all()), (none, s, i)
                else:
                    k, v = m.keys[s][none:seen].repeat_interleave(2, 1), m.values[s][none:seen].repeat_interleave(2, 1)
                    z = torch.einsum("hd,khd->hk", q.double(), k) * 0.125
                    p = torch.softmax(z, 1)
                    ref, sizes = torch.einsum("hk,khd->hd", p, v), torch.einsum("hk,khd->hd", p, v.abs())
                    u = half_step(dtype)
                    assert bool(((out[row].double() - ref).abs() <= sizes * (u + 2.0 ** -10) + ref.abs() * u + 2.0 ** -20).all())
                row += 1


@pytest.mark.parametrize("dtype,store", TYPES)
@pytest.mark.parametrize("decode", [False, True])
def test_scores_below_32_bits(dtype, store, decode):
    m = Made(59, [1, 3, 140], [1, 200, 140], heads=4, kv_heads=2, dim=64, dtype=dtype, store=store, page=64)
    for s, n in enumerate(m.kv):
        refill(m, m.cache.k, m.cache.k_exp, m.keys, s, -torch.ones((n, 2, 64), device="cuda"))
    out, lse = attend(m, decode, torch.ones_like(m.q), 1e37)
    assert bool((out == 0).all()) and bool((lse == -torch.inf).all())


@pytest.mark.parametrize("decode", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("k_size,v_size,scale", [(2.0 ** 17, 1.0, 2.0 ** -20), (1.0, 2.0 ** 12, 0.125),
                                                  (2.0 ** -18, 1.0, 2.0 ** 14), (1.0, 2.0 ** -14, 0.125)])
def test_fp16_rows_on_codes_beyond_fp16(decode, dim, k_size, v_size, scale):
    """Codes of a cache that was filled from bf16: what they stand for need not fit fp16, the result does."""
    m = Made(71, [1, 3, 140], [1, 200, 140], heads=4, kv_heads=2, dim=dim, dtype=FP16, store=E4M3, page=64)
    g = torch.Generator(device="cuda").manual_seed(1)
    for s, n in enumerate(m.kv):
        refill(m, m.cache.k, m.cache.k_exp, m.keys, s, m.keys[s] * k_size)
        big = 1.0 + 15.0 * (torch.rand((n, 1, 1), generator=g, device="cuda") < 0.1) if v_size > 1 and n > 1 else 1.0
        refill(m, m.cache.v, m.cache.v_exp, m.values, s, m.values[s] * v_size * big)
    out, lse = attend(m, decode, m.q, scale)
    want = m.expected(m.q, scale, decode)
    want[2] += 2.0 ** -25                                    # a result below fp16's normal range: half a step of 2^-24
    fits = want[0].abs().amax((1, 2)) < 65000                # (rows of few keys may not)
    assert int(fits.sum()) >= fits.numel() // 2
    check(out[fits], lse[fits], [w[fits] for w in want], FP16)


@pytest.mark.parametrize("decode", [False, True])
def test_the_largest_fp16_value_in_a_row_of_codes(decode):
    m = Made(73, [140], [140], heads=4, kv_heads=2, dim=64, dtype=FP16, store=E4M3, page=64)
    v = m.values[0].clone()
    v[3, :, 9] = 65504.0                                     # rounds to a code that stands for 65,536
    refill(m, m.cache.v, m.cache.v_exp, m.values, 0, v)
    q = m.q * 0.1
    q[:20] = 0                                               # (rows of few keys: their share of it fits)
    out, lse = attend(m, decode, q, 0.125)
    want = m.expected(q, 0.125, decode)
    fits = want[0].abs().amax((1, 2)) < 65000
    assert int(fits.sum()) >= fits.numel() // 2
    check(out[fits], lse[fits], [w[fits] for w in want], FP16)


@pytest.mark.parametrize("decode", [False, True])
def test_values_far_apart_in_size(decode):
    """Rows of zeros beside one of about 2^125, all scores zero: each key counts the same."""
    for kv in (2, 40, 300, 9000):
        for at in (0, kv // 2, kv - 1):
            m = Made(79, [1], [kv], heads=4, kv_heads=2, dim=64, store=E4M3, page=64)
            v = torch.zeros((kv, 2, 64), dtype=torch.float64, device="cuda")
            v[at] = 2.0 ** 125
            refill(m, m.cache.v, m.cache.v_exp, m.values, 0, v)
            out, lse = attend(m, decode, m.q * 0, 0.125)
            want = v[at, 0, 0] / kv
            assert bool(((out.double() - want).abs() <= want * (2 * 2.0 ** -8 + 2.0 ** -10)).all()), (kv, at)
            assert bool(((lse.double() - torch.log(torch.tensor(float(kv)))).abs() < 1e-4).all())
