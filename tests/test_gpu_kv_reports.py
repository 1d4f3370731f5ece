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


def test_read_leaves_rows_without_a_place():
    from paper_2602_11688_b200 import binding as gb
    m = Made(89, [3, 4, 2], [30, 70, 40], page=16)
    m.batch.cu_new[2] = 100
    out = [torch.full((9, 2, 64), 7.0, dtype=BF16, device="cuda") for _ in "kv"]
    m.cache.read(m.batch, out=tuple(out))
    assert int(m.batch.status.item()) == gb.GORGO_KV_BAD_LENGTH
    for o, kept in zip(out, (m.keys, m.values)):
        assert torch.equal(o[:3], kept[0][-3:].to(BF16)) and bool((o[3:] == 7).all())


def test_prefill_leaves_rows_without_a_place():
    from paper_2602_11688_b200 import binding as gb
    m = Made(89, [3, 4, 2], [30, 70, 40], page=16)
    m.batch.cu_new[2] = 100
    want = m.expected(m.q, 0.125, False)
    out = torch.full((9, 4, 64), 7.0, dtype=BF16, device="cuda")
    m.cache.prefill(m.batch, m.q, out=out)
    assert int(m.batch.status.item()) == gb.GORGO_KV_BAD_LENGTH
    check(out[:3], None, [w[:3] for w in want], BF16)
    assert bool((out[3:] == 7).all())


def test_write_touches_nothing_for_rows_without_a_place():
    for fault in ("beyond", "decreasing", "short"):
        m = Made(89, [3, 4, 2], [30, 70, 40], page=16)
        if fault == "beyond":
            m.batch.cu_new[2] = 100                          # rows 0 to 2 are the first sequence's, the others nobody's
        elif fault == "decreasing":
            m.batch.cu_new[2] = 2
        else:
            m.batch.kv_len[1] = 3                            # four new tokens of three: the first has no position
        x = torch.ones((9, 2, 64), dtype=BF16, device="cuda")
        before = m.cache.k.clone()
        m.cache.write(m.batch, x, x)
        assert int(m.batch.status.item()) == 2
        changed = (m.cache.k.view(torch.int16) != before.view(torch.int16)).any(-1)
        allowed = torch.zeros_like(changed)
        for s, lo, hi in ((0, 27, 30),) + {"beyond": (), "decreasing": ((2, 33, 40),), "short": ((1, 0, 3), (2, 38, 40))}[fault]:
            pg, slot = m.where(s, torch.arange(lo, hi, device="cuda"))
            allowed[pg, :, slot] = True
        assert not bool((changed & ~allowed).any())
        pg, slot = m.where(0, torch.arange(27, 29 if fault == "decreasing" else 30, device="cuda"))   # (row 2 is two sequences' there)
        assert bool((m.cache.k[pg, :, slot] == 1).all())


@pytest.mark.parametrize("call", ["write", "read", "prefill"])
def test_more_new_tokens_than_max_new(call):
    """The first sequence's rows, six of at most four, are reported and left; the others are served."""
    from paper_2602_11688_b200 import binding as gb
    m = Made(97, [3, 4, 2], [30, 70, 40], page=16)
    m.batch.cu_new[1:3] = torch.tensor([6, 8], dtype=torch.int32)
    want = [m.row(1, m.q[6 + i], 69 + i, 0.125) for i in range(2)] + [m.row(2, m.q[8], 40, 0.125)]
    x = torch.zeros((9, 2, 64), dtype=BF16, device="cuda")
    if call == "write":
        before = m.cache.k.clone()
        m.cache.write(m.batch, x, x)
        for s, lo, hi, same in ((0, 24, 30, True), (1, 68, 70, False), (2, 39, 40, False)):
            pg, slot = m.where(s, torch.arange(lo, hi, device="cuda"))
            assert torch.equal(m.cache.k[pg, :, slot], before[pg, :, slot] if same else x[:hi - lo])
    elif call == "read":
        out = x + 7
        m.cache.read(m.batch, out=(out, x))
        assert bool((out[:6] == 7).all()) and torch.equal(out[6:], torch.cat([m.keys[1][-2:], m.keys[2][-1:]]).to(BF16))
    else:
        out = torch.full((9, 4, 64), 7.0, dtype=BF16, device="cuda")
        m.cache.prefill(m.batch, m.q, out=out)
        assert bool((out[:6] == 7).all())
        check(out[6:], None, [torch.stack([w[i] for w in want]) for i in range(3)], BF16)
    assert int(m.batch.status.item()) == gb.GORGO_KV_BAD_LENGTH
