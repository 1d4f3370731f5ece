"""Waits of the attention kernels that run out: a short limit on the host's side makes them, the calls end with their status,
and the next ones are as before."""
import pytest
import torch

from tests.kv_util import BF16, E4M3, FP16, Made

pytestmark = pytest.mark.gpu


@pytest.fixture
def limit():
    from paper_2602_11688_b200 import binding as gb

    def set_limit(ticks):
        assert gb.gorgo_debug_set(None, gb.GORGO_DEBUG_KV_WAIT_TICKS, ticks) == gb.GORGO_OK

    yield set_limit
    set_limit((1 << 32) - 1)


@pytest.mark.parametrize("dtype,store", [(BF16, BF16), (FP16, E4M3)])
@pytest.mark.parametrize("new,kv,heads,kv_heads,dim", [
    ((3,), (30,), 4, 2, 64), ((1000, 7, 300), (1000, 900, 3000), 8, 2, 128), ((64, 64), (20000, 9000), 16, 2, 64)])
def test_prefill_gives_up(limit, dtype, store, new, kv, heads, kv_heads, dim):
    """Rows are right, NaN or untouched, whenever a role gives up; nothing behind the rows is written."""
    from paper_2602_11688_b200 import binding as gb
    m = Made(127, new, kv, heads=heads, kv_heads=kv_heads, dim=dim, dtype=dtype, store=store, page=64)
    n = sum(new)
    first = m.cache.prefill(m.batch, m.q)
    m.batch.check()
    said = []
    for ticks in (0, 300, 1000, 2000, 4000, 8000, 16000, 64000):
        limit(ticks)
        out = torch.full((n + 2, heads, dim), 7.0, dtype=dtype, device="cuda")
        for _ in range(5):
            out.fill_(7.0)
            m.cache.prefill(m.batch, m.q, out=out)
            same = (out[:n].view(torch.int16) == first.view(torch.int16)).all(-1)
            assert bool((same | torch.isnan(out[:n]).all(-1) | (out[:n] == 7).all(-1)).all())
            assert bool((out[n:] == 7).all())
            said.append(int(m.batch.status.item()))
            assert said[-1] in (0, gb.GORGO_KV_WAIT_LIMIT)
            if said[-1] == 0:
                assert bool(same.all())
            m.batch.status.zero_()
        limit((1 << 32) - 1)
        assert torch.equal(m.cache.prefill(m.batch, m.q).view(torch.int16), first.view(torch.int16))
        m.batch.check()
    if n > 1000:
        assert said[0] == gb.GORGO_KV_WAIT_LIMIT


@pytest.mark.parametrize("dtype,store", [(BF16, BF16), (FP16, FP16), (BF16, E4M3), (FP16, E4M3)])
@pytest.mark.parametrize("kv,heads,kv_heads,dim", [((1,), 4, 2, 64), ((30000, 0, 300, 60000), 16, 8, 128), ((70,) * 200, 16, 1, 64)])
def test_decode_gives_up(limit, dtype, store, kv, heads, kv_heads, dim):
    from paper_2602_11688_b200 import binding as gb
    m = Made(131, [1] * len(kv), kv, heads=heads, kv_heads=kv_heads, dim=dim, dtype=dtype, store=store, page=64)
    n = len(kv)
    first = m.cache.decode(m.batch, m.q)
    m.batch.check()
    said = []
    for ticks in (0, 300, 1000, 2000, 4000, 16000):
        limit(ticks)
        out = torch.empty((n + 2, heads, dim), dtype=dtype, device="cuda")
        for _ in range(5):
            out.fill_(7.0)
            m.cache.decode(m.batch, m.q, out=out)
            same = (out[:n].view(torch.int16) == first.view(torch.int16)).all(-1)
            assert bool((same | torch.isnan(out[:n]).all(-1)).all())
            assert bool((out[n:] == 7).all())
            said.append(int(m.batch.status.item()))
            assert said[-1] == (0 if bool(same.all()) else gb.GORGO_KV_WAIT_LIMIT)
            m.batch.status.zero_()
        limit((1 << 32) - 1)
        assert torch.equal(m.cache.decode(m.batch, m.q).view(torch.int16), first.view(torch.int16))
        m.batch.check()
    if max(kv) > 1000 and store != E4M3:                     # more than the L2 holds; codes may arrive before they are waited for
        assert gb.GORGO_KV_WAIT_LIMIT in said[:5]
