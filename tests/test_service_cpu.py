"""Host side of the measured service model: shapes, fits and the requests it draws from a workload."""
import numpy as np
import pytest

from paper_2602_11688_b200 import service as S
from paper_2602_11688_b200 import tune
from paper_2602_11688_b200 import workloads as W


def test_shapes_are_parsed_and_bad_ones_refused():
    s = S.EngineShape.parse("32x4096x14336x32x8x128")
    assert (s.layers, s.hidden, s.ffn, s.heads, s.kv_heads, s.head_dim) == (32, 4096, 14336, 32, 8, 128)
    assert s.block_bytes(512, "bf16") == 32 * 2 * 8 * 512 * 256
    assert s.block_bytes(512, "e4m3") == 32 * 2 * 8 * 512 * 129
    assert s.weight_bytes() == 2 * 32 * (4096 * 48 * 128 + 32 * 128 * 4096 + 3 * 4096 * 14336)
    for bad in ("", "32x4096", "32x4096x14336x32x8x96", "32x4096x14336x30x8x128", "0x8x8x8x8x64", "1x10x8x8x8x64",
                "1x8x8x129x1x64", "ax8x8x8x8x64"):
        with pytest.raises(ValueError):
            S.EngineShape.parse(bad)
        with pytest.raises(SystemExit):
            tune.main(["--engine", bad])


def test_fits_recover_what_they_model():
    assert S.fit_prefill([10, 100, 1000], [0.5, 5.0, 50.0]) == pytest.approx(0.05)
    tpot, slow = S.fit_decode([1, 4, 16], [20.0 * (1 + 0.03 * (b - 1)) for b in (1, 4, 16)])
    assert (tpot, slow) == (pytest.approx(20.0), pytest.approx(0.03))
    assert S.fit_decode([1], [7.0]) == (7.0, 0.0)
    assert S.fit_decode([1, 2], [7.0, 5.0]) == (6.0, 0.0)    # faster with more slots: no slow-down


def test_requests_are_what_the_previous_turn_leaves_uncached():
    reqs = [(0.0, 1000, 1, [1, 2]), (1.0, 1600, 1, [1, 3, 4, 5]), (2.0, 700, 1, [9, 8]), (3.0, 2000, 1, [1, 3, 4, 6])]
    w = W.handmade(np.array([5.0, 6.0]), reqs, slots=2, cache_blocks=50, params=np.ones((1, 3)))
    w.session[:] = [0, 0, 1, 0]
    got = sorted(S.requests_of(w, 10))
    assert got == sorted([(1000, 1000), (1600 - 512, 1600), (700, 700), (2000 - 3 * 512, 2000)])
    assert len(S.requests_of(w, 2)) == 2


def test_memory_is_given_once():
    """What the prefix cache holds and what the running requests' answers take is the memory that there is."""
    reqs = [(0.0, 1000, 600, [1, 2]), (1.0, 1600, 1030, [1, 3, 4, 5])]
    w = W.handmade(np.array([5.0, 6.0]), reqs, slots=3, cache_blocks=50, params=np.ones((1, 3)))
    blocks, tokens = S.cache_and_budget(100, w)
    assert blocks == 100 - 3 * 3                             # three slots, answers of up to 1,030 tokens
    assert tokens == blocks * 512                            # prompts of running requests lie in the cache's blocks
    assert S.cache_and_budget(10, w) == (1, 512)
    with pytest.raises(ValueError):
        S.cache_and_budget(9, w)
