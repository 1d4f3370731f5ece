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
