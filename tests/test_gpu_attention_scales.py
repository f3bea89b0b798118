"""Softmax scales at the ends of what fp32 holds."""
import pytest
import torch

from paper_2511_22972_b200 import ChunkAttention, binding as Bd
from tests._cache import rows
from tests.test_gpu_attention import held, run, stream

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("n", [3, 40])
@pytest.mark.parametrize("scale", [1e-300, 4e-46, 1e-44, 1e-38, 1e-12, 1e-9])
def test_scales_that_leave_nothing_of_the_scores(fmt, n, scale):
    # every row is the mean of the values that it sees, rows of zero queries too
    pool = held([200, 33], n, 2, 64, 16, fmt, seed=7)
    q = rows(2, n, 8, 64, torch.Generator(device="cuda").manual_seed(4))
    q[0, 0] = 0
    q[1, n - 1, 3] = 0
    run(pool, n, 8, scale=scale, q=q, rows_of={0, n - 1})
    run(pool, n, 8, 40, 3, scale=scale, q=q, rows_of={0, n - 1})


@pytest.mark.parametrize("scale", [2.5e38, 1e39, 1e300])
def test_scales_beyond_fp32_are_refused(scale):
    # (a score of 0 times infinity would be NaN)
    pool = held([20], 2, 2, 64)
    q, att = torch.zeros(1, 2, 8, 64, dtype=torch.bfloat16, device="cuda"), ChunkAttention(1, 2, 8, 2, 64)
    with pytest.raises(Bd.FlyError) as e:
        att.run(pool.cache, q, torch.zeros_like(q), scale=scale, stream=stream())
    assert e.value.status == Bd.FLY_ERR_UNSUPPORTED
    run(pool, 2, 8, q=q, scale=2.0 ** 127)
