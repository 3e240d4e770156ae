"""Token log-probabilities of rows that the usual ones do not show: blocks of NaN.

Tolerances as in test_gpu_logprob.py, whose plain forms these tests use."""
import pytest
import torch

from tests.test_gpu_logprob import check, rows, tokens

pytestmark = pytest.mark.gpu


def blocks_of_nan(n, V, dtype, seed):
    """Rows with NaN in their first half, their first 2048 columns, alternate blocks of 1024, the first two
    entries of each eight, and all but the last five."""
    x = rows(n, V, 0, dtype, seed).clone()
    v = torch.arange(V, device="cuda")
    for i in range(0, n, 5):
        x[i, : V // 2] = float("nan")
        x[i + 1, : min(2048, V - 9)] = float("nan")
        x[i + 2, v // 1024 % 2 == 0] = float("nan")
        x[i + 3, v % 8 < 2] = float("nan")
        x[i + 4, : V - 5] = float("nan")
    return x


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V", [(5, 700), (5, 8192), (5, 50000), (600, 20000), (1100, 5003)])
@pytest.mark.parametrize("m", [1, 9, 16])
def test_blocks_of_nan_rank_last(dtype, n, V, m):
    """A row in several pieces, in one of four waves, in one of one wave."""
    check(blocks_of_nan(n, V, dtype, V + m), tokens(n, V, m), m, 1.0)
