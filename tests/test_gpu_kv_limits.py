"""fk_kv_attend at the ends of its ranges: windows as long as the type holds, with more queries than tokens.  Inputs, comparison
and tolerance as in test_gpu_kv_attend.py."""
import pytest
import torch

from tests.test_gpu_kv_attend import BF16, F16, run

pytestmark = pytest.mark.gpu
LAST = 2 ** 31 - 1


# few sequences, whose workgroups share the rows; many short ones, several to a workgroup; more rows than a tile in enough workgroups, a wave each
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window", [LAST, LAST - 1, LAST - 40, 2 ** 30, 2 ** 30 + 1])
def test_the_longest_windows(window, causal):
    run(F16, [2, 33], [40, 90], 2, 2, 64, 16, window=window, causal=causal, seed=31)
    run(BF16, [2, 33, 5000], [5, 1, 9], 1, 4, 128, 16, window=window, causal=causal, seed=32)
    run(BF16, [3, 0, 30] * 40, [5, 2, 1] * 40, 3, 2, 96, 16, window=window, causal=causal, seed=33)
    run(F16, [2, 100, 17, 64] * 8, [70, 100, 40, 20] * 8, 8, 3, 128, 16, window=window, causal=causal, seed=34)
