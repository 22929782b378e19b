"""fk_kv_attend on many short sequences, whose waves have sequences of their own: numbers of sequences around a workgroup's waves, none to several
tiles of rows each, empty ones among them.  Inputs, comparison and tolerance as in test_gpu_kv_attend.py."""
import pytest
import torch

from tests.test_gpu_kv_attend import BF16, F16, run

pytestmark = pytest.mark.gpu


def ragged(B, most, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(0, most + 1, (B,), generator=g).tolist()


@pytest.mark.parametrize("t", [F16, BF16])
@pytest.mark.parametrize("d", [32, 64, 96, 128, 160, 192, 224, 256])
def test_every_width(t, d):
    run(t, ragged(19, 60, d), [1] * 19, 3, 4, d, 16, seed=d)


@pytest.mark.parametrize("B", [1, 2, 7, 8, 9, 15, 16, 17, 63])
@pytest.mark.parametrize("most", [1, 33, 64])
def test_numbers_of_sequences(B, most):
    run(F16, [most] + ragged(B - 1, most, B), [1] * B, 2, 3, 64, 32, seed=B + most)


@pytest.mark.parametrize("G", [1, 16, 17, 40, 100, 120, 130])
@pytest.mark.parametrize("window", [0, 5])
def test_tiles_of_a_sequence(G, window):
    run(BF16, ragged(11, 50, G), [1] * 11, 2, G, 64, 16, window=window, seed=G)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d", [64, 128, 256])
def test_several_queries_each(causal, d):
    queries = ragged(13, 9, 3)
    lens = [max(n, 2 * n + 11) if n else 0 for n in queries]
    run(F16, lens, queries, 2, 4, d, 16, causal=causal, seed=d)
    run(BF16, [40] * 10, [9, 0, 1, 40, 2, 3, 17, 8, 33, 5], 2, 4, d, 16, causal=causal, seed=d + 1)
