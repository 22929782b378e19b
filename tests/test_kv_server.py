"""What kv_cache.Server and learn_levels refuse, before it touches the device: no kernel is launched here and no tensor is on a GPU."""
import pytest
import torch

from paper_2603_09229_amd import kv_cache


def server(held, max_len=20):
    s = object.__new__(kv_cache.Server)
    s.lens, s.max_len = torch.tensor(held, dtype=torch.int32), max_len
    return s


def rows(*T):
    return [torch.zeros(t, 2, 32) for t in T]


@pytest.mark.parametrize("held,counts", [
    ([0, 0], [21, 0]), ([20, 3], [1, 1]), ([3, 19], [0, 2]), ([20, 20], [1, 0]),        # (a page holds 16: 32 would still have a place)
])
def test_a_sequence_that_would_pass_its_room(held, counts):
    s = server(held)
    with pytest.raises(ValueError, match="more than 20 tokens"):
        s.step(*rows(*[sum(counts)] * 3), counts)
    assert s.lens.tolist() == held


@pytest.mark.parametrize("counts,T", [([1], (1, 1, 1)), ([1, 1, 1], (3, 3, 3)), ([2, -1], (1, 1, 1)), ([1, 1], (3, 3, 3)), ([1, 1], (2, 1, 2)),
                                      ([1, 1], (2, 2, 3)), ([], (0, 0, 0))])
def test_counts_that_are_not_those_of_the_rows(counts, T):
    with pytest.raises(ValueError, match="counts"):
        server([0, 0]).step(*rows(*T), counts)


def test_a_step_without_tokens_is_over_at_once():
    s = server([5, 20])
    assert s.step(*rows(0, 0, 0), [0, 0]).shape == (0, 2, 32) and s.lens.tolist() == [5, 20]


@pytest.mark.parametrize("batch,max_len", [(0, 10), (3, 0), (2, -5)])
def test_no_room_at_all(batch, max_len):
    with pytest.raises(ValueError, match="positive"):
        kv_cache.Server(torch.zeros(1, 16), torch.zeros(1, 16), 64, batch, max_len)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_levels_are_not_learned_from_rows_that_are_not_finite(dtype, bad):
    rows = torch.randn(50, 2, 32).to(dtype)
    rows[49, 1, 31] = bad
    with pytest.raises(ValueError, match="finite"):
        kv_cache.learn_levels(rows)


def test_levels_are_not_learned_from_nothing():
    with pytest.raises(ValueError, match="at least one row"):
        kv_cache.learn_levels(torch.zeros(0, 2, 32, dtype=torch.float16))
