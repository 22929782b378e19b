"""Which positions kv_cache.Server gives out after evictions, when it refuses the next ones, and that nothing changes where it does.  No kernel is
launched here."""
import pytest
import torch

from paper_2603_09229_amd import kv_cache
from tests.test_kv_server import rows, server


def evicted(held, gone, max_len=20, max_pos=20):
    s = server(held, max_len)
    s.max_pos, s.gone = max_pos, torch.tensor(gone, dtype=torch.int32)
    return s


@pytest.mark.parametrize("max_pos", [20, 21, 30])
def test_positions_end_at_max_pos_whether_it_is_max_len_or_more(max_pos):
    for held, gone in (([5, 3], [max_pos - 7, 0]), ([3, 5], [1000, max_pos - 5]), ([0, 0], [max_pos - 2, 0])):
        s = evicted(held, gone, max_pos=max_pos)
        for call in (lambda: s.step(*rows(3, 3, 3), [3, 0]), lambda: s.draft(*rows(3, 3, 3), [[-1, 0, 1], []])):
            with pytest.raises(ValueError, match=rf"sequences \[0\S* would pass position {max_pos}"):
                call()
            assert s.lens.tolist() == held and s.gone.tolist() == gone and s._draft is None


def test_the_last_position_is_given_out():
    s = evicted([5, 3], [13, 0])
    s._check(*rows(5, 5, 5), [2, 3])                              # up to position 19 of 20
    with pytest.raises(ValueError, match=r"sequences \[0\] would pass position 20"):
        s._check(*rows(6, 6, 6), [3, 3])
