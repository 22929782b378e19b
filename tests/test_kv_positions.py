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


class Passed(Exception):
    """What a server here does instead of its first launch."""


def test_a_wide_tree_is_measured_by_its_depth():
    """Drafted tokens stand side by side: 60 of them in 3 levels take 60 places, and 3 positions."""
    def launch(*_):
        raise Passed
    tree = [-1] * 20 + list(range(40))
    for gone, refused in (([97, 0], None), ([98, 0], 0), ([0, 97], None), ([0, 98], 1)):
        s = evicted([0, 0], gone, max_len=60, max_pos=100)
        s._append = launch
        trees = [tree, [-1]] if gone[0] else [[-1], tree]
        with pytest.raises(ValueError, match="more than 60 tokens"):
            s.draft(*rows(62, 62, 62), [t + [0] if t is tree else t for t in trees])
        with pytest.raises(Passed) if refused is None else pytest.raises(ValueError, match=rf"sequences \[{refused}\] would pass position 100"):
            s.draft(*rows(61, 61, 61), trees)
