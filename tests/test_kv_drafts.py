"""kv_cache.tree_masks, and what kv_cache.Server refuses of drafts and evictions before it touches the device: no kernel is launched here."""
import pytest
import torch

from paper_2603_09229_amd import kv_cache
from tests.test_kv_server import rows, server


def test_masks_of_a_tree():
    masks, depths = kv_cache.tree_masks([[-1, 0, 0, 2, -1], [], [-1, 0]])
    assert masks.tolist() == [[0b1], [0b11], [0b101], [0b1101], [0b10000], [0b1], [0b11]] and depths == [0, 1, 1, 2, 0, 0, 1]


def test_masks_of_more_than_64_tokens():
    masks, depths = kv_cache.tree_masks([list(range(-1, 129))])
    assert masks.shape == (130, 3) and depths == list(range(130))
    for i, row in enumerate(masks.tolist()):
        assert sum((x & (1 << 64) - 1) << 64 * w for w, x in enumerate(row)) == (2 << i) - 1
    assert kv_cache.tree_masks([[], []])[0].shape == (0, 1) and kv_cache.tree_masks([[-1] * 64])[0][63].tolist() == [-1 << 63]


@pytest.mark.parametrize("tree", [[0], [-2], [-1, 1], [-1, 2, 0], [-1, -1, 5]])
def test_parents_that_do_not_come_before_their_children(tree):
    with pytest.raises(ValueError, match="before"):
        kv_cache.tree_masks([[-1], tree])
    with pytest.raises(ValueError, match="before"):
        server([0, 0]).draft(*rows(*[1 + len(tree)] * 3), [[-1], tree])


def test_drafts_that_would_pass_the_room():
    s = server([17, 3])
    with pytest.raises(ValueError, match="more than 20 tokens"):
        s.draft(*rows(5, 5, 5), [[-1, 0, 1, -1], [-1]])
    with pytest.raises(ValueError, match="counts"):
        s.draft(*rows(4, 4, 4), [[-1, 0], [-1]])
    s.max_pos, s.gone = 25, torch.tensor([0, 20], dtype=torch.int32)
    with pytest.raises(ValueError, match="position 25"):
        s.draft(*rows(3, 3, 3), [[], [-1, 0, 1]])
    with pytest.raises(ValueError, match="position 25"):
        s.step(*rows(3, 3, 3), [0, 3])
    assert s.draft(*rows(0, 0, 0), [[], []]).shape == (0, 2, 32) and s._draft is None


def test_branches_that_are_none():
    s = server([5, 5])
    with pytest.raises(ValueError, match="no draft"):
        s.accept([[], []])
    s._draft = ([[-1, 0, 0, 1], [-1]], None, None)
    for bad in ([[0]], [[1], []], [[0, 3], []], [[0, 1, 2], []], [[4], []], [[], [0, 0]], [[-1], []]):
        with pytest.raises(ValueError):
            s.accept(bad)
        assert s._draft is not None
    for call in (lambda: s.step(*rows(1, 1, 1), [1, 0]), lambda: s.draft(*rows(1, 1, 1), [[-1], []])):
        with pytest.raises(ValueError, match="accept"):
            call()
    s.accept([[], []])
    assert s._draft is None and s.lens.tolist() == [5, 5]


def test_evictions_without_weights():
    with pytest.raises(ValueError, match="weights=True"):
        server([5, 5]).evict(3)
    s = server([5, 5])
    s.mass, s._draft = torch.zeros(1), ([[-1], []], None, None)
    with pytest.raises(ValueError, match="accept"):
        s.evict(3)


def test_positions_before_the_room():
    with pytest.raises(ValueError, match="max_pos"):
        kv_cache.Server(torch.zeros(1, 16), torch.zeros(1, 16), 64, 2, 20, max_pos=19)
