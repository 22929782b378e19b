"""kv_cache.Server where no sequence has a tree this time: `draft` and `accept` as in any other pass of a loop.  No kernel is launched
here."""
import pytest
import torch

from paper_2603_09229_amd import kv_cache
from tests.test_kv_server import rows, server


def test_a_draft_for_no_one_is_accepted():
    s = server([5, 20])
    for _ in range(3):
        assert s.draft(*rows(0, 0, 0), [[], []]).shape == (0, 2, 32)
        for bad, word in ([[0], []], "no branch"), ([[], [-1]], "no branch"), ([[]], "1 branches for 2"):
            with pytest.raises(ValueError, match=word):
                s.accept(bad)
        s.accept([[], []])
        assert s.lens.tolist() == [5, 20]
        with pytest.raises(ValueError, match="no draft"):         # once
            s.accept([[], []])


def test_nothing_waits_for_an_accept_that_has_nothing_to_do():
    s = server([5, 20])
    s.draft(*rows(0, 0, 0), [[], []])
    assert s.step(*rows(0, 0, 0), [0, 0]).shape == (0, 2, 32)     # not held up, and the draft is over
    with pytest.raises(ValueError, match="no draft"):
        s.accept([[], []])
    s.draft(*rows(0, 0, 0), [[], []])
    s.mass = torch.zeros(1)
    with pytest.raises(Exception) as caught:                      # an eviction is not held up either
        s.evict(3)
    assert "accept" not in str(caught.value)
