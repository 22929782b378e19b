"""kv_cache.Server.draft keeps what the trees were, whatever its caller does with the lists until `accept`.  No kernel is launched here."""
import pytest
import torch

from paper_2603_09229_amd import kv_cache
from tests.test_kv_server import rows, server


def test_lists_that_are_used_again_before_accept(monkeypatch):
    s = server([5, 5])
    s._append = lambda q, k, v, counts, depths: (q, torch.tensor([0, 3, 4]))
    s.cache = s.pages = None
    monkeypatch.setattr(kv_cache.fk, "fk_kv_attend_tree", lambda cache, q, *args, **named: q)
    trees = [[-1, 0, 0], [-1]]
    s.draft(*rows(4, 4, 4), trees)
    trees[0][:] = [-1, 0, 1, 2, 3]                                # the next step's
    trees[1].append(0)
    trees.append([-1])
    for bad in ([[0, 1, 2], []], [[], [0, 1]], [[], [], []]):
        with pytest.raises(ValueError):
            s.accept(bad)
    s.accept([[], []])
