"""How many tensors kv_cache.Server.step makes beside its calls of the library: where nothing can be evicted, positions are places, and a step makes
no more than that takes.  The calls of the library are left out, so that no kernel is launched here."""
import pytest
import torch
from torch.utils._python_dispatch import TorchDispatchMode

from paper_2603_09229_amd import kv_cache
from tests.test_kv_server import rows, server


class Count(TorchDispatchMode):
    def __init__(self):
        super().__init__()
        self.names = []

    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        name = func.overloadpacket.__name__
        if not any(r.alias_info and not r.alias_info.is_write for r in func._schema.returns):   # views launch nothing
            self.names.append(name)
        return func(*args, **(kwargs or {}))


@pytest.mark.parametrize("weights", [False, True])
def test_a_step_without_evictions(monkeypatch, weights):
    s = server([5, 3])
    s.max_pos, s.gone, s.cos_sin = 40, torch.tensor([0, 4 if weights else 0], dtype=torch.int32), None
    s.pages = torch.tensor([[0, 2], [1, 3]], dtype=torch.int32)
    s.cache = type("Cache", (), {"page_size": 16})
    s.mass = torch.zeros(1) if weights else None
    got = {}

    def append(cache, k, v, slots, positions, cos_sin, q):
        got.update(slots=slots, positions=positions)
        return q
    monkeypatch.setattr(kv_cache.fk, "fk_kv_append", append)
    monkeypatch.setattr(kv_cache.fk, "fk_kv_attend", lambda cache, q, *args, lse, **named: (q, None) if lse else q)
    monkeypatch.setattr(kv_cache.fk, "fk_kv_weigh", lambda *args, **named: None)
    x = rows(5, 5, 5)
    with Count() as count:
        s.step(*x, [2, 3])
    assert got["slots"].tolist() == [5, 6, 19, 20, 21] and s.lens.tolist() == [7, 6]
    assert got["positions"].dtype == torch.int32 and got["positions"].tolist() == ([5, 6, 7, 8, 9] if weights else [5, 6, 3, 4, 5])
    # Lengths and what is gone (1); starts (zeros, sum, copy: 3); sequences (arange, repetition, which looks up: 3); places (length, arange, sum, start,
    # difference: 5); slots (quotient, widened, page, widened, product, remainder, sum: 7); new lengths (difference of starts, sum: 2).  With weights:
    # lengths before, and positions (what is gone of each token, sum: 2).
    assert len(count.names) <= 21 + (3 if weights else 0), " ".join(count.names)
