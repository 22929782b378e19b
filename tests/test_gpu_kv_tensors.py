"""KVCache over tensors that its owner replaces or moves: calls go where the tensors are, and tensors that do not fit are refused."""
import pytest
import torch

from paper_2603_09229_amd import binding as fk
from tests import kv_plain

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
NAMES = ("k_codes", "v_codes", "k_scale", "v_scale", "k_levels", "v_levels")


def make():
    lv = [kv_plain.levels(2, torch.float16, s, DEV) for s in (1, 2)]
    cache = fk.KVCache.empty(3, 16, *lv, 64)
    x = torch.randn(20, 2, 64, device=DEV).half()
    fk.fk_kv_append(cache, x, x, torch.arange(20, device=DEV))
    return cache, x


def results(cache):
    slots = torch.arange(20, device=DEV)
    q = torch.ones(1, 4, 64, device=DEV, dtype=torch.float16)
    pages = torch.tensor([[0, 1]], dtype=torch.int32, device=DEV)
    return (*fk.fk_kv_read(cache, slots), fk.fk_kv_attend(cache, q, pages, torch.tensor([20], dtype=torch.int32, device=DEV)))


@pytest.mark.parametrize("name", NAMES)
def test_a_tensor_that_is_replaced(name):
    cache, x = make()
    old, want = getattr(cache, name), results(cache)
    new = old.clone()
    setattr(cache, name, new)
    old.fill_(0)                                                      # no longer read
    assert all(torch.equal(a, b) for a, b in zip(results(cache), want))
    new.fill_(1)
    was = old.clone()
    fk.fk_kv_append(cache, x, x, torch.arange(20, device=DEV))
    assert torch.equal(old, was) and (name.endswith("levels") or not (new == 1).all())


@pytest.mark.parametrize("name", NAMES)
def test_a_tensor_that_moves(name):
    cache, _ = make()
    want = results(cache)
    getattr(cache, name).set_(getattr(cache, name).clone())
    assert all(torch.equal(a, b) for a, b in zip(results(cache), want))


def test_more_pages():
    cache, x = make()
    want = results(cache)
    for name in NAMES[:4]:
        old = getattr(cache, name)
        setattr(cache, name, torch.cat([old, torch.zeros_like(old)]))
    assert all(torch.equal(a, b) for a, b in zip(results(cache), want)) and cache.pages == 6
    fk.fk_kv_append(cache, x, x, torch.arange(70, 90, device=DEV))
    assert cache.k_scale[4:].any()


@pytest.mark.parametrize("name", NAMES)
def test_tensors_that_do_not_fit(name):
    cache, x = make()
    good = getattr(cache, name)
    for bad in (good[:1], good.cpu(), good.int(), torch.stack([good, good], -1)[..., 0]):
        setattr(cache, name, bad)
        with pytest.raises(ValueError):
            results(cache)
        with pytest.raises(ValueError):
            fk.fk_kv_append(cache, x, x, torch.arange(20, device=DEV))
        with pytest.raises(ValueError):
            fk.fk_kv_workspace_bytes(cache, 1, 4, 1, 1, 20)
    setattr(cache, name, good)
    results(cache)
