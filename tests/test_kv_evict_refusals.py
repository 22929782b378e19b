"""What the calls that draft on the 4-bit key/value cache and keep it small refuse, all of it on the host before the first HIP call.  No kernel
is launched here."""
import ctypes

import pytest
import torch

from paper_2603_09229_amd import binding as fk
from tests.test_kv_refusals import EINVAL, EUNSUPPORTED, EWORKSPACE, P, cache


def call(name, a, other, c=None):
    a = dict(a)
    assert set(other) <= set(a)
    a.update(other)
    return getattr(fk.lib(), name)(ctypes.byref(c or cache()), *a.values(), None)


def tree(c=None, **other):
    return call("fk_kv_attend_tree", dict(q=P, qt=4096, qh=128, heads=32, Tq=20, pages=P, max_pages=3, lens=P, q_start=None, B=4, max_q=5,
                                          max_len=100, scale=1.0, window=0, tree=P, words=1, out=P, lse=None, ws=P, room=1 << 30), other, c)


def weigh(c=None, **other):
    return call("fk_kv_weigh", dict(q=P, qt=4096, qh=128, heads=32, Tq=4, lse=P, pages=P, max_pages=3, lens=P, q_start=None, B=4, max_q=1,
                                    max_len=100, scale=1.0, causal=1, window=0, known=None, decay=1.0, mass=P, out=P, ws=P, room=1 << 30), other, c)


def choose(c=None, **other):
    return call("fk_kv_choose", dict(mass=P, pages=P, max_pages=3, lens=P, B=4, max_len=100, keep=50, first=4, last=10, kept=P, counts=P,
                                     ws=P, room=1 << 30), other, c)


def compact(c=None, **other):
    return call("fk_kv_compact", dict(pages=P, max_pages=3, kept=P, kept_heads=8, max_kept=20, counts=P, start=None, to=None, to_max=0, B=4,
                                      mass=None), other, c)


@pytest.mark.parametrize("other,status", [
    (dict(t=fk.FK_F32), EUNSUPPORTED), (dict(t=7), EINVAL), (dict(pages=0), EINVAL), (dict(page_size=48), EUNSUPPORTED),
    (dict(heads=0), EINVAL), (dict(heads=257), EUNSUPPORTED), (dict(d=100), EUNSUPPORTED), (dict(k_codes=None), EINVAL),
    (dict(v_codes=8), EINVAL), (dict(k_scale=None), EINVAL), (dict(k_levels=None), EINVAL),
])
def test_caches_that_are_refused(other, status):
    c = cache(**other)
    assert tree(c, window=-1) == status and weigh(c, window=-1) == status and choose(c, keep=0) == status and compact(c, max_kept=-1) == status
    assert fk.lib().fk_last_error()


QUERIES = [
    (dict(heads=0), EINVAL), (dict(heads=12), EINVAL), (dict(B=0), EINVAL), (dict(max_q=0), EINVAL), (dict(Tq=-1), EINVAL), (dict(Tq=3), EINVAL),
    (dict(max_len=-1), EINVAL), (dict(max_pages=0), EINVAL), (dict(window=-1), EINVAL), (dict(max_pages=1 << 26), EUNSUPPORTED),
    (dict(max_len=1 << 31), EUNSUPPORTED), (dict(q=None), EINVAL), (dict(q=P + 1), EINVAL), (dict(pages=None), EINVAL), (dict(lens=None), EINVAL),
    (dict(q_start=P + 2), EINVAL), (dict(out=None), EINVAL), (dict(scale=float("inf")), EINVAL), (dict(scale=float("nan")), EINVAL),
    (dict(scale=2e38), EINVAL),
]


@pytest.mark.parametrize("other,status", QUERIES + [
    (dict(out=P + 4), EINVAL), (dict(lse=P + 2), EINVAL), (dict(ws=None), EINVAL), (dict(ws=P + 16), EINVAL), (dict(words=0), EINVAL),
    (dict(words=-1), EINVAL), (dict(max_q=65, Tq=260), EINVAL), (dict(max_q=129, Tq=516, words=2), EINVAL), (dict(tree=None), EINVAL),
    (dict(tree=P + 4), EINVAL), (dict(words=1 << 29, Tq=20), EUNSUPPORTED), (dict(B=1, max_q=1 << 25, Tq=1 << 25, words=1 << 19), EUNSUPPORTED),
    (dict(B=70000, Tq=350000), EUNSUPPORTED), (dict(room=64, max_len=60000), EWORKSPACE),
])
def test_trees_that_are_refused(other, status):
    assert tree(**other) == status


@pytest.mark.parametrize("other,status", QUERIES + [
    (dict(lse=None), EINVAL), (dict(lse=P + 2), EINVAL), (dict(known=P + 1), EINVAL), (dict(mass=None), EINVAL), (dict(mass=P + 2), EINVAL),
    (dict(out=P + 2), EINVAL), (dict(decay=float("nan")), EINVAL), (dict(decay=float("-inf")), EINVAL), (dict(B=70000, Tq=70000), EUNSUPPORTED),
    (dict(max_q=1000, Tq=4000, ws=None), EINVAL), (dict(max_q=1000, Tq=4000, ws=P + 128), EINVAL), (dict(max_q=1000, Tq=4000, room=64), EWORKSPACE),
])
def test_weights_that_are_refused(other, status):
    assert weigh(**other) == status


def test_more_workgroups_than_a_launch_has():
    big = cache(heads=256, d=32)
    assert weigh(big, heads=256, B=65535, Tq=65535, max_pages=1 << 20, max_len=1 << 20) == EUNSUPPORTED and b"workgroups" in fk.lib().fk_last_error()


@pytest.mark.parametrize("other,status", [
    (dict(keep=0), EINVAL), (dict(keep=-5), EINVAL), (dict(first=-1), EINVAL), (dict(last=-1), EINVAL), (dict(first=41), EINVAL),
    (dict(first=2 ** 31 - 1, last=2 ** 31 - 1), EINVAL), (dict(max_len=-1), EINVAL), (dict(B=0), EINVAL), (dict(B=70000), EUNSUPPORTED),
    (dict(max_pages=0), EINVAL), (dict(max_pages=1 << 26), EUNSUPPORTED), (dict(keep=(1 << 30) + 1), EUNSUPPORTED),
    (dict(max_len=1 << 31), EUNSUPPORTED), (dict(mass=None), EINVAL), (dict(mass=P + 2), EINVAL), (dict(pages=None), EINVAL),
    (dict(lens=P + 2), EINVAL), (dict(kept=None), EINVAL), (dict(counts=None), EINVAL), (dict(kept=P + 1), EINVAL),
])
def test_choices_that_are_refused(other, status):
    assert choose(**other) == status


@pytest.mark.parametrize("other,status", [
    (dict(max_kept=-1), EINVAL), (dict(kept_heads=0), EINVAL), (dict(kept_heads=2), EINVAL), (dict(max_kept=(1 << 30) + 1), EUNSUPPORTED),
    (dict(B=0), EINVAL), (dict(B=1 << 16), EUNSUPPORTED), (dict(max_pages=0), EINVAL), (dict(max_pages=1 << 26), EUNSUPPORTED),
    (dict(to=P + 64, to_max=0), EINVAL), (dict(to=P + 64, to_max=1 << 26), EUNSUPPORTED), (dict(to=P + 2, to_max=3), EINVAL),
    (dict(pages=None), EINVAL), (dict(kept=None), EINVAL), (dict(counts=P + 2), EINVAL), (dict(start=P + 1), EINVAL), (dict(mass=P + 2), EINVAL),
])
def test_compactions_that_are_refused(other, status):
    assert compact(**other) == status


def test_calls_without_work_are_done_at_once():
    assert tree(Tq=0, q_start=P, q=None, out=None) == 0
    assert compact(max_kept=0, kept=None, counts=None) == 0


def test_no_cache_at_all():
    L = fk.lib()
    assert L.fk_kv_compact(None, P, 3, P, 8, 20, P, None, None, 0, 4, None, None) == EINVAL and b"NULL" in L.fk_last_error()
    assert L.fk_kv_choose_workspace_bytes(None, 1, 100) == 0


def test_the_binding_refuses_integers_beyond_32_bits_before_it_looks_at_tensors():
    class Cache:
        heads, d, pages, page_size, device, dtype, _index = 2, 64, 3, 16, "cpu", torch.float16, -1

        def _here(self):
            return None
    z = torch.zeros(1, 3, dtype=torch.int32)
    for bad in (dict(keep=1 << 31), dict(keep=5, first=1 << 40), dict(keep=5, last=-1 << 40)):
        with pytest.raises(ValueError):
            fk.fk_kv_choose(Cache(), None, z, z[:, 0], **bad)
    q = torch.zeros(1, 4, 64, dtype=torch.float16)
    for bad in (dict(max_q=1 << 32), dict(max_q=-1 << 40), dict(max_q=1, window=-1 << 40)):
        with pytest.raises(ValueError):
            fk.fk_kv_weigh(Cache(), q, None, z, z[:, 0], None, **bad)
        with pytest.raises(ValueError):
            fk.fk_kv_attend_tree(Cache(), q, z, z[:, 0], torch.zeros(1, 1, dtype=torch.int64), **bad)


def test_workspaces():
    L, c = fk.lib(), ctypes.byref(cache(k_codes=None, k_levels=None))
    weigh_bytes = lambda heads=32, Tq=1, B=1, max_q=1, max_len=1000: L.fk_kv_weigh_workspace_bytes(c, heads, Tq, B, max_q, max_len)  # noqa: E731
    assert weigh_bytes() == 0 and weigh_bytes(max_len=1 << 30) == 0                     # few rows are not divided
    assert weigh_bytes(max_q=2000, Tq=2000) > 0
    for bad in (dict(heads=12), dict(max_len=0), dict(B=0), dict(max_q=0), dict(max_len=1 << 31)):
        assert weigh_bytes(**bad) == 0 and L.fk_last_error()
    choose_bytes = lambda B, max_len: L.fk_kv_choose_workspace_bytes(c, B, max_len)     # noqa: E731
    assert choose_bytes(1, 16384) == 0 and choose_bytes(1, 16385) > 0 and choose_bytes(4096, 1 << 20) == 0
    for bad in ((0, 100), (70000, 100), (1, 0), (1, 1 << 31)):
        assert choose_bytes(*bad) == 0 and L.fk_last_error()
    for B in (1, 2, 7, 30, 63, 64, 65, 1000, 65535):
        sizes = [choose_bytes(B, n) for n in (1, 16384, 16385, 33000, 66000, 200000, 1 << 20, 1 << 24, 1 << 30)]
        assert all(a <= b and b % 256 == 0 for a, b in zip(sizes, sizes[1:])) and sizes[-1] < 1 << 26
        for max_q in (1, 33, 500, 4096, 1 << 20):
            for n in (1, 100, 5000, 1 << 20, 1 << 30):
                size = weigh_bytes(Tq=min(B * max_q, 1 << 30), B=B, max_q=max_q, max_len=n)
                assert size % 256 == 0 and size < 1 << 26             # at most 64 parts of what fills the chip four times
