"""What the calls of the 4-bit key/value cache refuse, all of it on the host before the first HIP call, and the size of the
workspace.  No kernel is launched here."""
import ctypes

import pytest
import torch

from paper_2603_09229_amd import binding as fk

EINVAL, EUNSUPPORTED, EWORKSPACE = 1, 2, 3
P = 256                                          # an aligned address that is never dereferenced


def cache(**other):
    f = dict(k_codes=P, v_codes=P, k_scale=P, v_scale=P, k_levels=P, v_levels=P, pages=10, page_size=64, heads=8, d=128, t=fk.FK_F16)
    f.update(other)
    return fk._KVCacheStruct(**f)


def append(c=None, **other):
    a = dict(k=P, kt=1024, kh=128, v=P, vt=1024, vh=128, slots=P, T=5, cs=P, pos=P, max_pos=100, rot=128, inter=0, q=None, qt=0, qh=0,
             heads=0, q_out=None)
    a.update(other)
    return fk.lib().fk_kv_append(ctypes.byref(c or cache()), *a.values(), None)


def attend(c=None, **other):
    a = dict(q=P, qt=4096, qh=128, heads=32, Tq=4, pages=P, max_pages=3, lens=P, q_start=None, B=4, max_q=1, max_len=100, scale=1.0,
             causal=1, window=0, out=P, lse=None, ws=P, room=1 << 30)
    a.update(other)
    return fk.lib().fk_kv_attend(ctypes.byref(c or cache()), *a.values(), None)


def read(c=None, **other):
    a = dict(slots=P, T=5, k=P, v=P)
    a.update(other)
    return fk.lib().fk_kv_read(ctypes.byref(c or cache()), *a.values(), None)


# q without q_out is refused last of the cache's checks, so that a sound cache does not reach a launch either
@pytest.mark.parametrize("other,status", [
    (dict(t=fk.FK_F32), EUNSUPPORTED), (dict(t=7), EINVAL), (dict(pages=0), EINVAL), (dict(pages=1 << 31), EUNSUPPORTED),
    (dict(page_size=0), EINVAL), (dict(page_size=8), EUNSUPPORTED), (dict(page_size=48), EUNSUPPORTED),
    (dict(page_size=1 << 17), EUNSUPPORTED), (dict(heads=0), EINVAL), (dict(heads=257), EUNSUPPORTED), (dict(d=0), EINVAL),
    (dict(d=100), EUNSUPPORTED), (dict(d=288), EUNSUPPORTED), (dict(k_codes=None), EINVAL), (dict(v_codes=8), EINVAL),
    (dict(k_scale=None), EINVAL), (dict(v_scale=2), EINVAL), (dict(k_levels=None), EINVAL), (dict(v_levels=4), EINVAL),
])
def test_caches_that_are_refused(other, status):
    c = cache(**other)
    assert append(c, q=P) == status and read(c, T=-1) == status and attend(c, window=-1) == status
    assert fk.lib().fk_last_error()


@pytest.mark.parametrize("other,status", [
    (dict(T=-1), EINVAL), (dict(T=1 << 31), EUNSUPPORTED), (dict(rot=-16), EINVAL), (dict(rot=144), EINVAL), (dict(rot=24), EUNSUPPORTED),
    (dict(k=None), EINVAL), (dict(k=P + 1), EINVAL), (dict(v=None), EINVAL), (dict(slots=None), EINVAL), (dict(slots=P + 4), EINVAL),
    (dict(cs=None), EINVAL), (dict(cs=P + 4), EINVAL), (dict(pos=None), EINVAL), (dict(max_pos=0), EINVAL), (dict(q=P), EINVAL),
    (dict(q_out=P, heads=4), EINVAL), (dict(q=P, q_out=P, heads=0), EINVAL), (dict(q=P, q_out=P + 8, heads=4), EINVAL),
    (dict(q=P, q_out=P, heads=1 << 17), EUNSUPPORTED),
])
def test_appends_that_are_refused(other, status):
    assert append(**other) == status


@pytest.mark.parametrize("other,status", [
    (dict(T=-1), EINVAL), (dict(T=1 << 31), EUNSUPPORTED), (dict(slots=None), EINVAL), (dict(slots=P + 4), EINVAL),
    (dict(k=P + 8), EINVAL), (dict(v=P + 2), EINVAL),
])
def test_reads_that_are_refused(other, status):
    assert read(**other) == status


@pytest.mark.parametrize("other,status", [
    (dict(heads=0), EINVAL), (dict(heads=12), EINVAL), (dict(B=0), EINVAL), (dict(max_q=0), EINVAL), (dict(Tq=-1), EINVAL),
    (dict(Tq=5), EINVAL), (dict(max_len=-1), EINVAL), (dict(max_pages=0), EINVAL), (dict(window=-1), EINVAL),
    (dict(B=70000, Tq=70000), EUNSUPPORTED), (dict(max_pages=1 << 26), EUNSUPPORTED), (dict(max_q=1 << 30, Tq=1 << 32), EUNSUPPORTED),
    (dict(max_len=1 << 31), EUNSUPPORTED), (dict(q=None), EINVAL), (dict(q=P + 1), EINVAL), (dict(pages=None), EINVAL),
    (dict(lens=None), EINVAL), (dict(q_start=P + 2), EINVAL), (dict(out=None), EINVAL), (dict(out=P + 4), EINVAL),
    (dict(lse=P + 2), EINVAL), (dict(ws=None), EINVAL), (dict(ws=P + 16), EINVAL), (dict(room=64, max_len=60000), EWORKSPACE),
])
def test_attentions_that_are_refused(other, status):
    assert attend(**other) == status


def test_calls_without_work_are_done_at_once():
    assert append(T=0, k=None, v=None, slots=None, cs=None, pos=None) == 0
    assert read(T=0) == 0 and read(k=None, v=None) == 0
    assert attend(Tq=0, q_start=P, q=None, out=None) == 0


def test_no_cache_at_all():
    L = fk.lib()
    assert L.fk_kv_read(None, P, 5, P, P, None) == EINVAL and b"NULL" in L.fk_last_error()
    assert L.fk_kv_workspace_bytes(None, 8, 1, 1, 1, 100) == 0


def test_workspace():
    def need(c=None, heads=32, Tq=1, B=1, max_q=1, max_len=1000):
        return fk.lib().fk_kv_workspace_bytes(ctypes.byref(c or cache(k_codes=None, k_levels=None)), heads, Tq, B, max_q, max_len)
    assert need() > 0 and need() % 256 == 0
    assert need(max_len=100000) > need(max_len=100)                        # split along the tokens
    assert need(max_len=100000, B=4096, Tq=4096) <= 256                    # more sequences than the chip holds: not split
    assert need(max_len=8192, max_q=8192, Tq=8192, B=64) <= 256
    for bad in (dict(heads=12), dict(max_len=0), dict(B=0), dict(max_q=0), dict(c=cache(d=40))):
        assert need(**bad) == 0
    # what a shorter sequence or a window asks for is never more
    for max_q in (1, 5, 64):
        sizes = [need(max_len=n, max_q=max_q, Tq=max_q) for n in range(1, 70000, 517)]
        assert all(a <= b for a, b in zip(sizes, sizes[1:]))


def test_the_binding_refuses_host_tensors_and_wrong_shapes():
    z = torch.zeros
    t = torch.float16
    with pytest.raises(ValueError):
        fk.KVCache(z(2, 1, 16, 32, dtype=torch.uint8), z(2, 1, 16, 32, dtype=torch.uint8), z(2, 1, 16, dtype=t), z(2, 1, 16, dtype=t),
                   z(1, 16, dtype=t), z(1, 16, dtype=t))
    with pytest.raises(ValueError):
        fk.KVCache(z(2, 16, 32, dtype=torch.uint8), None, z(2, 1, 16, dtype=t), None, None, None)
