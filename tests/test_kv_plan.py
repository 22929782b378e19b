"""fk_kv_plan: the form, tiles and splits that fk_kv_attend takes, as text, and what it refuses; what the other calls of the 4-bit cache refuse
beside test_kv_refusals.py.  No kernel is launched here."""
import ctypes
import re

import pytest
import torch

from paper_2603_09229_amd import binding as fk
from tests.test_kv_refusals import EINVAL, EUNSUPPORTED, attend, cache


def plan(c=None, heads=32, B=1, max_q=1, max_len=1000, window=0, room=256):
    buf = ctypes.create_string_buffer(b"?" * room, room)
    status = fk.lib().fk_kv_plan(ctypes.byref(c or cache(k_codes=None, k_levels=None)), heads, B, max_q, max_len, window, buf, room)
    return status, buf.value.decode()


def test_forms():
    assert plan()[1].startswith("rows_shared(tiles=1,row_blocks=1,splits=1,chunk=0)")
    assert re.match(r"rows_shared\(tiles=1,row_blocks=1,splits=(\d\d),chunk=\d+\)", plan(max_len=100000)[1])
    assert "splits=1," in plan(max_len=100000, window=500)[1]
    assert plan(B=8, max_q=1024, max_len=4096)[1].startswith("rows_own(tiles=3,row_blocks=86,waves=4)")
    assert plan(B=32, max_q=25, max_len=4096)[1].startswith("rows_own(tiles=3,row_blocks=3,waves=4,packed)")
    assert plan(B=500, max_len=20)[1].startswith("rows_own(tiles=1,row_blocks=1,waves=8,packed)")
    assert plan(c=cache(d=256), B=8, max_q=1024, max_len=4096)[1].startswith("rows_own(tiles=1,row_blocks=256,waves=8)")


@pytest.mark.parametrize("B,max_q,max_len", [(1, 1, 1), (1, 1, 1 << 30), (65535, 1, 77), (3, 1 << 27, 1 << 30), (64, 5, 8192), (255, 1, 100000)])
@pytest.mark.parametrize("d", [32, 96, 128, 256])
def test_the_workspace_is_the_one_asked_for(B, max_q, max_len, d):
    c = cache(d=d)
    status, text = plan(c, 32, B, max_q, max_len)
    assert status == 0 and int(text.rsplit("=", 1)[1]) == fk.lib().fk_kv_workspace_bytes(ctypes.byref(c), 32, 1, B, max_q, max_len)


@pytest.mark.parametrize("other,status", [
    (dict(heads=12), EINVAL), (dict(B=0), EINVAL), (dict(max_q=0), EINVAL), (dict(max_len=0), EINVAL), (dict(window=-1), EINVAL),
    (dict(B=70000), EUNSUPPORTED), (dict(max_len=1 << 31), EUNSUPPORTED), (dict(c=cache(d=40)), EUNSUPPORTED),
])
def test_what_is_refused(other, status):
    assert plan(**other) == (status, "unsupported")


def test_the_text_is_cut_to_the_buffer():
    assert plan(room=9) == (0, "rows_sha") and plan(room=1) == (0, "")
    assert fk.lib().fk_kv_plan(ctypes.byref(cache()), 32, 1, 1, 100, 0, None, 5) == EINVAL
    assert fk.lib().fk_kv_plan(None, 32, 1, 1, 100, 0, ctypes.create_string_buffer(8), 8) == EINVAL


@pytest.mark.parametrize("other,word", [(dict(max_len=0), b"max_len"), (dict(B=0), b"positive"), (dict(max_len=1 << 31), b"max_len")])
def test_a_workspace_of_nothing_says_why(other, word):
    fk.lib().fk_kv_read(None, None, 0, None, None, None)              # an error of another call
    a = dict(heads=32, Tq=1, B=1, max_q=1, max_len=100)
    a.update(other)
    assert fk.lib().fk_kv_workspace_bytes(ctypes.byref(cache()), *a.values()) == 0
    assert b"fk_kv_workspace_bytes" in fk.lib().fk_last_error() and word in fk.lib().fk_last_error()


@pytest.mark.parametrize("scale", [float("nan"), float("inf"), -float("inf"), 3e38])
def test_scales_that_are_no_numbers(scale):
    assert attend(scale=scale, window=0) == EINVAL and b"scale" in fk.lib().fk_last_error()
    assert attend(scale=-1e38, q=None) == EINVAL and b" q is NULL" in fk.lib().fk_last_error()      # past that check


@pytest.mark.parametrize("d", range(32, 257, 32))
def test_one_workspace_is_enough_for_any_call(d):
    """256 (d + 2) bytes a compute unit (256 of them) and 512; a smaller batch may need more than a larger one."""
    for H in (1, 3, 8, 64, 256):
        c = cache(heads=H, d=d)
        for G in (1, 4, 16, 100):
            for B in (1, 2, 3, 9, 31, 64, 127, 255, 1000):
                for max_q in (1, 5, 64, 1000):
                    for max_len in (1, 700, 5000, 131072, 1 << 30):
                        assert 0 < fk.lib().fk_kv_workspace_bytes(ctypes.byref(c), H * G, 1, B, max_q, max_len) <= 256 * 256 * (d + 2) + 512
    need = lambda B: fk.lib().fk_kv_workspace_bytes(ctypes.byref(cache(d=d)), 32, B, B, 1, 8192)
    assert need(1) > need(64)


def test_a_page_beyond_32_bits_is_not_cut():
    """2^32 + 64 tokens a page are not a page of 64 (sizes alone: nothing is allocated)."""
    codes, scale = torch.empty(1, 1, 2 ** 32 + 64, 16, dtype=torch.uint8, device="meta"), torch.empty(1, 1, 2 ** 32 + 64, dtype=torch.float16, device="meta")
    levels = torch.empty(1, 16, dtype=torch.float16, device="meta")
    with pytest.raises(ValueError, match="page_size=4294967360 is beyond 32 bits"):
        fk.KVCache(codes, codes, scale, scale, levels, levels)
