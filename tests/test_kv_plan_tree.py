"""fk_kv_plan_tree: what fk_kv_attend_tree launches, as text, what it refuses, and that its workspace is never more than the one of fk_kv_attend.  No
kernel is launched here."""
import ctypes

import pytest

from paper_2603_09229_amd import binding as fk
from tests.test_gpu_kv_tree_forms import LONG, MOST, SHARED, WINDOWED
from tests.test_kv_refusals import EINVAL, EUNSUPPORTED, cache


def plan(c=None, heads=32, B=1, max_q=1, max_len=1000, window=0, room=256, call="fk_kv_plan_tree"):
    buf = ctypes.create_string_buffer(b"?" * room, room)
    status = getattr(fk.lib(), call)(ctypes.byref(c or cache(k_codes=None, k_levels=None)), heads, B, max_q, max_len, window, buf, room)
    return status, buf.value.decode()


def test_the_forms_that_are_compared_on_the_gpu():
    for d in MOST:
        assert set(SHARED[d]) == set(LONG[d]) == set(range(1, MOST[d] + 1)) and (MOST[d] == 1 or set(WINDOWED[d]) == set(range(2, MOST[d] + 1)))
        for table, end in ((SHARED, ")"), (LONG, ",longest_first)"), (WINDOWED, ")")):
            for tiles, (H, G, B, n, L, *window) in table.get(d, {}).items():
                text = plan(cache(heads=H, d=d), H * G, B, n, L, *window)[1]
                assert text.startswith(f"rows_shared(tiles={tiles},row_blocks={-(-n * G // (16 * tiles))},splits=1,chunk=0{end} workspace="), (d, tiles, text)


@pytest.mark.parametrize("other,status", [
    (dict(heads=12), EINVAL), (dict(B=0), EINVAL), (dict(max_q=0), EINVAL), (dict(max_len=0), EINVAL), (dict(window=-1), EINVAL),
    (dict(B=70000), EUNSUPPORTED), (dict(max_len=1 << 31), EUNSUPPORTED), (dict(c=cache(d=40)), EUNSUPPORTED),
])
def test_what_is_refused(other, status):
    assert plan(**other) == (status, "unsupported") and b"fk_kv_plan_tree" in fk.lib().fk_last_error()


def test_the_text_is_cut_to_the_buffer():
    assert plan(room=9) == (0, "rows_sha") and plan(room=1) == (0, "")
    assert fk.lib().fk_kv_plan_tree(ctypes.byref(cache()), 32, 1, 1, 100, 0, None, 5) == EINVAL
    assert fk.lib().fk_kv_plan_tree(None, 32, 1, 1, 100, 0, ctypes.create_string_buffer(8), 8) == EINVAL


@pytest.mark.parametrize("d", range(32, 257, 32))
def test_the_workspace_of_queries_in_a_row_is_enough(d):
    for H in (1, 3, 8):
        c = cache(heads=H, d=d)
        for G in (1, 4, 16):
            for B in (1, 2, 9, 31, 100, 255):
                for max_q in (1, 13, 64, 200):
                    for max_len in (1, 700, 5000, 131072, 1 << 30):
                        for window in (0, 1, 300, 4000, 2 ** 31 - 1):
                            status, text = plan(c, H * G, B, max_q, max_len, window)
                            assert status == 0 and int(text.rsplit("=", 1)[1]) <= fk.lib().fk_kv_workspace_bytes(ctypes.byref(c), H * G, 1, B, max_q, max_len)
