"""fk_kv_choose with its counts where the lengths are: workgroups of other heads would read lengths that the first has cut down.  Refused on the
host; no kernel is launched here."""
import pytest

from paper_2603_09229_amd import binding as fk
from tests.test_kv_evict_refusals import choose
from tests.test_kv_refusals import EINVAL, P


@pytest.mark.parametrize("counts", [4096, 4096 + 4, 4096 + 12, 4096 - 4, 4096 - 12])
def test_counts_on_top_of_lengths(counts):
    assert choose(lens=4096, counts=counts, ws=None) == EINVAL and b"counts" in fk.lib().fk_last_error()


@pytest.mark.parametrize("counts", [4096 + 16, 4096 - 16])
def test_counts_beside_lengths(counts):
    # (4 sequences; max_len in parts, so that the missing workspace is what ends the call)
    assert choose(lens=4096, counts=counts, B=4, max_pages=1 << 12, max_len=1 << 18, ws=P + 1) == EINVAL
    assert b"ws" in fk.lib().fk_last_error()
