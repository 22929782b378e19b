"""fk_kv_weigh in each of its forms at every width: rows that stay, shared by one, two or four waves, and rows that stream by in several whole blocks one
after the other, divided among workgroups or not (its workspace says which).  Inputs, comparison and tolerance as in test_gpu_kv_weigh.py."""
import pytest
import torch

from paper_2603_09229_amd import binding as fk
from tests import kv_plain
from tests.test_gpu_kv_attend import BF16, DEV, F16
from tests.test_gpu_kv_weigh import run
from tests.test_gpu_kv_weigh_rows import run as rows_that_add_nothing

pytestmark = pytest.mark.gpu
WIDTHS = [32, 64, 96, 128, 160, 192, 224, 256]
KEPT = {32: 512, 64: 256, 96: 128, 128: 128, 160: 64, 192: 64, 224: 64, 256: 64}        # rows that a workgroup keeps
BLOCK = {32: 512, 64: 256, 96: 160, 128: 128, 160: 96, 192: 64, 224: 64, 256: 64}      # and those of a block that streams by
STEP = {d: 512 if d <= 128 else 256 for d in WIDTHS}                                    # tokens of a workgroup's step there


def splits(H, G, d, B, n, L):
    """Workgroups among which the rows are divided."""
    lv = kv_plain.levels(H, F16, 1, DEV)
    size = fk.fk_kv_weigh_workspace_bytes(fk.KVCache.empty(1, 64, lv, lv, d), B, H * G, B * n, n, L)
    return max(1, size // (4 * B * H * -(-L // STEP[d]) * STEP[d]))


def divided(d, less):
    """-> (heads, query heads to each, queries, tokens): rows for five blocks to two workgroups."""
    H, G, L = 8, max(4, BLOCK[d] // 32) - less, 2100
    return H, G, -(-5 * BLOCK[d] * (1024 // (H * -(-L // STEP[d])) + 1) // (2 * G)), L


@pytest.mark.parametrize("t", [F16, BF16])
@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("less", [0, 1])
def test_divided_rows_of_several_blocks(less, d, t):
    """Blocks that follow each other, and a last one that is not whole; groups that divide a block and others."""
    H, G, n, L = divided(d, less)
    for tokens, other in ((L + n, {}), (max(L, n), dict(causal=False)), (max(L, n), dict(window=L // 2))):
        parts = splits(H, G, d, 1, n, tokens)
        assert parts > 1 and 2 * parts * BLOCK[d] < n * G
        run(t, [tokens], [n], H, G, d, 64, seed=d + G, **other)


@pytest.mark.parametrize("t", [F16, BF16])
@pytest.mark.parametrize("d", WIDTHS)
def test_rows_of_several_blocks_that_are_not_divided(d, t):
    G, H, B = 4, 8, 32 if d > 128 else 64
    n, L = 7 * BLOCK[d] // (2 * G) + 3, 1000
    assert n * G > KEPT[d] and splits(H, G, d, B, n, L) == 1
    lens = [L - 90 * (b % 10) for b in range(B)]
    queries = [min(m, max(1, n - 11 * (b % 7))) for b, m in enumerate(lens)]
    queries[0] = n
    run(t, lens, queries, H, G, d, 32, seed=d)
    run(t, lens, queries, H, G, d, 32, causal=False, window=300, seed=d + 1)


@pytest.mark.parametrize("t", [F16, BF16])
@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("tiles", [1, 3, 4, 7, 8, 16])
def test_rows_that_stay(tiles, d, t):
    """Few tokens, so that waves share them and divide the rows, from four tiles on two waves, from eight on four; and many tokens."""
    G = 4
    n = min(KEPT[d], 16 * tiles) // G
    run(t, [300, 5, 77], [n, 2, min(n, 77)], 2, G, d, 16, seed=d + tiles)
    run(t, [300, 40], [n, min(n, 40)], 1, G, d, 16, causal=False, window=25, seed=d + tiles + 1)
    run(t, [700 + 400 * b for b in range(6)], [n] * 6, 8, G, d, 64, seed=d + tiles + 2, known="none")


@pytest.mark.parametrize("d", [64, 128, 192, 256])
def test_one_row_that_adds_nothing_among_blocks_of_others(d):
    """The blocks before and after it are whole ones that all rows see."""
    H, G, n, L = divided(d, 0)
    for dead in ([n // 3], [n - 1], list(range(0, n, max(1, n // 7)))):
        rows_that_add_nothing(BF16 if d % 128 else F16, L + n, n, H, G, d, dead, float("nan"))
