"""fk_kv_attend in each of its forms, with the plan asked before every call: waves with rows of their own in several tiles (prompts, chunks),
packed and not, over many steps; many short sequences over several steps.  Inputs, comparison and tolerance as in test_gpu_kv_attend.py."""
import pytest
import torch

from paper_2603_09229_amd import binding as fk
from tests import kv_plain
from tests.test_gpu_kv_attend import BF16, DEV, F16, run

pytestmark = pytest.mark.gpu
WIDTHS = [32, 64, 96, 128, 160, 192, 224, 256]
TILES = {32: 4, 64: 4, 96: 3, 128: 3, 160: 2, 192: 2, 224: 1, 256: 1}
# queries and tokens of sequences: whole prompts, later chunks, none of either, more queries than tokens, one sequence of more than 32 steps
QUERIES = [200, 0, 1, 17, 200, 64, 130, 5, 199, 33, 100]
LENS = [300, 50, 0, 17, 77, 64, 1200, 5, 200, 1000, 131]


def planned(t, lens, queries, H, G, d, P, form, window=0, **other):
    lv = kv_plain.levels(H, t, 1, DEV)
    plan = fk.fk_kv_plan(fk.KVCache.empty(1, P, lv, lv, d), len(lens), H * G, max(queries), max(lens), window)
    assert plan.startswith(form), plan
    run(t, lens, queries, H, G, d, P, window=window, **other)


def own(tiles, blocks):
    waves = 8 if tiles == 1 else 4
    return f"rows_own(tiles={tiles},row_blocks={blocks},waves={waves}{',packed' if blocks < waves else ''})"


@pytest.mark.parametrize("t", [F16, BF16])
@pytest.mark.parametrize("d", WIDTHS)
def test_rows_of_their_own_of_every_width(t, d):
    planned(t, LENS, QUERIES, 8, 3, d, 16, own(TILES[d], -(-600 // (16 * TILES[d]))), seed=d)


@pytest.mark.parametrize("causal,window", [(False, 0), (True, 1), (True, 31), (True, 500), (False, 90), (True, 2 ** 31 - 1)])
@pytest.mark.parametrize("t,d", [(F16, 64), (BF16, 128), (F16, 192), (BF16, 256)])
def test_rows_of_their_own_under_every_mask(t, d, causal, window):
    planned(t, LENS, QUERIES, 8, 3, d, 64, own(TILES[d], -(-600 // (16 * TILES[d]))), causal=causal, window=window, seed=d + window % 97)


@pytest.mark.parametrize("G,n", [(1, 600), (5, 120), (12, 50), (48, 13), (7, 90)])
def test_groups_of_rows_of_their_own(G, n):
    queries = [min(q, n) for q in QUERIES] + [n]
    planned(BF16, LENS + [n], queries, 8, G, 128, 32, own(3, -(-n * G // 48)), seed=G)


@pytest.mark.parametrize("t", [F16, BF16])
@pytest.mark.parametrize("d", WIDTHS)
def test_packed_tiles_of_every_width(t, d):
    n = {4: 40, 3: 40, 2: 30, 1: 30}[TILES[d]]
    g = torch.Generator().manual_seed(d)
    queries = [n] + torch.randint(0, n + 1, (30,), generator=g).tolist() + [n]
    lens = [max(0, q + x) for q, x in zip(queries, torch.randint(-9, 90, (32,), generator=g).tolist())]
    lens[0] = 1100
    planned(t, lens, queries, 8, 3, d, 16, own(TILES[d], -(-3 * n // (16 * TILES[d]))), seed=d + 1)
    planned(t, lens, queries, 8, 3, d, 16, own(TILES[d], -(-3 * n // (16 * TILES[d]))), causal=False, window=40, seed=d + 2)


@pytest.mark.parametrize("t,d", [(F16, 64), (BF16, 64), (F16, 128), (BF16, 32)])
def test_short_sequences_of_several_steps(t, d):
    g = torch.Generator().manual_seed(d)
    lens = [100] + torch.randint(0, 101, (399,), generator=g).tolist()
    planned(t, lens, [1] * 400, 4, 2, d, 16, own(1, 1), seed=d)
    planned(t, lens, [1] * 400, 4, 2, d, 16, own(1, 1), window=60, seed=d + 1)


@pytest.mark.parametrize("G", [112, 120, 130, 200])
def test_single_tiles_of_one_sequence_in_several_waves(G):
    planned(F16, [9, 30, 0, 31], [1] * 4, 8, G, 64, 16, own(1, -(-G // 16)), seed=G)


def test_rows_of_their_own_at_odd_strides_and_scales():
    for scale in (0.0, 3.0, -0.7):
        planned(F16, LENS, QUERIES, 8, 3, 128, 16, own(3, 13), strided=True, scale=scale, seed=4)
