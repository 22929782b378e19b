"""fk_kv_attend_tree in each of its forms, with the plan asked before every call: workgroups that share their rows in every number of tiles, with and
without splits, waves with rows of their own, packed and not, and long ragged batches whose longest sequences come first.  Results go where NaN
stood.  Inputs, comparison and tolerance as in test_gpu_kv_tree.py."""
import math
import random

import pytest
import torch

from paper_2603_09229_amd import binding as fk
from tests import evict_plain as plain
from tests import kv_plain
from tests.test_gpu_kv_attend import BF16, DEV, F16, make
from tests.test_gpu_kv_tree import short, trees

pytestmark = pytest.mark.gpu
WIDTHS = [32, 64, 96, 128, 160, 192, 224, 256]
MOST = {32: 4, 64: 4, 96: 3, 128: 3, 160: 2, 192: 2, 224: 1, 256: 1}    # tiles of a wave


def planned(t, lens, queries, H, G, d, form, max_q, max_len, window=0, kind="tree", P=64, seed=0, also=""):
    """A call whose plan begins with `form`, every row of it compared."""
    assert max(queries) <= max_q and max(lens) <= max_len
    cache, q, table, starts = make(t, lens, queries, H, G, d, P, seed, window=window + 1 if window else 0)
    plan = fk.fk_kv_plan_tree(cache, len(lens), H * G, max_q, max_len, window)
    print(f"{plan} {t} lens={lens[:6]} queries={queries[:6]} H={H} G={G} d={d} window={window}", flush=True)
    assert plan.startswith(form) and also in plan
    masks = trees(queries, seed, kind)
    words = -(-max_q // 64)
    tree = torch.cat([plain.words_of(m, words) for m in masks]).to(DEV)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    got, lse = fk.fk_kv_attend_tree(cache, q, table, ints(lens), tree, q_start=ints(starts), max_q=max_q, max_len=max_len, window=window, lse=True,
                                    out=torch.full_like(q, math.nan))
    sees = [plain.tree_sees(m, L, n, window) if L >= n else short(m, L, n, window) for m, L, n in zip(masks, lens, queries)]
    values = [kv_plain.values(*x) for x in ((cache.k_codes, cache.k_scale, cache.k_levels), (cache.v_codes, cache.v_scale, cache.v_levels))]
    out, want_lse, mag, err = plain.attend(*values, q, table, lens, starts, d ** -0.5, sees)
    step = 2.0 ** -8 if t == BF16 else 2.0 ** -11
    allowed = step * 1.01 * out.abs() + (2.0 ** -10 + 2 * err[..., None]) * mag + 2.0 ** -24
    assert not got.isnan().any() and ((got.double() - out).abs() / allowed).max().item() <= 1.0
    assert torch.equal(lse == -math.inf, want_lse == -math.inf)
    live = want_lse > -math.inf
    assert ((lse.double() - want_lse).abs()[live] <= err[live] + 2.0 ** -20 * (1 + want_lse[live].abs())).all()


def ragged(B, n, max_len, seed, longest=2):
    """Lengths and numbers of queries: `longest` of max_len tokens, the others short, none among them, and some equal ones."""
    r = random.Random(seed)
    lens = [max_len] * min(longest, B) + [r.choice([0, 5, n, r.randint(0, 700), 300, 300]) for _ in range(B - longest)]
    queries = [n] + [r.choice([n, r.randint(0, n), n // 2]) for _ in range(B - 1)]
    order = list(range(1, B))
    r.shuffle(order)
    order.insert(r.randint(0, B - 1), 0)
    return [min(lens[i], max_len) for i in order], [queries[i] for i in order]


# tiles -> heads, query heads to each, sequences, tokens of a tree, tokens
SHARED = {
    32: {1: (1, 1, 1, 1, 200), 2: (1, 16, 2, 130, 1500), 3: (1, 3, 1, 13, 200), 4: (1, 48, 2, 130, 200)},
    64: {1: (1, 1, 1, 1, 200), 2: (1, 24, 1, 200, 300), 3: (1, 48, 1, 100, 200), 4: (1, 48, 2, 130, 200)},
    96: {1: (1, 1, 1, 1, 200), 2: (1, 48, 1, 100, 200), 3: (1, 48, 2, 100, 200)},
    128: {1: (1, 1, 1, 1, 200), 2: (1, 48, 1, 100, 200), 3: (1, 48, 2, 100, 200)},
    160: {1: (1, 1, 1, 1, 200), 2: (1, 48, 1, 100, 200)}, 192: {1: (1, 1, 1, 1, 200), 2: (1, 48, 1, 100, 200)},
    224: {1: (1, 1, 1, 1, 200)}, 256: {1: (1, 1, 1, 1, 200)},
}
WINDOWED = {
    32: {2: (1, 16, 2, 130, 5000, 1500), 3: (1, 3, 1, 13, 1400, 300), 4: (1, 48, 2, 130, 650, 50)},
    64: {2: (1, 16, 2, 130, 1400, 300), 3: (1, 16, 2, 130, 650, 50), 4: (1, 48, 2, 130, 650, 50)},
    96: {2: (1, 16, 2, 130, 650, 50), 3: (1, 16, 4, 130, 650, 50)}, 128: {2: (1, 16, 2, 130, 650, 50), 3: (1, 16, 4, 130, 650, 50)},
    160: {2: (1, 16, 2, 130, 650, 50)}, 192: {2: (1, 16, 2, 130, 650, 50)},
}
LONG = {
    32: {1: (8, 1, 40, 1, 9000), 2: (3, 1, 32, 130, 9000), 3: (1, 16, 8, 130, 9000), 4: (1, 48, 4, 130, 9000)},
    64: {1: (8, 1, 40, 1, 9000), 2: (1, 5, 24, 130, 9000), 3: (1, 12, 16, 100, 9000), 4: (1, 48, 4, 130, 9000)},
    96: {1: (1, 5, 24, 100, 9000), 2: (1, 48, 2, 130, 9000), 3: (1, 16, 8, 130, 9000)},
    128: {1: (3, 5, 32, 13, 9000), 2: (1, 48, 2, 130, 9000), 3: (1, 16, 8, 130, 9000)},
    160: {1: (1, 16, 4, 130, 12000), 2: (1, 16, 4, 130, 9000)}, 192: {1: (1, 16, 4, 130, 9000), 2: (1, 48, 2, 130, 9000)},
    224: {1: (1, 16, 2, 130, 9000)}, 256: {1: (1, 16, 2, 130, 9000)},
}
every = lambda table: [(d, tiles) for d in table for tiles in table[d]]  # noqa: E731


@pytest.mark.parametrize("t", [F16, BF16])
@pytest.mark.parametrize("d,tiles", every(SHARED))
def test_shared_rows_in_one_piece(d, tiles, t):
    H, G, B, n, L = SHARED[d][tiles]
    lens, queries = ragged(B, n, L, d + tiles, 1)
    planned(t, lens, queries, H, G, d, f"rows_shared(tiles={tiles},row_blocks={-(-n * G // (16 * tiles))},splits=1,chunk=0)", n, L, seed=d + tiles)


@pytest.mark.parametrize("d,tiles", every(WINDOWED))
def test_shared_rows_under_a_window(d, tiles):
    H, G, B, n, L, window = WINDOWED[d][tiles]
    lens, queries = ragged(B, n, L, d + tiles, 1)
    form = f"rows_shared(tiles={tiles},row_blocks={-(-n * G // (16 * tiles))},splits=1,chunk=0)"
    planned(F16, lens, queries, H, G, d, form, n, L, window=window, seed=d + tiles)
    planned(BF16, lens, queries, H, G, d, form, n, L, window=window, kind="any", seed=d + tiles + 1)


@pytest.mark.parametrize("t", [F16, BF16])
@pytest.mark.parametrize("d,tiles", [(d, tiles) for d in WIDTHS for tiles in range(1, MOST[d] + 1)])
def test_splits_and_their_joins(d, tiles, t):
    n, G = 13, {1: 1, 2: 2, 3: 3, 4: 4}[tiles]                    # 13, 26, 39 and 52 rows
    for L, splits in ((1500, 6), (3000, 12)):                     # joined by one wave and by eight
        planned(t, [L, 200], [n, 9], 1, G, d, f"rows_shared(tiles={tiles},row_blocks=1,splits={splits},chunk=256)", n, L, seed=d + L)
    planned(t, [9500, 90], [n, n], 1, G, d, f"rows_shared(tiles={tiles},row_blocks=1,splits=6,chunk=256)", n, 9500, window=1500, seed=d + 1)


@pytest.mark.parametrize("t", [F16, BF16])
@pytest.mark.parametrize("d", WIDTHS)
def test_rows_of_their_own(d, t):
    most = MOST[d]
    for tiles, H, G, B, n, L, packed in ((most, 1, 48, {4: 12, 3: 8, 2: 6, 1: 2}[most], 130, 200, ""),
                                         (most, *((4, most + 1, 64, 13) if most > 1 else (2, 1, 40, 100)), 200, ",packed"),
                                         (1, 1, 48, 2 if d > 64 else 3, 130, 200, ""),
                                         (1, *((4, 5, 40, 13) if d <= 64 else (3, 1, 32, 100)), 200, ",packed")):
        lens, queries = ragged(B, n, L, d + tiles)
        form = f"rows_own(tiles={tiles},row_blocks={-(-n * G // (16 * tiles))},waves={8 if tiles == 1 else 4}{packed})"
        planned(t, lens, queries, H, G, d, form, n, L, seed=d + tiles)


@pytest.mark.parametrize("d,H,G,B,n,L", [(32, 8, 2, 32, 40, 3000), (64, 8, 2, 32, 40, 1500), (96, 8, 4, 32, 13, 1500), (128, 8, 4, 32, 13, 1500),
                                         (160, 4, 1, 32, 130, 3000), (192, 4, 1, 32, 130, 3000)])
def test_rows_that_would_be_a_wave_s_own_in_a_row_are_shared_by_a_tree(d, H, G, B, n, L):
    lv = kv_plain.levels(H, F16, 1, DEV)
    rows = f"tiles={MOST[d]},row_blocks={-(-n * G // (16 * MOST[d]))},"
    assert fk.fk_kv_plan(fk.KVCache.empty(1, 64, lv, lv, d), B, H * G, n, L).startswith(f"rows_own({rows}")
    lens, queries = ragged(B, n, L, d)
    planned(F16 if d % 64 else BF16, lens, queries, H, G, d, f"rows_shared({rows}splits=1,chunk=0)", n, L, seed=d)


@pytest.mark.parametrize("t", [F16, BF16])
@pytest.mark.parametrize("d,tiles", every(LONG))
def test_the_longest_first_in_every_form(d, tiles, t):
    H, G, B, n, L = LONG[d][tiles]
    lens, queries = ragged(B, n, L, d + tiles)
    planned(t, lens, queries, H, G, d, f"rows_shared(tiles={tiles},row_blocks={-(-n * G // (16 * tiles))},splits=1,chunk=0,longest_first)", n, L,
            seed=d + tiles)


HEADS = {2: 48, 3: 32, 33: 20, 63: 12, 64: 12}                    # sequences -> query heads, so that there are rounds of workgroups


@pytest.mark.parametrize("order", ["up", "down", "equal", "none but one", "pairs", "any"])
@pytest.mark.parametrize("B", HEADS)
def test_orders_of_lengths(order, B):
    r = random.Random(B)
    lens = {"up": [40 + 9 * b for b in range(B)], "down": [700 - 9 * b for b in range(B)], "equal": [333] * B, "none but one": [0] * B,
            "pairs": [50 + b // 2 * 20 for b in range(B)], "any": [r.randint(0, 600) for _ in range(B)]}[order]
    lens[r.randint(0, B - 1)] = 8500
    n, G = 130 if B < 33 else 20, HEADS[B]
    planned(F16, lens, [n] + [r.randint(0, n) for _ in range(B - 1)], 1, G, 128, "rows_shared(tiles=", n, 8500, seed=B, also="longest_first")
    planned(BF16, lens, [n] * B, 1, G, 256, "rows_shared(tiles=1,", n, 8500, seed=B + 1, also="longest_first")


def test_more_sequences_than_a_wave_has_lanes_and_windows_come_in_their_order():
    lv = kv_plain.levels(1, F16, 1, DEV)
    c = fk.KVCache.empty(1, 64, lv, lv, 128)
    assert "longest_first" in fk.fk_kv_plan_tree(c, 64, 12, 20, 8500)
    assert "longest_first" not in fk.fk_kv_plan_tree(c, 65, 12, 20, 8500)
    assert "longest_first" not in fk.fk_kv_plan_tree(c, 64, 12, 20, 8500, 8400)
