"""fk_kv_attend_tree against the plain form in 64 bits: masks of trees and any others, lengths around the steps of 32 tokens, windows,
widths, splits, rows that see nothing, and a cache whose unread places hold NaN.  The tolerance is that of tests/test_gpu_kv_attend.py: the kernels
round in the same places."""
import math
import random

import pytest
import torch

from paper_2603_09229_amd import binding as fk
from tests import evict_plain as plain
from tests import kv_plain
from tests.test_gpu_kv_attend import BF16, DEV, F16, make

pytestmark = pytest.mark.gpu


def trees(queries, seed, kind="tree"):
    """Masks of each sequence: of a random tree, a chain, single tokens, any bits or none."""
    r, all_ = random.Random(seed), []
    for n in queries:
        rows = []
        for i in range(n):
            if kind == "tree":
                parent = r.randint(-1, i - 1)
                rows.append((rows[parent] if parent >= 0 else 0) | 1 << i)
            else:
                rows.append({"chain": (2 << i) - 1, "single": 1 << i, "any": r.getrandbits(n), "none": 0,
                             "beyond": r.getrandbits(64 * -(-n // 64))}[kind])
        all_.append(rows)
    return all_


def run(t, lens, queries, H, G, d, P, kind="tree", window=0, seed=0, strided=False, scale=None, words=None, max_len=None):
    # (places that some query may see are finite: with masks the window's first place is that of a row without marked tokens)
    cache, q, table, starts = make(t, lens, queries, H, G, d, P, seed, strided=strided, window=window + 1 if window else 0)
    masks = trees(queries, seed, kind)
    words = words or max(1, -(-max(queries) // 64))
    tree = torch.cat([plain.words_of(m, words) for m in masks]).to(DEV)
    scale = d ** -0.5 if scale is None else scale
    print(f"tree {t} lens={lens[:6]} queries={queries[:6]} H={H} G={G} d={d} P={P} kind={kind} window={window} words={words}", flush=True)
    got, lse = fk.fk_kv_attend_tree(cache, q, table, torch.tensor(lens, dtype=torch.int32, device=DEV), tree,
                                    q_start=torch.tensor(starts, dtype=torch.int32, device=DEV), max_q=max(1, max(queries)),
                                    max_len=max_len or max(1, max(lens)), scale=scale, window=window, lse=True)
    sees = [plain.tree_sees([x & (1 << n) - 1 for x in m], L, n, window) if L >= n else short(m, L, n, window)
            for m, L, n in zip(masks, lens, queries)]
    k = kv_plain.values(cache.k_codes, cache.k_scale, cache.k_levels)
    v = kv_plain.values(cache.v_codes, cache.v_scale, cache.v_levels)
    out, want_lse, mag, err = plain.attend(k, v, q, table, lens, starts, scale, sees)
    step = 2.0 ** -8 if t == BF16 else 2.0 ** -11
    allowed = step * 1.01 * out.abs() + (2.0 ** -10 + 2 * err[..., None]) * mag + 2.0 ** -24
    off = (got.double() - out).abs()
    assert not got.isnan().any() and (not off.numel() or (off / allowed).max().item() <= 1.0)
    assert torch.equal(lse == -math.inf, want_lse == -math.inf)
    live = want_lse > -math.inf
    assert ((lse.double() - want_lse).abs()[live] <= err[live] + 2.0 ** -20 * (1 + want_lse[live].abs())).all()
    return cache, q, table, starts, tree, got


def short(masks, L, n, window):
    """More queries than tokens: the first tokens of the tree do not exist."""
    sees = torch.zeros(n, L, dtype=torch.bool)
    for i in range(n):
        seen = [t for t in range(L) if masks[i] >> (t - L + n) & 1]
        sees[i, seen[-window:] if window else seen] = True
    return sees


@pytest.mark.parametrize("t", [F16, BF16])
@pytest.mark.parametrize("d", [32, 64, 96, 128, 160, 192, 224, 256])
def test_every_width(t, d):
    run(t, [45, 300, 700], [13, 1, 40], 2, 4, d, 16, seed=d)
    run(t, [300, 130], [70, 100], 2, 3, d, 32, seed=d + 1)


@pytest.mark.parametrize("kind", ["tree", "chain", "single", "any", "none", "beyond"])
@pytest.mark.parametrize("queries", [[1, 2], [31, 32, 33], [63, 64, 65, 0], [128, 129, 7]])
def test_masks(kind, queries):
    run(F16, [n + 17 * b for b, n in enumerate(queries)], queries, 2, 3, 64, 16, kind, seed=sum(queries))
    run(BF16, [n + 61 + 17 * b for b, n in enumerate(queries)], queries, 1, 4, 64, 16, kind, seed=sum(queries) + 1)


@pytest.mark.parametrize("before", [0, 1, 15, 16, 17, 30, 31, 32, 33, 63, 64, 65, 100])
def test_trees_that_begin_anywhere_in_a_step(before):
    run(F16, [before + 21, before + 64], [21, 64], 1, 2, 64, 16, "any", seed=before)


@pytest.mark.parametrize("window", [1, 2, 3, 5, 31, 32, 33, 64, 100, 100000])
@pytest.mark.parametrize("kind", ["tree", "chain", "any", "none"])
def test_windows(window, kind):
    run(BF16, [500, 129, 70], [40, 9, 70], 2, 3, 64, 16, kind, window=window, seed=window % 97)
    run(F16, [400], [200], 1, 2, 64, 16, kind, window=window, seed=window % 89)


def test_a_chain_sees_what_queries_in_a_row_see():
    for window in (0, 7, 50):
        cache, q, table, starts, tree, got = run(F16, [300, 90], [50, 50], 2, 4, 128, 16, "chain", window=window, seed=4)
        lens = torch.tensor([300, 90], dtype=torch.int32, device=DEV)
        row = fk.fk_kv_attend(cache, q, table, lens, max_q=50, max_len=300, window=window)
        # both are within 2^-11 of the value and 2^-10 of the mean magnitude, here below 8
        assert (row.float() - got.float()).abs().max() <= 2 * 8 * (2.0 ** -10 + 2.0 ** -11)


def test_fewer_tokens_than_the_tree():
    for kind in ("chain", "any", "none", "single"):
        run(F16, [2, 33, 0, 70], [3, 40, 5, 70], 2, 2, 64, 16, kind, seed=5)
        run(F16, [2, 33, 0, 70], [3, 40, 5, 70], 2, 2, 64, 16, kind, window=4, seed=6)


def test_wide_masks():
    run(F16, [1300, 900], [1000, 600], 1, 1, 64, 64, "tree", seed=1)
    run(BF16, [700, 90], [100, 20], 1, 8, 64, 64, "tree", seed=2, words=9)
    run(BF16, [700, 90], [100, 20], 1, 8, 64, 64, "any", seed=2, words=9, window=30)


def test_many_sequences():
    lens = [10 + 7 * b % 50 for b in range(150)]
    run(F16, [L + 9 for L in lens], [1 + b % 9 for b in range(150)], 2, 4, 64, 16, seed=3)
    run(BF16, [300 + L for L in lens[:40]], [30 + b % 20 for b in range(40)], 4, 4, 128, 16, seed=4)       # waves with rows of their own
    run(BF16, [300 + L for L in lens[:40]], [30 + b % 20 for b in range(40)], 4, 4, 128, 16, seed=4, window=77)


@pytest.mark.parametrize("lens", [[9000], [20000, 100], [30000] * 2])
def test_long_sequences_are_split_and_joined(lens):
    run(BF16, lens, [20] * len(lens), 1, 8, 128, 64, seed=3)
    run(F16, lens, [70] * len(lens), 1, 8, 64, 256, window=lens[0] // 2, seed=4)


@pytest.mark.parametrize("t", [F16, BF16])
def test_queries_at_odd_strides_and_scores_of_any_sign(t):
    run(t, [90, 300], [12, 64], 2, 4, 96, 16, strided=True)
    run(t, [90, 300], [12, 64], 2, 4, 64, 16, scale=-0.7)
    run(t, [90, 300], [12, 64], 2, 4, 64, 16, scale=0.0)


def test_a_wrong_upper_bound_of_the_lengths_costs_time_only():
    run(F16, [9000, 100], [20, 20], 1, 8, 64, 64, seed=8, max_len=1000)
    run(F16, [9000, 100], [20, 20], 1, 8, 64, 64, seed=8, max_len=1 << 20)


def test_nan_in_a_drafted_token_reaches_only_the_branch_below_it():
    cache, q, table, starts = make(F16, [200], [40], 1, 2, 64, 16, 13)
    lens = torch.tensor([200], dtype=torch.int32, device=DEV)
    masks = trees([40], 3)[0]
    tree = plain.words_of(masks, 1).to(DEV)
    clean = fk.fk_kv_attend_tree(cache, q, table, lens, tree, max_q=40)
    for which in (cache.v_scale, cache.k_scale):
        was = which.clone()
        place = 160 + 5
        which[table[0, place // 16].long(), 0, place % 16] = math.nan
        got = fk.fk_kv_attend_tree(cache, q, table, lens, tree, max_q=40)
        below = torch.tensor([m >> 5 & 1 == 1 for m in masks], device=DEV)
        assert below.any() and not below.all()
        assert torch.equal(got[~below], clean[~below]) and got[below].isnan().all()
        which.copy_(was)


def test_results_are_the_same_bits_every_time_and_under_a_graph():
    cache, q, table, starts = make(BF16, [9000, 700], [30, 30], 2, 4, 128, 64, 14)
    lens = torch.tensor([9000, 700], dtype=torch.int32, device=DEV)
    tree = torch.cat([plain.words_of(m, 1) for m in trees([30, 30], 9)]).to(DEV)
    ws = fk.make_kv_workspace(cache, 2, 8, 60, 30, 9000)
    out = torch.empty_like(q)
    call = lambda **more: fk.fk_kv_attend_tree(cache, q, table, lens, tree, max_q=30, max_len=9000, ws=ws, **more)  # noqa: E731
    first = call().clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        call(out=out)
        with torch.cuda.graph(graph, stream=side):
            call(out=out)
    for _ in range(4):
        ws.fill_(255)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first)
        ws.fill_(0)
        assert torch.equal(call(), first)
