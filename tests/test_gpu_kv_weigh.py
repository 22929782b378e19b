"""fk_kv_weigh against the plain form in 64 bits, with the tolerance derived there: single queries, chunks, windows, widths, groups, ragged
batches, tokens without weights, rows without a sum, and a cache whose unread places hold NaN."""
import math

import pytest
import torch

from paper_2603_09229_amd import binding as fk
from tests import evict_plain as plain
from tests import kv_plain
from tests.test_gpu_kv_attend import BF16, DEV, F16, make

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def run(t, lens, queries, H, G, d, P, causal=True, window=0, seed=0, strided=False, scale=None, max_len=None, known="old", decay=1.0,
        in_place=True):
    cache, q, table, starts = make(t, lens, queries, H, G, d, P, seed, strided=strided, window=window, causal=causal)
    cache.k_scale.copy_(torch.where(cache.k_scale.isnan(), 1.0, cache.k_scale.float()).to(t))   # (every token's key is read, in steps of 16)
    for b, L in enumerate(lens):                                                              # past the end anything may stand
        if L % P:
            cache.k_scale[table[b, L // P].long(), :, L % P:] = math.nan
    scale = d ** -0.5 if scale is None else scale
    k = kv_plain.values(cache.k_codes, cache.k_scale, cache.k_levels)
    sees = [plain.row_sees(L, n, causal, window) for L, n in zip(lens, queries)]
    lse = plain.attend(k, k, q, table, lens, starts, scale, sees)[1].float()
    g = torch.Generator(device=DEV).manual_seed(seed)
    mass = torch.rand(cache.pages, H, P, generator=g, device=DEV)
    known = {"old": [max(0, L - n) for L, n in zip(lens, queries)], "none": [0] * len(lens), "all": None}[known]
    upto = lens if known is None else known
    for b, L in enumerate(lens):                                  # what is not known is not read
        tok = torch.arange(upto[b], max(L, upto[b]), device=DEV)
        mass[table[b, tok // P].long(), :, tok % P] = math.nan
    out = None if in_place else torch.full_like(mass, -3.0)
    was = mass if in_place else out
    want, bound = plain.weigh(k, q, lse, table, lens, starts, scale, sees, upto, decay, mass, was)
    print(f"weigh {t} lens={lens[:6]} queries={queries[:6]} H={H} G={G} d={d} P={P} causal={causal} window={window}", flush=True)
    before = was.clone()
    got = fk.fk_kv_weigh(cache, q, lse, table, ints(lens), mass, q_start=ints(starts), max_q=max(1, max(queries)),
                         max_len=max_len or max(1, max(lens)), scale=scale, causal=causal, window=window,
                         known=None if known is None else ints(known), decay=decay, out=out)
    assert got is was
    inside = torch.zeros_like(mass, dtype=torch.bool)
    for b, L in enumerate(lens):
        tok = torch.arange(L, device=DEV)
        inside[table[b, tok // P].long(), :, tok % P] = True
    assert torch.equal(got[~inside].view(torch.int32), before[~inside].view(torch.int32))      # other places as they were
    assert not got[inside].isnan().any()
    worst = ((got.double() - want).abs() / bound.clamp_min(1e-300))[inside]
    assert not worst.numel() or worst.max().item() <= 1.0, f"{worst.max().item():.3f} of what is allowed"


@pytest.mark.parametrize("t", [F16, BF16])
@pytest.mark.parametrize("d", [32, 64, 96, 128, 160, 192, 224, 256])
def test_every_width(t, d):
    run(t, [1, 33, 700], [1, 1, 1], 2, 4, d, 16, seed=d)
    run(t, [300, 77], [70, 77], 2, 3, d, 32, seed=d + 1, known="none")


@pytest.mark.parametrize("lens", [[0], [1], [15], [16], [17], [31], [32], [33], [63, 64, 65], [255, 256, 257], [511, 513, 0, 1], [5000], [2049, 3, 0, 1000]])
@pytest.mark.parametrize("P", [16, 64])
def test_lengths_around_pages_and_steps(lens, P):
    run(F16, lens, [1] * len(lens), 1, 5, 64, P, seed=len(lens) + P)
    run(F16, lens, [1 if L else 0 for L in lens], 1, 5, 64, P, seed=len(lens) + P, known="all", decay=0.5, in_place=False)


@pytest.mark.parametrize("G", [1, 2, 7, 16, 17, 24, 33, 48, 64, 65, 100])
def test_groups(G):
    run(BF16, [301, 40], [1, 1], 3, G, 64, 32, seed=G)


@pytest.mark.parametrize("queries", [[2, 5, 1], [0, 3, 0], [16, 1, 15], [33, 64, 2], [130, 100, 0]])
@pytest.mark.parametrize("causal", [True, False])
def test_ragged_queries(queries, causal):
    run(F16, [400, 100, 64], queries, 2, 4, 128, 64, causal=causal, seed=sum(queries), decay=0.75)


@pytest.mark.parametrize("queries", [[1, 1], [9, 4], [200, 30]])
@pytest.mark.parametrize("window", [1, 2, 31, 32, 33, 100, 100000])
@pytest.mark.parametrize("causal", [True, False])
def test_windows(queries, window, causal):
    run(BF16, [500, 129], queries, 2, 3, 64, 16, causal=causal, window=window, seed=window % 97, known="all")


def test_more_queries_than_tokens():
    for queries in ([3, 40], [70, 90]):
        run(F16, [2, 33], queries, 2, 2, 64, 16, seed=5)
        run(F16, [2, 33], queries, 2, 2, 64, 16, window=7, seed=6, known="all")


@pytest.mark.parametrize("t", [F16, BF16])
def test_queries_at_odd_strides_and_scores_of_any_sign(t):
    run(t, [90, 300], [1, 1], 2, 4, 96, 16, strided=True)
    run(t, [90, 300], [64, 80], 2, 4, 128, 16, strided=True)
    for scale in (0.0, 3.0, -0.7):
        run(t, [1000, 31], [1, 7], 2, 4, 64, 16, scale=scale, seed=9)


@pytest.mark.parametrize("lens,queries", [([40000], [1]), ([20000, 100], [1, 1]), ([3000] * 3, [1500, 3, 700]), ([700], [700])])
def test_long_ones(lens, queries):
    run(BF16, lens, queries, 1, 8, 128, 64, seed=3, in_place=False)
    run(F16, lens, queries, 2, 3, 64, 256, window=lens[0] // 2, seed=4)


def test_many_sequences():
    lens = [1 + 37 * b % 200 for b in range(300)]
    run(F16, lens, [1] * 300, 3, 4, 64, 16, seed=1)
    run(BF16, [100 + L for L in lens[:60]], [b % 21 for b in range(60)], 5, 2, 96, 32, seed=2)


def test_a_wrong_upper_bound_of_the_lengths_costs_time_only():
    run(F16, [9000, 100], [1, 1], 1, 8, 64, 64, seed=8, max_len=1000)
    run(F16, [9000, 100], [5, 50], 1, 8, 64, 64, seed=8, max_len=1000)
    run(F16, [9000, 100], [1, 1], 1, 8, 64, 64, seed=8, max_len=1 << 20)


@pytest.mark.parametrize("n", [1, 300])
def test_tokens_whose_page_is_outside_the_cache_are_left_out(n):
    cache, q, table, starts = make(F16, [700, 400], [n, n], 2, 4, 64, 64, 3)
    k = kv_plain.values(cache.k_codes, cache.k_scale, cache.k_levels)
    sees = [plain.row_sees(L, n, True, 0) for L in (700, 400)]
    lse = plain.attend(k, k, q, table, [700, 400], starts, 0.125, sees)[1].float()
    mass = torch.rand(cache.pages, 2, 64, device=DEV)
    want, bound = plain.weigh(k, q, lse, table, [700, 400], starts, 0.125, sees, [700, 400], 1.0, mass, mass)
    wild, was = table.clone(), mass.clone()
    for b, p, page in ((0, 1, -1), (0, 8, cache.pages), (1, 0, 2 ** 31 - 1), (1, 3, -2 ** 31)):
        rows = table[b, p].long()
        want[rows], bound[rows] = was[rows].double(), 0.0
        wild[b, p] = page
    fk.fk_kv_weigh(cache, q, lse, wild, ints([700, 400]), mass, max_q=n)
    assert ((mass.double() - want).abs() <= bound).all()


def small(seed=13, n=40, L=200):
    cache, q, table, starts = make(F16, [L], [n], 1, 2, 64, 16, seed)
    lens = ints([L])
    _, lse = fk.fk_kv_attend(cache, q, table, lens, max_q=n, lse=True)
    return cache, q, lse, table, lens


def test_weights_of_a_query_add_up_to_one():
    cache, q, lse, table, lens = small()
    mass = torch.zeros(cache.pages, 1, 16, device=DEV)
    fk.fk_kv_weigh(cache, q, lse, table, lens, mass, max_q=40)
    # 80 rows of weights; logarithms and weights in 32 bits are off by less than 2^-18 here, where scores stay below 2^5
    assert abs(mass.double().sum().item() - 80) < 80 * 2.0 ** -17


def test_rows_without_a_sum_add_nothing_and_nan_stays_where_it_is_seen():
    cache, q, lse, table, lens = small()
    lse2 = lse.clone()
    lse2[7:] = -math.inf
    a = fk.fk_kv_weigh(cache, q, lse2, table, lens, torch.zeros(cache.pages, 1, 16, device=DEV), max_q=40)
    short = fk.fk_kv_weigh(cache, q[:7], lse[:7].contiguous(), table, lens - 33, torch.zeros(cache.pages, 1, 16, device=DEV), max_q=7)
    place = torch.arange(167, device=DEV)
    at = (table[0, place // 16].long(), 0, place % 16)
    # the same sums in another order of the additions: 14 numbers of one sign, twice
    assert ((a[at] - short[at]).abs() <= 28 * 2.0 ** -24 * a[at]).all() and a[at].sum() > 13
    bad = 180
    cache.k_scale[table[0, bad // 16].long(), 0, bad % 16] = math.nan
    clean = fk.fk_kv_weigh(cache, q, lse, table, lens, torch.zeros(cache.pages, 1, 16, device=DEV), max_q=40)
    assert clean.isnan().sum() == 1 and clean[table[0, bad // 16].long(), 0, bad % 16].isnan()
    gone = fk.fk_kv_weigh(cache, q[:20], lse[:20].contiguous(), table, lens - 20, torch.zeros(cache.pages, 1, 16, device=DEV), max_q=20)
    assert not gone.isnan().any()                                 # nobody sees it


def test_the_same_bits_every_time_and_under_a_graph():
    cache, q, lse, table, lens = small(14, 90, 3000)
    start = torch.rand(cache.pages, 1, 16, device=DEV)
    out = torch.empty_like(start)
    call = lambda o: fk.fk_kv_weigh(cache, q, lse, table, lens, start, max_q=90, out=o, decay=0.5)  # noqa: E731
    first = call(torch.zeros_like(start))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        call(out)
        with torch.cuda.graph(graph, stream=side):
            call(out)
    for _ in range(4):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first) and torch.equal(call(torch.zeros_like(start)), first)


def test_rows_divided_among_workgroups_in_a_used_workspace():
    """Few tokens and many queries: the parts' sums go through the workspace, whatever it holds, and nothing behind it is written."""
    cache, q, lse, table, lens = small(15, 900, 1000)
    n = fk.fk_kv_weigh_workspace_bytes(cache, 1, 2, 900, 900, 1000)
    assert n > 0
    first = fk.fk_kv_weigh(cache, q, lse, table, lens, torch.zeros(cache.pages, 1, 16, device=DEV), max_q=900, max_len=1000)
    for fill in (0, 255, 127):
        ws = torch.full((n + 4096,), fill, dtype=torch.uint8, device=DEV)
        ws[n:] = 91
        out = fk.fk_kv_weigh(cache, q, lse, table, lens, torch.zeros(cache.pages, 1, 16, device=DEV), max_q=900, max_len=1000, ws=ws[:n])
        assert torch.equal(out, first) and (ws[n:] == 91).all()
