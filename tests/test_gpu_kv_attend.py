"""fk_kv_attend against the plain form in 64 bits: lengths from nothing to many pages, ragged queries, windows, widths, groups, strides,
and a cache whose unread places hold NaN.

Tolerance, from how the result is computed: the weights are rounded to 11 significant bits (by 2^-11 of each at most, so of the mean of
|weight * value|), scores and exponentials in 32 bits add less than the same again at the sizes here: 2^-10 of that mean; the result is
rounded to its type, of 8 significant bits (2^-8) or 11 (2^-11)."""
import math

import pytest
import torch

from paper_2603_09229_amd import binding as fk
from tests import kv_plain

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
F16, BF16 = torch.float16, torch.bfloat16


def make(t, lens, queries, H, G, d, P, seed, spare=3, strided=False, window=0, causal=True):
    """Cache, queries and tables; scales outside of what any query sees are NaN."""
    g = torch.Generator().manual_seed(seed)
    held = [max(1, -(-L // P)) for L in lens]
    pages = sum(held) + spare
    order = torch.randperm(pages, generator=g).to(torch.int32)
    table = torch.full((len(lens), max(held) + 1), -7, dtype=torch.int32)
    seen = torch.zeros(pages, P, dtype=torch.bool)
    at = 0
    for b, (L, n) in enumerate(zip(lens, queries)):
        table[b, :held[b]] = order[at:at + held[b]]
        lo = max(0, L - n - window + 1) if window else 0
        for p in range(held[b]):
            tok = p * P + torch.arange(P)
            seen[int(order[at + p])] = (tok >= lo) & (tok < L)
        at += held[b]
    codes = [torch.randint(0, 256, (pages, H, P, d // 2), generator=g, dtype=torch.uint8) for _ in range(2)]
    scale = [(0.3 + 3 * torch.rand(pages, H, P, generator=g)).masked_fill(~seen[:, None], math.nan).to(t) for _ in range(2)]
    lv = [kv_plain.levels(H, t, seed + 1), kv_plain.levels(H, t, seed + 2)]
    starts = [sum(queries[:b]) for b in range(len(lens) + 1)]
    q = (torch.randn(starts[-1], H * G, d + (24 if strided else 0), generator=g) * 1.5).to(t).to(DEV)
    if strided:
        q = q[:, :, 3:3 + d]                                      # rows that start at odd elements
    cache = fk.KVCache(*(x.to(DEV) for x in (*codes, *scale, *lv)))
    return cache, q, table.to(DEV), starts


def check(cache, q, table, lens, starts, scale, causal, window, got, lse):
    t = q.dtype
    k = kv_plain.values(cache.k_codes, cache.k_scale, cache.k_levels)
    v = kv_plain.values(cache.v_codes, cache.v_scale, cache.v_levels)
    out, want_lse, mag, err = kv_plain.attend(k, v, q, table, lens, starts, scale, causal, window)
    step = 2.0 ** -8 if t == BF16 else 2.0 ** -11
    off = (got.double() - out).abs()
    allowed = step * 1.01 * out.abs() + (2.0 ** -10 + 2 * err[..., None]) * mag + 2.0 ** -24
    worst = (off / allowed).max().item() if off.numel() else 0.0
    assert not got.isnan().any() and worst <= 1.0, f"{worst:.3f} of what is allowed"
    assert torch.equal(lse == -math.inf, want_lse == -math.inf)
    live = want_lse > -math.inf
    assert ((lse.double() - want_lse).abs()[live] <= err[live] + 2.0 ** -20 * (1 + want_lse[live].abs())).all()


def run(t, lens, queries, H, G, d, P, causal=True, window=0, seed=0, strided=False, scale=None, max_len=None):
    cache, q, table, starts = make(t, lens, queries, H, G, d, P, seed, strided=strided, window=window)
    scale = d ** -0.5 if scale is None else scale
    print(f"attend {t} lens={lens[:6]} queries={queries[:6]} H={H} G={G} d={d} P={P} causal={causal} window={window}", flush=True)
    got, lse = fk.fk_kv_attend(cache, q, table, torch.tensor(lens, dtype=torch.int32, device=DEV),
                               q_start=torch.tensor(starts, dtype=torch.int32, device=DEV), max_q=max(1, max(queries)),
                               max_len=max_len or max(1, max(lens)), scale=scale, causal=causal, window=window, lse=True)
    check(cache, q, table, lens, starts, scale, causal, window, got, lse)


@pytest.mark.parametrize("t", [F16, BF16])
@pytest.mark.parametrize("d", [32, 64, 96, 128, 160, 192, 224, 256])
def test_single_tokens_of_every_width(t, d):
    run(t, [1, 33, 700], [1, 1, 1], 2, 4, d, 16, seed=d)


@pytest.mark.parametrize("t", [F16, BF16])
@pytest.mark.parametrize("d", [32, 64, 96, 128, 160, 192, 224, 256])
def test_chunks_of_every_width(t, d):
    run(t, [300, 77], [70, 77], 2, 3, d, 32, seed=d + 1)


@pytest.mark.parametrize("lens", [[0], [1], [15], [16], [17], [31], [32], [33], [63, 64, 65], [255, 256, 257], [511, 513, 0, 1], [5000], [2049, 3, 0, 1000]])
@pytest.mark.parametrize("P", [16, 64])
def test_lengths_around_pages_and_steps(lens, P):
    run(F16, lens, [1] * len(lens), 1, 5, 64, P, seed=len(lens) + P)


@pytest.mark.parametrize("G", [1, 2, 7, 16, 17, 24, 33, 48, 64, 65, 100])
def test_groups(G):
    run(BF16, [301, 40], [1, 1], 3, G, 64, 32, seed=G)


@pytest.mark.parametrize("queries", [[2, 5, 1], [0, 3, 0], [16, 1, 15], [33, 64, 2], [130, 100, 0]])
@pytest.mark.parametrize("causal", [True, False])
def test_ragged_queries(queries, causal):
    run(F16, [400, 100, 64], queries, 2, 4, 128, 64, causal=causal, seed=sum(queries))


@pytest.mark.parametrize("queries", [[1, 1], [9, 4], [200, 30]])
@pytest.mark.parametrize("window", [1, 2, 31, 32, 33, 100, 100000])
@pytest.mark.parametrize("causal", [True, False])
def test_windows(queries, window, causal):
    run(BF16, [500, 129], queries, 2, 3, 64, 16, causal=causal, window=window, seed=window % 97)


def test_more_queries_than_tokens_leave_rows_that_see_nothing():
    for queries in ([3, 40], [70, 90]):
        run(F16, [2, 33], queries, 2, 2, 64, 16, seed=5)
        run(F16, [2, 33], queries, 2, 2, 64, 16, window=7, seed=6)


@pytest.mark.parametrize("t", [F16, BF16])
def test_queries_at_odd_strides(t):
    run(t, [90, 300], [1, 1], 2, 4, 96, 16, strided=True)
    run(t, [90, 300], [64, 80], 2, 4, 128, 16, strided=True)


@pytest.mark.parametrize("lens", [[9000], [20000, 100], [40000] * 3])
def test_long_sequences_are_split_and_joined(lens):
    run(BF16, lens, [1] * len(lens), 1, 8, 128, 64, seed=3)
    run(F16, lens, [3] * len(lens), 1, 8, 64, 256, window=lens[0] // 2, seed=4)


def test_a_wrong_upper_bound_of_the_lengths_costs_time_only():
    run(F16, [9000, 100], [1, 1], 1, 8, 64, 64, seed=8, max_len=1000)
    run(F16, [9000, 100], [1, 1], 1, 8, 64, 64, seed=8, max_len=1 << 20)


def test_sharp_and_flat_scores():
    for scale in (0.0, 1e-4, 3.0, -0.7):
        run(F16, [1000, 31], [1, 1], 2, 4, 64, 16, scale=scale, seed=9)
        run(BF16, [200, 31], [70, 31], 2, 4, 64, 16, scale=scale, seed=9)


@pytest.mark.parametrize("t", [F16, BF16])
@pytest.mark.parametrize("first,later", [(1e-6, 1.0), (1.0, 1e-6), (1e-30, 1e30), (3e4, 1e-3)])
def test_scales_of_the_values_over_their_whole_range(t, first, later):
    """The weights' power of two follows the largest scale: neither tiny nor huge values lose their bits."""
    if t == F16 and later > 1e5:
        pytest.skip("beyond fp16")
    cache, q, table, starts = make(t, [600], [1], 1, 4, 64, 16, 12)
    lim = cache.v_scale.float()
    lim[table[0, :8].long()] *= first
    lim[table[0, 8:38].long()] *= later
    cache.v_scale.copy_(lim.clamp(max=torch.finfo(t).max).to(t))
    lens = torch.tensor([600], dtype=torch.int32, device=DEV)
    got, lse = fk.fk_kv_attend(cache, q, table, lens, lse=True)
    k = kv_plain.values(cache.k_codes, cache.k_scale, cache.k_levels)
    v = kv_plain.values(cache.v_codes, cache.v_scale, cache.v_levels)
    out, _, mag, err = kv_plain.attend(k, v, q, table, [600], starts, 64 ** -0.5, True, 0)
    step = 2.0 ** -8 if t == BF16 else 2.0 ** -11
    allowed = step * 1.01 * out.abs() + (2.0 ** -10 + 2 * err[..., None]) * mag + (2.0 ** -24 if t == F16 else 0.0)
    assert ((got.double() - out).abs() <= allowed).all()


def test_nan_in_a_visible_row_reaches_only_the_queries_that_see_it():
    cache, q, table, starts = make(F16, [200], [40], 1, 2, 64, 16, 13)
    lens = torch.tensor([200], dtype=torch.int32, device=DEV)
    clean = fk.fk_kv_attend(cache, q, table, lens, max_q=40)
    cache.v_scale[table[0, 180 // 16].long(), 0, 180 % 16] = math.nan
    got = fk.fk_kv_attend(cache, q, table, lens, max_q=40)
    assert torch.equal(got[:20], clean[:20]) and got[20:].isnan().all()


def test_results_are_the_same_bits_every_time_and_under_a_graph():
    cache, q, table, starts = make(BF16, [9000, 700], [1, 1], 2, 4, 128, 64, 14)
    lens = torch.tensor([9000, 700], dtype=torch.int32, device=DEV)
    ws = fk.make_kv_workspace(cache, 2, 8, 2, 1, 9000)
    out = torch.empty_like(q)
    first = fk.fk_kv_attend(cache, q, table, lens, max_len=9000, ws=ws).clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        fk.fk_kv_attend(cache, q, table, lens, max_len=9000, ws=ws, out=out)
        with torch.cuda.graph(graph, stream=side):
            fk.fk_kv_attend(cache, q, table, lens, max_len=9000, ws=ws, out=out)
    for _ in range(4):
        ws.fill_(255)
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first)
        ws.fill_(0)
        assert torch.equal(fk.fk_kv_attend(cache, q, table, lens, max_len=9000, ws=ws), first)


def test_workspace_is_not_written_past_its_end():
    cache, q, table, starts = make(F16, [9000], [1], 1, 8, 128, 64, 15)
    lens = torch.tensor([9000], dtype=torch.int32, device=DEV)
    n = fk.fk_kv_workspace_bytes(cache, 1, 8, 1, 1, 9000)
    buf = torch.full((n + 4096,), 91, dtype=torch.uint8, device=DEV)
    fk.fk_kv_attend(cache, q, table, lens, max_len=9000, ws=buf[:n])
    assert (buf[n:] == 91).all()
