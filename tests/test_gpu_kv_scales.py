"""fk_kv_attend where the values' scales differ by many powers of two: scales of tokens that a query does not see, a token that takes nearly all
of the softmax with hardly any value, rows of zeros.

Tolerance: as in test_gpu_kv_attend.py, and what weights lose that are far below a row's largest.  They are multiplied as fp16, in units in which the row's largest
weight times scale is at least 2^6; below fp16's smallest normal number each is off by at most 2^-25, so 2^-31 of the largest a token.  The largest one is
taken as at most twice the largest channel of the mean of |weight * value| (levels reach 0.6 of a scale and more)."""
import math

import pytest
import torch

from paper_2603_09229_amd import binding as fk
from tests import kv_plain
from tests.test_gpu_kv_attend import BF16, DEV, F16, make

pytestmark = pytest.mark.gpu


def attend(cache, q, table, lens, starts, **other):
    queries = [b - a for a, b in zip(starts, starts[1:])]
    return fk.fk_kv_attend(cache, q, table, torch.tensor(lens, dtype=torch.int32, device=DEV),
                           q_start=torch.tensor(starts, dtype=torch.int32, device=DEV), max_q=max(queries), max_len=max(lens), lse=True, **other)


def check(cache, q, table, lens, starts, window, got, lse):
    k = kv_plain.values(cache.k_codes, cache.k_scale, cache.k_levels)
    v = kv_plain.values(cache.v_codes, cache.v_scale, cache.v_levels)
    out, want_lse, mag, err = kv_plain.attend(k, v, q, table, lens, starts, q.shape[2] ** -0.5, True, window)
    step = 2.0 ** -8 if q.dtype == BF16 else 2.0 ** -11
    allowed = (step * 1.01 * out.abs() + (2.0 ** -10 + 2 * err[..., None]) * mag + max(lens) * 2.0 ** -30 * mag.amax(-1, keepdim=True)
               + (2.0 ** -24 if q.dtype == F16 else 0.0))
    off = (got.double() - out).abs()
    assert (off <= allowed).all(), f"{(off / allowed.clamp_min(1e-300)).max().item():.3g} of what is allowed"
    live = want_lse > -math.inf
    assert torch.equal(lse == -math.inf, ~live)
    assert ((lse.double() - want_lse).abs()[live] <= err[live] + 2.0 ** -20 * (1 + want_lse[live].abs())).all()


def places(table, positions, P):
    """Page and place of one position in each sequence."""
    return torch.tensor([int(table[b, p // P]) for b, p in enumerate(positions)], device=DEV), torch.tensor([p % P for p in positions], device=DEV)


# few sequences (shared rows), the same split along the tokens, waves with rows of their own in several tiles, and packed
FORMS = {"shared": ([400, 300], [240, 230], 1, 2, "rows_shared"), "split": ([9000], [6], 1, 4, "rows_shared"),
         "own": ([300, 170, 77, 64, 130, 500] * 2, [200, 170, 77, 30, 100, 150] * 2, 8, 3, "rows_own"),
         "packed": ([90, 40, 63, 35] * 8, [40, 40, 31, 35] * 8, 8, 3, "rows_own")}


@pytest.mark.parametrize("t", [F16, BF16])
@pytest.mark.parametrize("form,window", [("shared", 0), ("shared", 100), ("split", 0), ("own", 0), ("own", 12), ("packed", 0), ("packed", 12)])
def test_scales_that_a_query_does_not_see(form, t, window):
    """One token of each sequence, among its queries, has a value scale 2^20 to 2^26 times the others': queries before it, and those whose window it has left, give the
    same bits as without it; all of them are right."""
    lens, queries, H, G, name = FORMS[form]
    P, d = 16, 128
    cache, q, table, starts = make(t, lens, queries, H, G, d, P, 41)
    plan = fk.fk_kv_plan(cache, len(lens), H * G, max(queries), max(lens), window)
    assert plan.startswith(name) and (form != "split" or "splits=1," not in plan) and ("packed" in plan) == (form == "packed"), plan
    cache.v_scale.mul_(1e-3)
    big = [max(0, L - (n + 1) // 2) for L, n in zip(lens, queries)]
    page, place = places(table, big, P)
    clean, clean_lse = attend(cache, q, table, lens, starts, window=window)
    for times in (2.0 ** 20, 2.0 ** 24, 2.0 ** 26):
        was = cache.v_scale[page, :, place].clone()
        cache.v_scale[page, :, place] = (was.float() * times).clamp(max=torch.finfo(t).max).to(t)
        got, lse = attend(cache, q, table, lens, starts, window=window)
        for b, (L, n) in enumerate(zip(lens, queries)):
            pos = L - n + torch.arange(n, device=DEV)
            blind = (pos < big[b]) | ((pos - window >= big[b]) if window else False)
            s = slice(starts[b], starts[b + 1])
            assert blind.any() and not blind.all()
            assert torch.equal(got[s][blind], clean[s][blind]) and torch.equal(lse[s][blind], clean_lse[s][blind])
        check(cache, q, table, lens, starts, window, got, lse)
        cache.v_scale[page, :, place] = was


@pytest.mark.parametrize("t", [F16, BF16])
@pytest.mark.parametrize("lens,queries,H", [([5000], [1], 2), ([700, 40], [1, 1], 2), ([2000] * 6, [300] * 6, 8), ([90] * 32, [70] * 32, 8)])
@pytest.mark.parametrize("gap", [12.0, 24.0, 30.0])
def test_a_token_that_takes_the_softmax_with_hardly_any_value(t, lens, queries, H, gap):
    """The first token's score is `gap` powers of two above the others', its value's scale 2^-25 of theirs: the others make up the result."""
    P, d = 16, 64
    cache, q, table, starts = make(t, lens, queries, H, 1, d, P, 43)
    g = torch.Generator().manual_seed(44)
    base = 1.5 * torch.randn(H, d, generator=g)
    rows = base * (1 + 0.05 * torch.rand(q.shape[0], H, 1, generator=g))
    q = rows.to(t).to(DEV)
    cache.k_scale.mul_(0.01)
    cache.v_scale.mul_(9e3)
    page, place = places(table, [0] * len(lens), P)
    ids = torch.where(base > 0, 15, 0).to(torch.uint8)
    cache.k_codes[page, :, place] = (ids[:, 0::2] | ids[:, 1::2] << 4).to(DEV)
    reach = (base.abs() * torch.where(base > 0, cache.k_levels.float().cpu()[:, 15:], -cache.k_levels.float().cpu()[:, :1])).sum(1) / math.sqrt(d)
    cache.k_scale[page, :, place] = (gap * math.log(2) / reach).to(t).to(DEV)
    cache.v_scale[page, :, place] = 1e-3
    got, lse = attend(cache, q, table, lens, starts)
    check(cache, q, table, lens, starts, 0, got, lse)


@pytest.mark.parametrize("t", [F16, BF16])
@pytest.mark.parametrize("lens,queries,H", [([700], [1], 1), ([300] * 12, [150] * 12, 8), ([60] * 32, [40] * 32, 8)])
def test_values_of_zero(t, lens, queries, H):
    """Rows of zeros before others, after others and alone: they count in the softmax and add nothing."""
    P, d = 16, 64
    for zeros in (slice(0, 3), slice(1, 2), slice(0, 99)):
        cache, q, table, starts = make(t, lens, queries, H, 3, d, P, 45)
        for b in range(len(lens)):
            held = table[b, :-(-lens[b] // P)][zeros].long()
            cache.v_scale[held] = 0.0
        got, lse = attend(cache, q, table, lens, starts)
        check(cache, q, table, lens, starts, 0, got, lse)


@pytest.mark.parametrize("first,later", [(2.0 ** -80, 2.0 ** 60), (2.0 ** 60, 2.0 ** -80), (2.0 ** -80, 2.0 ** -80), (2.0 ** 100, 2.0 ** 100)])
def test_the_range_of_scales_in_bf16(first, later):
    lens, queries = [600, 70], [1, 60]
    cache, q, table, starts = make(BF16, lens, queries, 1, 4, 64, 16, 46)
    cache.v_scale[table[0, :8].long()] *= first
    cache.v_scale[table[0, 8:38].long()] *= later
    cache.v_scale[table[1, :2].long()] *= first
    cache.v_scale[table[1, 2:5].long()] *= later
    got, lse = attend(cache, q, table, lens, starts)
    check(cache, q, table, lens, starts, 0, got, lse)


@pytest.mark.parametrize("t", [F16, BF16])
@pytest.mark.parametrize("lens,queries,H,G", [([700], [1], 2, 3), ([9000], [2], 1, 4), ([300] * 12, [150] * 12, 8, 3), ([20] * 40, [1] * 40, 8, 2)])
@pytest.mark.parametrize("largest", [1.0, 2.0 ** -12])
def test_levels_of_the_values_far_below_the_largest(t, lens, queries, H, G, largest):
    """A channel whose values are all coded by levels of 3e-6 to 1e-7 of a head's largest keeps them to the type's bits."""
    P, d = 16, 64
    if t == F16:
        largest = 1.0                                             # (levels of 1e-7 are fp16's own smallest numbers)
    cache, q, table, starts = make(t, lens, queries, H, G, d, P, 47)
    small = torch.tensor([1.07e-7, 1.3e-6, 2.9e-6, 1.7e-5, 1.1e-4])
    lv = torch.cat([torch.linspace(-1, -0.2, 5), -small[:3].flip(0), small, torch.tensor([0.3, 0.7, 1.0])]) * largest
    cache.v_levels.copy_(lv.expand(H, 16).to(t))
    cache.v_codes[..., 3] = cache.v_codes[..., 3] % 3 + 8 | (cache.v_codes[..., 3] >> 4) % 3 + 5 << 4   # channel 6: above 0; 7: below
    got, lse = attend(cache, q, table, lens, starts)
    check(cache, q, table, lens, starts, 0, got, lse)
