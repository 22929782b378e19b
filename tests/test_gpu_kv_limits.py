"""The 4-bit cache at the ends of its ranges: windows as long as the type holds, with more queries than tokens; sequences that fill their room.
Inputs, comparison and tolerance as in test_gpu_kv_attend.py."""
import pytest
import torch

from paper_2603_09229_amd import binding as fk
from paper_2603_09229_amd import kv_cache
from tests import kv_plain
from tests.test_gpu_kv_attend import BF16, DEV, F16, make, run

pytestmark = pytest.mark.gpu
LAST = 2 ** 31 - 1


# few sequences, whose workgroups share the rows; many short ones, several to a workgroup; more rows than a tile in enough workgroups, a wave each
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window", [LAST, LAST - 1, LAST - 40, 2 ** 30, 2 ** 30 + 1])
def test_the_longest_windows(window, causal):
    run(F16, [2, 33], [40, 90], 2, 2, 64, 16, window=window, causal=causal, seed=31)
    run(BF16, [2, 33, 5000], [5, 1, 9], 1, 4, 128, 16, window=window, causal=causal, seed=32)
    run(BF16, [3, 0, 30] * 40, [5, 2, 1] * 40, 3, 2, 96, 16, window=window, causal=causal, seed=33)
    run(F16, [2, 100, 17, 64] * 8, [70, 100, 40, 20] * 8, 8, 3, 128, 16, window=window, causal=causal, seed=34)


def test_a_server_fills_its_sequences_to_the_last_token_and_no_further():
    """max_len is no multiple of the page: the last tokens are turned by their own angles, one more is refused and changes nothing."""
    g = torch.Generator().manual_seed(35)
    lv = kv_plain.levels(2, F16, 7, DEV)
    server = kv_cache.Server(lv, lv, 64, 2, 37, page_size=16)
    rows = lambda T: [torch.randn(T, h, 64, generator=g).half().to(DEV) for h in (4, 2, 2)]
    server.step(*rows(66), [36, 30])
    q, k, v = rows(3)
    with pytest.raises(ValueError):
        server.step(q, k, v, [2, 1])
    assert server.lens.tolist() == [36, 30]
    out = server.step(q, k, v, [1, 2])
    assert server.lens.tolist() == [37, 32]
    pos = torch.tensor([36, 30, 31], device=DEV)
    cache = server.cache
    slots = server.pages[torch.tensor([0, 1, 1], device=DEV), pos // 16].long() * 16 + pos % 16
    want = kv_plain.turned(k, server.cos_sin, pos, False)
    assert torch.equal(cache.k_scale[slots // 16, :, slots % 16], want.abs().amax(-1))
    assert server.step(*rows(0), [0, 0]).shape == (0, 4, 64) and out.shape == (3, 4, 64)


@pytest.mark.parametrize("B,max_pages", [(0, 3), (0, 0), (1, 0)])
@pytest.mark.parametrize("own", [False, True])
def test_no_sequence_and_no_page_are_refused(B, max_pages, own):
    lv = kv_plain.levels(1, F16, 7, DEV)
    cache = fk.KVCache.empty(3, 16, lv, lv, 64)
    pages, lens = torch.zeros(B, max_pages, dtype=torch.int32, device=DEV), torch.zeros(B, dtype=torch.int32, device=DEV)
    with pytest.raises(fk.FlashKMError, match="positive|max_pages"):
        fk.fk_kv_attend(cache, torch.zeros(B, 2, 64, dtype=F16, device=DEV), pages, lens,
                        ws=torch.empty(4096, dtype=torch.uint8, device=DEV) if own else None)


def test_integers_beyond_32_bits_are_not_cut():
    lv = kv_plain.levels(1, F16, 7, DEV)
    cache = fk.KVCache.empty(3, 16, lv, lv, 64)
    x = torch.randn(40, 1, 64, device=DEV).half()
    fk.fk_kv_append(cache, x, x, torch.arange(40, device=DEV))
    pages, lens = torch.tensor([[0, 1, 2]], dtype=torch.int32, device=DEV), torch.tensor([40], dtype=torch.int32, device=DEV)
    q, start = x[:4], torch.tensor([0, 4], dtype=torch.int32, device=DEV)
    want = fk.fk_kv_attend(cache, q, pages, lens, max_q=4)
    for window in (2 ** 31, 2 ** 32 + 5, 2 ** 40, 10 ** 30):
        assert torch.equal(fk.fk_kv_attend(cache, q, pages, lens, max_q=4, window=window), want)
        assert fk.fk_kv_plan(cache, 1, 1, 4, 48, window) == fk.fk_kv_plan(cache, 1, 1, 4, 48)
    for bad in (2 ** 31, 2 ** 32 + 4, -2 ** 32 + 4):
        with pytest.raises(ValueError, match="32 bits"):
            fk.fk_kv_attend(cache, q, pages, lens, q_start=start, max_q=bad)
        with pytest.raises(ValueError, match="32 bits"):
            fk.fk_kv_attend(cache, q, pages, lens, max_q=4, window=-2 ** 32 + 4)
        with pytest.raises(ValueError, match="32 bits"):
            fk.make_kv_workspace(cache, 1, 1, 4, bad, 48)
        with pytest.raises(ValueError, match="32 bits"):
            fk.fk_kv_plan(cache, bad, 1, 4, 48)
    for other in (dict(max_q=-1, q_start=start), dict(max_q=4, window=-1)):
        with pytest.raises(fk.FlashKMError):
            fk.fk_kv_attend(cache, q, pages, lens, **other)


@pytest.mark.parametrize("t", [F16, BF16])
@pytest.mark.parametrize("lens,queries,H,G", [([300], [40], 1, 2), ([9000], [6], 1, 4), ([300, 170] * 6, [200, 170] * 6, 8, 3), ([90, 40] * 16, [40, 40] * 16, 8, 3)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_value_that_is_not_finite_leaves_the_softmax_alone(t, lens, queries, H, G, bad):
    """Rows that see it give no number, others the same bits; the logarithm of the sum is a matter of the keys, wherever in a step the token lies."""
    cache, q, table, starts = make(t, lens, queries, H, G, 64, 16, 51)
    at = [L - n // 2 for L, n in zip(lens, queries)]                    # among the queries
    call = lambda: fk.fk_kv_attend(cache, q, table, torch.tensor(lens, dtype=torch.int32, device=DEV), max_q=max(queries), max_len=max(lens), lse=True,
                                   q_start=torch.tensor(starts, dtype=torch.int32, device=DEV))
    clean, clean_lse = call()
    for places in (at, [5] * len(lens)):
        was = cache.v_scale.clone()
        for b, p in enumerate(places):
            cache.v_scale[table[b, p // 16].long(), :, p % 16] = bad
        got, lse = call()
        cache.v_scale.copy_(was)
        for b, (L, n) in enumerate(zip(lens, queries)):
            sees = L - n + torch.arange(n, device=DEV) >= places[b]
            s = slice(starts[b], starts[b + 1])
            assert not got[s][sees].isfinite().any() and torch.equal(got[s][~sees], clean[s][~sees]) and torch.equal(lse[s][~sees], clean_lse[s][~sees])
        # (another reference rounds it otherwise: two sums of fp32 numbers, none negative)
        assert ((lse - clean_lse).abs() <= 2.0 ** -20 * (1 + clean_lse.abs())).all()


@pytest.mark.parametrize("t", [F16, BF16])
@pytest.mark.parametrize("lens,queries,H,G", [([301, 7], [1, 1], 2, 4), ([9003], [6], 1, 4), ([305, 171] * 6, [200, 170] * 6, 8, 3), ([91, 44] * 16, [40, 40] * 16, 8, 3)])
@pytest.mark.parametrize("window", [0, 30])
def test_what_no_query_sees_may_be_anything(t, lens, queries, H, G, window):
    """Past the end, in pages of nobody and before every window: numbers of either sign, infinities and NaN, mixed or all alike, give the same bits."""
    cache, q, table, starts = make(t, lens, queries, H, G, 64, 16, 52, window=window)
    call = lambda: fk.fk_kv_attend(cache, q, table, torch.tensor(lens, dtype=torch.int32, device=DEV), max_q=max(queries), max_len=max(lens), lse=True,
                                   q_start=torch.tensor(starts, dtype=torch.int32, device=DEV), window=window)
    free = cache.v_scale.isnan()                                        # as make() leaves them
    want, want_lse = call()
    assert want.isfinite().all()
    big = torch.finfo(t).max
    mixed = torch.tensor([-1e-4, float("inf"), -big, 0.0, -float("inf"), big, -0.0, float("nan"), 1e-6], device=DEV).to(t)
    for fill in [mixed] + [mixed[i:i + 1] for i in range(len(mixed))]:
        for scale in (cache.k_scale, cache.v_scale):
            n = int(free.sum())
            scale[free] = fill.repeat(-(-n // len(fill)))[:n]
        got, lse = call()
        assert torch.equal(got, want) and torch.equal(lse, want_lse)


def test_nothing_carries_a_gradient():
    """Inputs that ask for one: results do not, and learned levels are those of the same rows (not the first guess with a gradient of its own)."""
    rows = torch.randn(40, 2, 64, device=DEV, generator=torch.Generator(DEV).manual_seed(5)).half()
    lv = kv_cache.learn_levels(rows)
    asking = rows.clone().requires_grad_()
    got = kv_cache.learn_levels(asking)
    assert not got.requires_grad and torch.equal(got, lv)
    server = kv_cache.Server(lv, lv, 64, 1, 64)
    assert not server.step(asking, asking, asking, [40]).requires_grad
