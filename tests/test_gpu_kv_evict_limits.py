"""Drafting and eviction at the ends of the ranges: a cache whose rows pass 2^31 and whose codes pass 2^35 bytes, the widest group, and other
streams than the current one."""
import pytest
import torch

from paper_2603_09229_amd import binding as fk
from tests import evict_plain as plain
from tests import kv_plain

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def small_cache(H, d, P, pages, seed, t=torch.float16):
    g = torch.Generator(device=DEV).manual_seed(seed)
    codes = [torch.randint(0, 256, (pages, H, P, d // 2), generator=g, dtype=torch.uint8, device=DEV) for _ in range(2)]
    scale = [(0.3 + torch.rand(pages, H, P, generator=g, device=DEV)).to(t) for _ in range(2)]
    lv = [kv_plain.levels(H, t, s, DEV) for s in (1, 2)]
    return fk.KVCache(*codes, *scale, *lv), torch.rand(pages, H, P, generator=g, device=DEV), g


def calls(cache, mass, pages, to, q, lens, tree, kept, counts):
    """One after the other, as a server makes them -> what they give."""
    out, lse = fk.fk_kv_attend_tree(cache, q, pages, lens, tree, max_q=20, lse=True)
    fk.fk_kv_weigh(cache, q, lse, pages, lens, mass, max_q=20)
    chosen = fk.fk_kv_choose(cache, mass, pages, lens, 300, first=4, last=20)
    fk.fk_kv_compact(cache, pages, kept, counts, to_pages=to, mass=mass)
    fk.fk_kv_compact(cache, pages, *chosen, mass=mass)
    P = cache.page_size
    place = torch.arange(300, device=DEV)
    rows = lambda x, table: x[table[0, place // P].long(), :, place % P].clone()  # noqa: E731
    return [out, lse, *chosen] + [rows(x, t) for t in (pages, to) for x in (cache.k_codes, cache.v_codes, cache.k_scale, cache.v_scale, mass)]


def test_a_cache_beyond_32_bits():
    H, d, P, n = 2, 32, 4096, 6
    cache, mass, g = small_cache(H, d, P, n, 1)
    pages = (1 << 31) // (H * P) + n
    big_mass = torch.empty(pages, H, P, device=DEV)
    big = fk.KVCache(*(torch.empty(pages, *x.shape[1:], dtype=x.dtype, device=DEV) for x in (cache.k_codes, cache.v_codes, cache.k_scale, cache.v_scale)),
                     cache.k_levels, cache.v_levels)
    at = torch.arange(pages - n, pages, device=DEV)
    for x, y in [(getattr(big, k), getattr(cache, k)) for k in ("k_codes", "v_codes", "k_scale", "v_scale")] + [(big_mass, mass)]:
        x[at] = y
    # pages that the same places would have if a number of rows were cut to 32 bits, or to 31
    others = torch.cat([torch.arange(n, device=DEV), at - (1 << 31) // (H * P) + (1 << 30) // (H * P)])
    for x in (big.k_codes, big.v_codes, big.k_scale, big.v_scale, big_mass):
        x[others] = 1
    q = torch.randn(20, 4, d, generator=g, device=DEV).half()
    lens = torch.tensor([9000], dtype=torch.int32, device=DEV)
    tree = plain.words_of([(1 << i + 1) - 1 - (1 << i // 2 if i > 3 else 0) for i in range(20)], 1).to(DEV)
    kept = torch.arange(50, 350, device=DEV, dtype=torch.int32).view(1, 1, -1)
    counts = torch.tensor([300], dtype=torch.int32, device=DEV)
    table, to = torch.tensor([[4, 1, 3]], dtype=torch.int32, device=DEV), torch.tensor([[5]], dtype=torch.int32, device=DEV)
    want = calls(cache, mass, table, to, q, lens, tree, kept, counts)
    got = calls(big, big_mass, table + (pages - n), to + (pages - n), q, lens, tree, kept, counts)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    for x in (big.k_codes, big.v_codes, big.k_scale, big.v_scale, big_mass):
        assert (x[others] == 1).all()


@pytest.mark.parametrize("G", [300, 1000])
def test_more_heads_to_a_group_than_a_block_of_rows(G):
    cache, mass, g = small_cache(1, 128, 64, 12, 3)
    q = torch.randn(5, G, 128, generator=g, device=DEV).half()
    lens, table = torch.tensor([700], dtype=torch.int32, device=DEV), torch.randperm(12, device=DEV).int()[None]
    masks = [1, 3, 5, 13, 16]
    tree = plain.words_of(masks, 1).to(DEV)
    out, lse = fk.fk_kv_attend_tree(cache, q, table, lens, tree, max_q=5, lse=True)
    k = kv_plain.values(cache.k_codes, cache.k_scale, cache.k_levels)
    v = kv_plain.values(cache.v_codes, cache.v_scale, cache.v_levels)
    want, want_lse, mag, err = plain.attend(k, v, q, table, [700], [0, 5], 128 ** -0.5, [plain.tree_sees(masks, 700, 5, 0)])
    assert ((out.double() - want).abs() <= 2.0 ** -11 * 1.01 * want.abs() + (2.0 ** -10 + 2 * err[..., None]) * mag + 2.0 ** -24).all()
    sees = [plain.row_sees(700, 5, True, 0)]
    lse = plain.attend(k, k, q, table, [700], [0, 5], 128 ** -0.5, sees)[1].float()
    got = fk.fk_kv_weigh(cache, q, lse, table, lens, mass.clone(), max_q=5, decay=0.5)
    want, bound = plain.weigh(k, q, lse, table, [700], [0, 5], 128 ** -0.5, sees, [700], 0.5, mass, mass)
    page, place = table[0, torch.arange(700, device=DEV) // 64].long(), torch.arange(700, device=DEV) % 64
    assert ((got.double() - want).abs() <= bound)[page, :, place].all()


def test_calls_on_another_stream_wait_for_what_was_issued_there():
    cache, mass, g = small_cache(2, 64, 16, 80, 5)
    table, to = torch.randperm(80, device=DEV).int()[None, :60], None
    q = torch.randn(20, 4, 64, generator=g, device=DEV).half()
    lens = torch.tensor([900], dtype=torch.int32, device=DEV)
    tree = plain.words_of([2 << i for i in range(20)], 1).to(DEV)
    spare = torch.tensor([[x for x in range(80) if x not in table[0].tolist()]], dtype=torch.int32, device=DEV)
    kept = torch.arange(50, 350, device=DEV, dtype=torch.int32).view(1, 1, -1)[:, :, :300]
    counts = torch.tensor([300], dtype=torch.int32, device=DEV)
    state = [x.clone() for x in (cache.k_codes, cache.v_codes, cache.k_scale, cache.v_scale, mass)]
    want = calls(cache, mass, table.contiguous(), spare, q, lens, tree, kept, counts)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for x, y in zip((cache.k_codes, cache.v_codes, cache.k_scale, cache.v_scale, mass), state):
            x.copy_(y)
        got = calls(cache, mass, table.contiguous(), spare, q, lens, tree, kept, counts)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
