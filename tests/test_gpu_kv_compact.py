"""fk_kv_compact bit by bit against copies on the host: in place and into other pages, a choice for each head or one for all, behind a prefix,
rows that are left out, and everything else as it was."""
import pytest
import torch

from paper_2603_09229_amd import binding as fk
from tests import evict_plain as plain
from tests import kv_plain

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
NAMES = ("k_codes", "v_codes", "k_scale", "v_scale")


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def make(room, H, d, P, seed, t=torch.float16, more=0):
    """Cache of random bits, tables of sequences with `room` places each, weights; `more` pages behind."""
    g = torch.Generator().manual_seed(seed)
    held = [max(1, -(-r // P)) for r in room]
    pages = sum(held) + more + 2
    order = torch.randperm(pages, generator=g).to(torch.int32)
    table = torch.full((len(room), max(held)), -5, dtype=torch.int32)
    at = 0
    for b, n in enumerate(held):
        table[b, :n] = order[at:at + n]
        at += n
    bits = lambda *s: torch.randint(-2 ** 15, 2 ** 15, s, generator=g, dtype=torch.int16)  # noqa: E731
    cache = fk.KVCache(*(torch.randint(0, 256, (pages, H, P, d // 2), generator=g, dtype=torch.uint8).to(DEV) for _ in range(2)),
                       *(bits(pages, H, P).view(t).to(DEV) for _ in range(2)), *[kv_plain.levels(H, t, 1, DEV)] * 2)
    mass = torch.randn(pages, H, P, generator=g).to(DEV)
    return cache, table, mass, order[at:at + more], g


def bits_of(x):
    return x if x.dtype == torch.uint8 else x.view(torch.int16 if x.element_size() == 2 else torch.int32)


def check(cache, mass, table, kept, counts, start, to, weights=True):
    host = [bits_of(getattr(cache, n)).cpu() for n in NAMES] + [bits_of(mass).cpu()]
    want = plain.compact(host, table, kept, [min(c, kept.shape[2]) for c in counts], start, table if to is None else to)
    print(f"compact d={cache.d} P={cache.page_size} H={cache.heads} counts={counts[:6]} start={start[:6]} {'in place' if to is None else ''}", flush=True)
    fk.fk_kv_compact(cache, table.to(DEV), kept.to(DEV), ints(counts), start=ints(start) if any(start) else None,
                     to_pages=None if to is None else to.to(DEV), mass=mass if weights else None)
    got = [bits_of(getattr(cache, n)).cpu() for n in NAMES] + [bits_of(mass).cpu()]
    for name, x, y, z in zip(NAMES + ("mass",), got, want, host):
        assert torch.equal(x, z if name == "mass" and not weights else y), name


def places(lens, keep, heads, g):
    kept = torch.full((len(lens), heads, max(keep)), -1, dtype=torch.int32)
    for b, (L, n) in enumerate(zip(lens, keep)):
        for h in range(heads):
            kept[b, h, :n] = torch.randperm(L, generator=g)[:n].sort().values.int()
    return kept


@pytest.mark.parametrize("d", [32, 64, 96, 128, 160, 192, 224, 256])
@pytest.mark.parametrize("in_place", [True, False])
def test_every_width(d, in_place):
    lens, keep = [300, 40, 90], [170, 40, 1]
    cache, table, mass, more, g = make(lens, 3, d, 16, d, torch.bfloat16, 11 * 3)
    check(cache, mass, table, places(lens, keep, 3, g), keep, [0, 0, 0], None if in_place else more.view(3, 11))


@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 255, 256, 257, 511, 512, 513, 1024, 1025, 2000])
@pytest.mark.parametrize("heads", [1, 2])
def test_numbers_of_rows(n, heads):
    lens = [n + n // 3 + 1, n]
    cache, table, mass, more, g = make(lens, 2, 64, 32, n, more=2 * (n // 32 + 1))
    kept = places(lens, [n, n], heads, g)
    check(cache, mass, table, kept, [n, n], [0, 0], more.view(2, -1))
    check(cache, mass, table, kept, [n, n], [0, 0], None)


def test_one_row_is_dropped_and_all_behind_it_move():
    cache, table, mass, _, _ = make([3000], 2, 128, 64, 3)
    kept = torch.tensor([t for t in range(3000) if t != 2], dtype=torch.int32).view(1, 1, -1)
    check(cache, mass, table, kept, [2999], [0], None)


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("share", [0.1, 0.5, 0.95])
def test_long_sequences_in_place(d, share):
    """More rows than a tile: those from behind what is written, and those that are moved in order."""
    lens = [9000, 5000]
    cache, table, mass, _, g = make([L + 30 for L in lens], 2, d, 64, int(d + 10 * share))
    keep = [int(L * share) for L in lens]
    check(cache, mass, table, places(lens, keep, 2, g), keep, [0, 0], None)
    kept = places(lens, keep, 2, g)
    kept[:, :, 5::7] = -1                                         # places that are left out
    check(cache, mass, table, kept, keep, [30, 17], None)


def test_the_first_and_the_last_tokens_of_long_sequences_in_place():
    cache, table, mass, _, _ = make([20000], 2, 64, 64, 9)
    kept = torch.cat([torch.arange(4), torch.arange(20000 - 8000, 20000)]).int().view(1, 1, -1)
    check(cache, mass, table, kept, [8004], [0], None)
    kept = torch.cat([torch.arange(4), torch.arange(20000 - 18000, 20000)]).int().view(1, 1, -1)
    check(cache, mass, table, kept, [18004], [0], None)


def test_a_branch_behind_a_prefix():
    cache, table, mass, _, _ = make([150, 40, 20], 4, 64, 16, 4)
    kept = torch.tensor([[0, 3, 7, 11], [2, 3, -1, -1], [0, 1, 2, 9]], dtype=torch.int32)[:, None]
    check(cache, mass, table, kept, [4, 2, 4], [120, 17, 5], None, weights=False)


def test_nothing_to_move():
    cache, table, mass, _, _ = make([50, 60], 2, 64, 16, 5)
    kept = torch.arange(50, dtype=torch.int32).expand(2, 2, 50).contiguous()
    check(cache, mass, table, kept, [50, 0], [0, 0], None)
    fk.fk_kv_compact(cache, table.to(DEV), kept[:, :, :0].contiguous().to(DEV), ints([0, 0]))


def test_rows_outside_are_left_out():
    cache, table, mass, _, _ = make([64], 2, 64, 16, 6)
    was = [getattr(cache, n).clone() for n in NAMES]
    kept = torch.tensor([0, 5, -1, 70, 1 << 30, 2 ** 31 - 1, -2 ** 31, 9], dtype=torch.int32, device=DEV).view(1, 1, -1)
    fk.fk_kv_compact(cache, table.to(DEV), kept, ints([100]))                             # more than there are: 8
    for n, x in zip(NAMES, was):
        flat = x[table[0].long()].transpose(0, 1).flatten(1, 2)
        for j, p in ((1, 5), (7, 9)):
            flat[:, j] = flat[:, p]
        assert torch.equal(bits_of(getattr(cache, n)[table[0].long()].transpose(0, 1).flatten(1, 2)), bits_of(flat))
    now = [getattr(cache, n).clone() for n in NAMES]
    far = torch.tensor([[3, -1, 1 << 30, 7]], dtype=torch.int32, device=DEV)
    for start in (-1000, 2 ** 31 - 1, -2 ** 31, 64):                                      # all rows outside the table
        fk.fk_kv_compact(cache, table.to(DEV), kept, ints([8]), start=ints([start]))
    fk.fk_kv_compact(cache, table.to(DEV), kept, ints([8]), to_pages=far[:, 1:2].contiguous())
    fk.fk_kv_compact(cache, far[:, 1:3].contiguous(), kept, ints([8]))
    fk.fk_kv_compact(cache, table.to(DEV), kept, ints([-3]))
    assert all(torch.equal(bits_of(getattr(cache, n)), bits_of(x)) for n, x in zip(NAMES, now))


def test_many_sequences():
    lens = [20 + 7 * b % 60 for b in range(200)]
    keep = [1 + b * 3 % L for b, L in enumerate(lens)]
    cache, table, mass, _, g = make(lens, 2, 32, 16, 7)
    check(cache, mass, table, places(lens, keep, 2, g), keep, [0] * 200, None)


def test_a_graph_and_another_stream():
    lens = [700, 300]
    cache, table, mass, more, g = make(lens, 2, 128, 32, 8, more=2 * 10)
    kept, tb, to = places(lens, [300, 200], 2, g).to(DEV), table.to(DEV), more.view(2, 10).to(DEV)
    counts = ints([300, 200])
    fk.fk_kv_compact(cache, tb, kept, counts, to_pages=to, mass=mass)
    want = [getattr(cache, n).clone() for n in NAMES] + [mass.clone()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        fk.fk_kv_compact(cache, tb, kept, counts, to_pages=to, mass=mass)
    for _ in range(3):
        for n in NAMES:
            getattr(cache, n)[to.long()] = 0
        mass[to.long()] = 0
        graph.replay()
        torch.cuda.synchronize()
        # (what the first call wrote; the rest of the pages is cleared)
        for n, x in zip(NAMES + ("mass",), want):
            y = getattr(cache, n, None) if n != "mass" else mass
            for b, c in enumerate([300, 200]):
                a = torch.arange(c, device=DEV)
                at = (to[b, a // 32].long(), slice(None), a % 32)
                assert torch.equal(bits_of(x[at]), bits_of(y[at]))
