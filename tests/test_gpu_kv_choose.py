"""fk_kv_choose against a sort on the host, place by place: ties, infinities, NaN and zeros of both signs, lengths around `keep`, protected ends,
short and long sequences."""
import math

import pytest
import torch

from paper_2603_09229_amd import binding as fk
from tests import evict_plain as plain
from tests import kv_plain

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")


def make(lens, H, P, seed, kind="normal", spare=2):
    g = torch.Generator().manual_seed(seed)
    held = [max(1, -(-L // P)) for L in lens]
    pages = sum(held) + spare
    order = torch.randperm(pages, generator=g).to(torch.int32)
    table = torch.full((len(lens), max(held) + 1), 1 << 30, dtype=torch.int32)
    at = 0
    for b, n in enumerate(held):
        table[b, :n] = order[at:at + n]
        at += n
    mass = torch.randn(pages, H, P, generator=g)
    if kind == "ties":
        mass = torch.randint(-2, 3, mass.shape, generator=g).float() * 0.25
    elif kind == "equal":
        mass.fill_(0.125)
    elif kind == "close":                                         # values that differ in their last bits only
        mass = (0x3f800000 + torch.randint(0, 40, mass.shape, generator=g, dtype=torch.int32)).view(torch.float32)
    elif kind == "odd":
        pick = torch.tensor([0.0, -0.0, math.inf, -math.inf, math.nan, -math.nan, 1e-42, -1e-42, 3e38, -3e38, 1.0, -1.0])
        mass = pick[torch.randint(0, len(pick), mass.shape, generator=g)]
    elif kind == "weights":
        mass = (1.5 * mass).exp()
    lv = kv_plain.levels(H, torch.float16, 1, DEV)
    return fk.KVCache.empty(pages, P, lv, lv, 32), mass, table


def run(lens, H, P, keep, first=0, last=0, kind="normal", seed=0, max_len=0):
    cache, mass, table = make(lens, H, P, seed, kind)
    print(f"choose lens={lens[:6]} H={H} P={P} keep={keep} first={first} last={last} {kind}", flush=True)
    kept, counts = fk.fk_kv_choose(cache, mass.to(DEV), table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), keep, first=first,
                                   last=last, max_len=max_len)
    want = plain.choose(mass, table, lens, P, keep, first, last)
    assert torch.equal(counts.cpu(), want[1])
    assert torch.equal(kept.cpu(), want[0])


@pytest.mark.parametrize("kind", ["normal", "ties", "equal", "close", "odd", "weights"])
def test_values(kind):
    run([700, 300, 90], 3, 16, 100, 4, 30, kind)
    run([3000], 1, 64, 1700, 0, 0, kind, seed=1)
    run([3000, 2000], 2, 32, 5, 1, 1, kind, seed=2)


@pytest.mark.parametrize("L", [0, 1, 2, 15, 16, 17, 63, 64, 65, 255, 256, 257, 1023, 1024, 1025, 2047, 2049, 4095, 4096, 4097])
def test_lengths(L):
    for keep in sorted({1, 2, max(1, L // 3), max(1, L - 1), max(1, L), L + 1}):
        run([L], 1, 16, keep, 0, 0, "ties", seed=L)
        run([L, 7], 1, 16, keep, keep // 3, keep // 2, "weights", seed=L)


def test_protected_ends_alone():
    run([500, 40, 41], 2, 16, 40, 10, 30, "odd")                  # nothing is chosen by weight
    run([500], 2, 16, 40, 40, 0)
    run([500], 2, 16, 40, 0, 40)


@pytest.mark.parametrize("L", [9000, 20000, 40000])
@pytest.mark.parametrize("kind", ["normal", "ties", "equal", "close"])
def test_long_sequences(L, kind):
    run([L, L // 2, 77], 2, 64, L // 5, 16, 100, kind, seed=L)
    run([L], 1, 256, L - 3, 0, 1, kind, seed=L)


def test_a_wrong_upper_bound_of_the_lengths_costs_time_only():
    run([9000, 100], 1, 64, 800, 4, 4, max_len=300)
    run([9000, 100], 1, 64, 800, 4, 4, max_len=9000)


def test_many_sequences():
    run([1 + 37 * b % 300 for b in range(300)], 3, 16, 64, 4, 16, "weights")


def test_very_long_sequences_by_their_sorted_weights():
    L, keep = 300000, 50000
    cache, _, table = make([L], 2, 256, 5)
    for kind in ("weights", "equal", "few"):
        g = torch.Generator().manual_seed(3)
        flat = torch.randn(2, L, generator=g).exp() if kind == "weights" else torch.full((2, L), 0.5)
        if kind == "few":
            flat = torch.randint(0, 7, (2, L), generator=g).float()
        mass = torch.zeros(cache.pages, 2, 256)
        t = torch.arange(L)
        mass[table[0, t // 256].long(), :, t % 256] = flat.T.contiguous()
        kept, counts = fk.fk_kv_choose(cache, mass.to(DEV), table.to(DEV), torch.tensor([L], dtype=torch.int32, device=DEV), keep, first=10,
                                       last=500, max_len=L)
        order = flat[:, 10:L - 500].sort(dim=1, descending=True, stable=True).indices[:, :keep - 510] + 10
        want = torch.cat([torch.arange(10).expand(2, 10), order, torch.arange(L - 500, L).expand(2, 500)], dim=1).sort(dim=1).values
        short = fk.fk_kv_choose(cache, mass.to(DEV), table.to(DEV), torch.tensor([L], dtype=torch.int32, device=DEV), keep, first=10, last=500,
                                max_len=40000)                    # a wrong bound: fewer parts, each in several rounds
        assert torch.equal(short[0], kept)
        assert torch.equal(kept[0].cpu(), want.int()) and counts.item() == keep


def test_a_graph_and_a_used_workspace():
    cache, mass, table = make([30000, 500], 2, 64, 4, "weights")
    m, tb, lens = mass.to(DEV), table.to(DEV), torch.tensor([30000, 500], dtype=torch.int32, device=DEV)
    first = [x.clone() for x in fk.fk_kv_choose(cache, m, tb, lens, 300, first=4, last=20, max_len=30000)]
    n = fk.fk_kv_choose_workspace_bytes(cache, 2, 30000)
    ws = torch.full((n + 4096,), 91, dtype=torch.uint8, device=DEV)
    kept, counts = torch.empty_like(first[0]), torch.empty_like(first[1])
    call = lambda: fk.fk_kv_choose(cache, m, tb, lens, 300, first=4, last=20, max_len=30000, kept=kept, counts=counts, ws=ws[:n])  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        call()
        with torch.cuda.graph(graph, stream=side):
            call()
    for fill in (0, 255, 17, 0):
        ws[:n].fill_(fill)
        kept.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(kept, first[0]) and torch.equal(counts, first[1]) and (ws[n:] == 91).all()
