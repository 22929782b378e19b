"""Drafted trees, accepted branches, attention weights and evictions together, as kv_cache.Server makes the calls: every result against a plain
model that keeps, for each sequence and head, what the cache should hold."""
import math

import pytest
import torch

from paper_2603_09229_amd import kv_cache
from tests import evict_plain as plain
from tests import kv_plain

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda:0")
TREE = [-1, -1, 0, 0, 1, 2, 2]
BRANCHES = [[0, 2, 6], [], [1, 4], [0, 3], [1]]


def values(server):
    c = server.cache
    return kv_plain.values(c.k_codes, c.k_scale, c.k_levels), kv_plain.values(c.v_codes, c.v_scale, c.v_levels)


def rows_of(x, server, b, L):
    """What sequence b's first L places hold, [heads, L, ...]."""
    return x[server.pages[b].long()].transpose(0, 1).flatten(1, 2)[:, :L]


def check(out, want, mag, err, dtype):
    step = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -11        # as in test_gpu_kv_attend.py
    assert ((out.double() - want).abs() <= step * 1.01 * want.abs() + (2.0 ** -10 + 2 * err[..., None]) * mag + 2.0 ** -24).all()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_drafts_branches_and_evictions(dtype):
    g = torch.Generator().manual_seed(3)
    H, G, d, counts, keep, first, last = 2, 4, 64, [130, 20, 77], 60, 4, 10
    lv = [kv_plain.levels(H, dtype, 7, DEV), kv_plain.levels(H, dtype, 8, DEV)]
    server = kv_cache.Server(*lv, d, 3, 160, page_size=16, max_pos=400, weights=True)
    draw = lambda n, h: torch.randn(n, h, d, generator=g).to(dtype).to(DEV)  # noqa: E731
    scale = 1 / math.sqrt(d)
    server.step(draw(sum(counts), H * G), draw(sum(counts), H), draw(sum(counts), H), counts)
    total = [float(c * G) for c in counts]                            # weight that a sequence's heads have been given
    at = list(counts)                                                 # positions
    for i in range(6):
        trees = [TREE[:3 + i], TREE, TREE[:1]]
        ns = [len(t) for t in trees]
        starts = [sum(ns[:b]) for b in range(4)]
        q, k, v = draw(sum(ns), H * G), draw(sum(ns), H), draw(sum(ns), H)
        held = server.lens.tolist()
        out = server.draft(q, k, v, trees)
        assert server.lens.tolist() == held
        masks, depths = kv_cache.tree_masks(trees)
        pos = torch.tensor([at[b] + depths[starts[b] + j] for b in range(3) for j in range(ns[b])], device=DEV)
        qt = kv_plain.turned(q, server.cos_sin, pos, False)
        lens = [L + n for L, n in zip(held, ns)]
        sees = [plain.tree_sees([m[0] for m in masks[s:s + n].tolist()], L, n, 0) for s, n, L in zip(starts, ns, lens)]
        kk, vv = values(server)
        want, _, mag, err = plain.attend(kk, vv, qt, server.pages, lens, starts, scale, sees)
        check(out, want, mag, err, dtype)

        branches = [[j for j in BRANCHES[(i + b) % 5] if j < len(t)] for b, t in enumerate(trees)]
        branches = [br if all(t[j] == p for p, j in zip([-1] + br, br)) else [] for br, t in zip(branches, trees)]
        was = [x.clone() for x in (server.cache.k_codes, server.cache.v_codes)]
        server.accept(branches)
        assert server.lens.tolist() == [L + len(br) for L, br in zip(held, branches)]
        for b, br in enumerate(branches):
            for x, now in zip(was, (server.cache.k_codes, server.cache.v_codes)):
                old = rows_of(x, server, b, held[b] + ns[b])
                assert torch.equal(rows_of(now, server, b, held[b] + len(br)), torch.cat([old[:, :held[b]], old[:, [held[b] + j for j in br]]], 1))
            total[b] += len(br) * G
            at[b] += len(br)
            # weights of every query add up to 1: in 32 bits, with scores below 2^5, to 2^-17 of it (two roundings of 2^-24 of the exponent, 2^6
            # powers of two, and a sum of some hundred numbers)
            mine = rows_of(server.mass, server, b, server.lens[b].item()).double().sum(1)
            assert ((mine - total[b]).abs() <= 2.0 ** -17 * total[b]).all()
        if i in (2, 5):
            lens = server.lens.tolist()
            weights = [rows_of(server.mass, server, b, L).cpu() for b, L in enumerate(lens)]
            codes = [rows_of(server.cache.k_codes, server, b, L).cpu() for b, L in enumerate(lens)]
            server.evict(keep, first, last)
            assert server.lens.tolist() == [min(L, keep) for L in lens]
            for b, L in enumerate(lens):
                n = min(L, keep)
                kept, _ = plain.choose(weights[b].T[:, :, None].contiguous(), torch.arange(L)[None], [L], 1, keep, first, last)
                for h in range(H):
                    stay = kept[0, h, :n].long()
                    assert torch.equal(rows_of(server.mass, server, b, n)[h].cpu(), weights[b][h, stay])
                    assert torch.equal(rows_of(server.cache.k_codes, server, b, n)[h].cpu(), codes[b][h, stay])
                total[b] = rows_of(server.mass, server, b, n).double().sum(1) if L > keep else total[b]
    assert server.gone.tolist() == [a - L for a, L in zip(at, server.lens.tolist())] and max(server.gone.tolist()) > 0
    # a step after all of this: positions run on
    q, k, v = draw(3, H * G), draw(3, H), draw(3, H)
    out = server.step(q, k, v, [1, 1, 1])
    qt = kv_plain.turned(q, server.cos_sin, torch.tensor(at, device=DEV), False)
    lens = server.lens.tolist()
    want, _, mag, err = kv_plain.attend(*values(server), qt, server.pages, lens, [0, 1, 2, 3], scale, True, 0)
    check(out, want, mag, err, dtype)


def test_weights_do_not_change_what_a_step_gives():
    g = torch.Generator().manual_seed(5)
    lv = [kv_plain.levels(2, torch.float16, s, DEV) for s in (1, 2)]
    torch.manual_seed(0)
    plain_server = kv_cache.Server(*lv, 64, 2, 100, page_size=16)
    torch.manual_seed(0)
    weighing = kv_cache.Server(*lv, 64, 2, 100, page_size=16, weights=True)
    for c in ([30, 50], [1, 1], [3, 0]):
        x = [torch.randn(sum(c), h, 64, generator=g).half().to(DEV) for h in (8, 2, 2)]
        assert torch.equal(plain_server.step(*x, c), weighing.step(*x, c))


def test_the_example():
    result = kv_cache.demo_eviction(batch=2, heads=1, group=2, prompt=150, steps=12, keep=64)
    assert 0 < result["share"] <= 1.001 and result["held"] <= 150 + 6
