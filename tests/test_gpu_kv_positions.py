"""kv_cache.Server past an eviction with the number of positions that it has by default: results as long as there are angles, a refusal behind
them.  Comparison and tolerance as in test_gpu_kv_drafts.py."""
import math

import pytest
import torch

from paper_2603_09229_amd import kv_cache
from tests import evict_plain as plain
from tests import kv_plain
from tests.test_gpu_kv_drafts import DEV, check, values

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_a_server_without_max_pos_evicts_and_stops_at_its_last_angle(dtype):
    g = torch.Generator().manual_seed(11)
    H, G, d, max_len = 2, 4, 64, 90
    server = kv_cache.Server(*[kv_plain.levels(H, dtype, s, DEV) for s in (7, 8)], d, 2, max_len, page_size=16, weights=True)
    draw = lambda n: [torch.randn(n, h, d, generator=g).to(dtype).to(DEV) for h in (H * G, H, H)]  # noqa: E731
    server.step(*draw(80 + 60), [80, 60])
    server.evict(50, 4, 10)
    assert server.lens.tolist() == [50, 50] and server.gone.tolist() == [30, 10]
    for i in range(10):                                           # positions 80 to 89 and 60 to 69
        q, k, v = draw(2)
        out = server.step(q, k, v, [1, 1])
        qt = kv_plain.turned(q, server.cos_sin, torch.tensor([80 + i, 60 + i], device=DEV), False)
        want, _, mag, err = kv_plain.attend(*values(server), qt, server.pages, [51 + i, 51 + i], [0, 1, 2], 1 / math.sqrt(d), True, 0)
        check(out, want, mag, err, dtype)
    was = [x.clone() for x in (server.cache.k_codes, server.mass, server.lens, server.gone)]
    for call in (lambda: server.step(*draw(2), [1, 1]), lambda: server.draft(*draw(2), [[-1], [-1]])):
        with pytest.raises(ValueError, match=r"sequences \[0\] would pass position 90"):
            call()
    assert all(torch.equal(x, y) for x, y in zip(was, (server.cache.k_codes, server.mass, server.lens, server.gone)))
    assert server.step(*draw(1), [0, 1]).isfinite().all()         # the other one goes on


def test_a_wide_tree_up_to_the_last_angle():
    g = torch.Generator().manual_seed(12)
    H, G, d = 2, 4, 64
    server = kv_cache.Server(*[kv_plain.levels(H, torch.float16, s, DEV) for s in (7, 8)], d, 1, 80, page_size=16, max_pos=83, weights=True)
    draw = lambda n: [torch.randn(n, h, d, generator=g).half().to(DEV) for h in (H * G, H, H)]  # noqa: E731
    server.step(*draw(80), [80])
    server.evict(50, 4, 10)
    tree = [-1] * 10 + list(range(10)) + list(range(10, 20))      # 30 tokens, positions 80 to 82
    q, k, v = draw(30)
    out = server.draft(q, k, v, [tree])
    masks, depths = kv_cache.tree_masks([tree])
    assert max(depths) == 2
    qt = kv_plain.turned(q, server.cos_sin, torch.tensor([80 + x for x in depths], device=DEV), False)
    sees = [plain.tree_sees([m[0] for m in masks.tolist()], 80, 30, 0)]
    want, _, mag, err = plain.attend(*values(server), qt, server.pages, [80], [0, 30], 1 / math.sqrt(d), sees)
    check(out, want, mag, err, torch.float16)
    server.accept([[3, 13, 23]])
    with pytest.raises(ValueError, match="position 83"):
        server.step(*draw(1), [1])
