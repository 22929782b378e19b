"""fk_kv_weigh with rows whose lse is -inf: they add nothing, whatever their queries hold and whatever the keys that they alone see, as the padded
rows of a batch.  Comparison and tolerance as in test_gpu_kv_weigh.py."""
import math

import pytest
import torch

from paper_2603_09229_amd import binding as fk
from tests import evict_plain as plain
from tests import kv_plain
from tests.test_gpu_kv_attend import BF16, DEV, F16, make
from tests.test_gpu_kv_weigh import ints

pytestmark = pytest.mark.gpu


def run(t, L, n, H, G, d, dead, fill, causal=True, window=0):
    """dead: of the n queries."""
    cache, q, table, starts = make(t, [L], [n], H, G, d, 16, n + d)
    k = kv_plain.values(cache.k_codes, cache.k_scale, cache.k_levels)
    sees = plain.row_sees(L, n, causal, window)
    lse = plain.attend(k, k, q, table, [L], starts, d ** -0.5, [sees])[1].float()
    lse[dead] = -math.inf
    q[dead] = 0
    mass = torch.rand(cache.pages, H, 16, generator=torch.Generator().manual_seed(n)).to(DEV)
    want, bound = plain.weigh(k, q, lse, table, [L], starts, d ** -0.5, [sees], [L], 0.5, mass, mass)
    print(f"weigh {t} L={L} n={n} H={H} G={G} d={d} dead={len(dead)} fill={fill} causal={causal} window={window}", flush=True)
    q[dead] = fill
    live = torch.ones(n, dtype=torch.bool)
    live[dead] = False
    unseen = (~sees[live].any(0)).nonzero().flatten().to(DEV)     # by a row that adds anything
    cache.k_scale[table[0, unseen // 16].long(), :, unseen % 16] = math.nan
    fk.fk_kv_weigh(cache, q, lse, table, ints([L]), mass, q_start=ints(starts), max_q=n, max_len=L, scale=d ** -0.5, causal=causal, window=window,
                   decay=0.5)
    assert not mass.isnan().any()
    assert ((mass.double() - want).abs() <= bound).all()


def patterns(n):
    return [list(range(0, n, 3)), list(range(n - (n + 3) // 4, n)), list(range(n)), [n // 2]]


@pytest.mark.parametrize("fill", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("t,L,n,H,G,d", [(F16, 300, 1, 2, 4, 64), (BF16, 500, 20, 2, 3, 128), (F16, 200, 9, 1, 5, 256), (BF16, 900, 64, 1, 2, 64)])
def test_few_rows(t, L, n, H, G, d, fill):
    for dead in patterns(n):
        run(t, L, n, H, G, d, dead, fill)
        run(t, L, n, H, G, d, dead, fill, causal=False)
        run(t, L, n, H, G, d, dead, fill, window=40)


@pytest.mark.parametrize("fill", [math.nan, math.inf])
@pytest.mark.parametrize("t,L,n,H,G,d", [(BF16, 1500, 300, 2, 4, 128), (F16, 1200, 500, 1, 3, 64), (F16, 900, 150, 1, 4, 256), (BF16, 900, 150, 2, 4, 160),
                                         (F16, 700, 3, 1, 200, 128)])
def test_rows_that_stream_by(t, L, n, H, G, d, fill):
    for dead in patterns(n):
        run(t, L, n, H, G, d, dead, fill)
        run(t, L, n, H, G, d, dead, fill, causal=False)
    run(t, L, n, H, G, d, patterns(n)[0], fill, window=100)
