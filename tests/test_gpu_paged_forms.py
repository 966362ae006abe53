"""GPU checks of the float32 attention over the paged cache on both sides of the rule
that chooses how many rows are taken at a time: chunks between and beside the sizes
where it changes, with tables of few and of many positions."""

import math

import pytest
import torch

from paper_2607_15105_amd import hga
from tests import paged_norms as pn
from tests.test_gpu_paged import F32, _cache, _cfg, _context, _fill_table, _rows, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    hga.lib()


@pytest.mark.parametrize("rows", [[15, 1, 0], [17, 4, 17], [33, 1, 40], [255, 3, 64], [256, 0, 1], [257, 5, 1]])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("cap", [40, 400])
def test_float32_chunks(rows, e4m3, cap):
    """Four query heads to a kv head: 60 to 1,028 rows x heads of the longest sequence,
    three sequences of two kv heads, pages of 16: 3,840 rows of K, or 38,400."""
    say(f"[attend] float32 chunks, rows {rows}, e4m3 {e4m3}, {16 * cap} positions")
    gen = torch.Generator().manual_seed(61)
    cfg = _cfg(8, 2, 64, F32)
    ctx = [600, 333, 290] if cap < 100 else [6001, 333, 2900]
    cache = _cache(cfg, 3, cap, 600, 16, e4m3, "token", fill=0xFF)
    _fill_table(cache, ctx, gen)
    Kd, Vd = _context(cfg, cache, ctx, gen, e4m3)
    cache.page_table[0, 5:8] = -1
    first = [1]
    for r in rows:
        first.append(first[-1] + r)
    n = first[-1] + 1
    Q = torch.randn(n, 8, 64, generator=gen).cuda()
    begin = [c - r for c, r in zip(ctx, rows)]
    for max_rows in (max(rows), n):
        O, lse = torch.full_like(Q, 7.0), torch.full((n, 8), 7.0, device="cuda")
        ws = torch.full((hga.paged_workspace_size(cfg, n, max_rows),), 255, dtype=torch.uint8, device="cuda")
        hga.attend_paged_fwd(cfg, cache, Q, _rows(first), _rows(begin), O, lse, ws, max_rows)
        torch.cuda.synchronize()
        table = cache.page_table.cpu()
        for s in range(3):
            a, b = first[s], first[s + 1]
            if a == b:
                continue
            ok = table[s][torch.arange(ctx[s]) // 16] >= 0
            ref = pn.reference(Q[a:b].cpu(), Kd[s], Vd[s], ok, begin[s] + torch.arange(b - a), 1 / math.sqrt(64))
            eo, ez = pn.excess(O[a:b].cpu(), lse[a:b].cpu(), ref, False, False)
            assert eo <= 1 and ez <= 1, (max_rows, s, eo, ez)
        for x in (O, lse):  # of no sequence
            assert bool((x[0] == 7).all()) and bool((x[-1] == 7).all())
