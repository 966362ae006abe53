"""GPU checks of the paged attention over long contexts and in every form, held to
the error that it should have (tests/paged_norms.py): tables of pages past 64
tiles, long shares, results joined from many parts, and P as a pair of bf16 values
where rows are few."""

import math

import pytest
import torch

from paper_2607_15105_amd import hga
from tests import paged_norms as pn
from tests.test_gpu_paged import BF, F32, _cache, _cfg, _context, _fill_table, _rows, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    hga.lib()


def _attend(cfg, cache, Q, first, begin, max_rows):
    n = Q.shape[0]
    O, lse = torch.full_like(Q, 7.0), torch.full((n, cfg.n_q_heads), 7.0, device="cuda")
    ws = torch.full((hga.paged_workspace_size(cfg, n, max_rows),), 255, dtype=torch.uint8, device="cuda")
    hga.attend_paged_fwd(cfg, cache, Q, _rows(first), _rows(begin), O, lse, ws, max_rows)
    torch.cuda.synchronize()
    return O.cpu(), lse.cpu()


def _check(cfg, cache, Q, first, begin, Kd, Vd, max_rows, what, only=None):
    """The call's rows, each with the bounds of the form that it runs: P is a pair up to
    16 rows x heads, or 64 with d = 64, of the most that a sequence may have, and
    in sequences of at most 16 beside such. Returns (O, O64) of the rows looked at."""
    O, lse = _attend(cfg, cache, Q, first, begin, max_rows)
    G, page, table = cfg.n_q_heads // cfg.n_kv_heads, cache.desc.page_size, cache.page_table.cpu()
    bf16 = Q.dtype == BF
    most = min(max_rows, Q.shape[0]) * G
    out, worst = [], [0.0, 0.0]
    for s in range(len(begin)):
        a, b = first[s], first[s + 1]
        if b <= a or (only is not None and s not in only):
            continue
        entry = table[s][torch.arange(Kd[s].shape[0]) // page]
        ok = (entry >= 0) & (entry < cache.desc.n_pages)
        ref = pn.reference(Q[a:b].cpu(), Kd[s], Vd[s], ok, begin[s] + torch.arange(b - a), 1 / math.sqrt(cfg.head_dim))
        few = most <= (64 if cfg.head_dim == 64 else 16) or ((b - a) * G <= 16 and len(begin) > 1)
        eo, ez = pn.excess(O[a:b], lse[a:b], ref, bf16, few)
        worst = [max(worst[0], eo), max(worst[1], ez)]
        assert eo <= 1 and ez <= 1, (what, s, eo, ez)
        out.append((O[a:b], ref[0], few))
    say(f"   {what}: O {worst[0]:.3f}, lse {worst[1]:.3f} of the bounds")
    return out


@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F32, 64)])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("rows", [1, 5, 16, 100])
def test_long_contexts(dtype, d, e4m3, rows):
    """One context of 20,011 positions and a row beside it: hundreds of shares, tables of
    pages for 313 tiles of 64 keys; a few pages absent."""
    say(f"[attend] norms, {dtype}, d {d}, e4m3 {e4m3}, {rows} rows over 20,011")
    gen = torch.Generator().manual_seed(51)
    cfg = _cfg(4, 1, d, dtype)
    ctx = [20011, 300]
    cache = _cache(cfg, 2, 640, 700, 32, e4m3, "head", fill=0xFF)
    _fill_table(cache, ctx, gen)
    Kd, Vd = _context(cfg, cache, ctx, gen, e4m3)
    cache.page_table[0, 400:403] = -1
    Q = torch.randn(rows + 1, 4, d, generator=gen).to(dtype).cuda()
    first, begin = [0, rows, rows + 1], [ctx[0] - rows, 299]
    for max_rows in sorted({1, rows}):
        _check(cfg, cache, Q, first, begin, Kd, Vd, max_rows, f"max_rows {max_rows}")


@pytest.mark.parametrize("rows", [3, 70])
@pytest.mark.parametrize("e4m3", [False, True])
def test_contexts_of_the_largest_pages(rows, e4m3):
    say(f"[attend] norms, {rows} rows over 65,737, e4m3 {e4m3}")
    gen = torch.Generator().manual_seed(52)
    cfg = _cfg(2, 1, 64, BF)
    cache = _cache(cfg, 1, 2, 3, 65536, e4m3, "head", fill=0xFF)
    cache.page_table.copy_(torch.tensor([[2, 0]]))
    ctx = 65536 + 201
    Kd, Vd = _context(cfg, cache, [ctx], gen, e4m3)
    Q = torch.randn(rows, 2, 64, generator=gen).to(BF).cuda()
    _check(cfg, cache, Q, [0, rows], [ctx - rows], Kd, Vd, rows, "large pages")


@pytest.mark.parametrize("d,rows,e4m3", [(64, 1, True), (64, 3, False), (128, 1, False), (128, 9, True)])
def test_shares_of_hundreds_of_tiles(d, rows, e4m3):
    """64 sequences over the same 20,000 positions, so that a workgroup follows one
    context over hundreds of tiles and look-ups of 64 of them."""
    say(f"[attend] norms, long shares, d {d}, {rows} rows, e4m3 {e4m3}")
    gen = torch.Generator().manual_seed(53)
    cfg = _cfg(16, 2, d, BF)
    ctx, S = 20000, 64
    cache = _cache(cfg, S, 157, 158, 128, e4m3, "token", fill=0xFF)
    _fill_table(cache, [ctx] + [0] * (S - 1), gen)
    Kd, Vd = _context(cfg, cache, [ctx] + [0] * (S - 1), gen, e4m3)
    cache.page_table[1:] = cache.page_table[0]
    cache.page_table[40, 70] = -1
    Q = torch.randn(rows * S, 16, d, generator=gen).to(BF).cuda()
    begin = [ctx - rows - 37 * s for s in range(S)]
    _check(cfg, cache, Q, [rows * s for s in range(S + 1)], begin, [Kd[0]] * S, [Vd[0]] * S, rows, "long shares",
           only=(0, 7, 40, 63))


@pytest.mark.parametrize("d,hq,hkv,rows", [(128, 8, 2, [1] * 9), (128, 4, 4, [16, 9, 1, 12]), (64, 8, 2, [1, 4, 2, 4]),
                                           (64, 8, 1, [8, 5, 1, 7]), (128, 8, 2, [300, 1, 4, 3, 2, 4, 4]),
                                           (64, 8, 2, [140, 1, 4, 3, 2, 4, 4])])
@pytest.mark.parametrize("e4m3", [False, True])
def test_few_rows_have_p_as_a_pair(d, hq, hkv, rows, e4m3):
    """Over the rows of the forms of 16 and 32 (alone, or beside a chunk) the error is
    that of rounding O."""
    say(f"[attend] pairs, {hq}/{hkv} heads, d {d}, rows {rows}, e4m3 {e4m3}")
    gen = torch.Generator().manual_seed(54)
    cfg = _cfg(hq, hkv, d, BF)
    ctx = [700 + 150 * s for s in range(len(rows))]
    cache = _cache(cfg, len(rows), 30, sum(-(-c // 64) for c in ctx), 64, e4m3, "head", fill=0xFF)
    _fill_table(cache, ctx, gen)
    Kd, Vd = _context(cfg, cache, ctx, gen, e4m3)
    first = [0]
    for r in rows:
        first.append(first[-1] + r)
    Q = torch.randn(first[-1], hq, d, generator=gen).to(BF).cuda()
    got = _check(cfg, cache, Q, first, [c - r for c, r in zip(ctx, rows)], Kd, Vd, max(rows), "pairs")
    few = [(o, z) for o, z, pair in got if pair]
    assert len(few) >= len(rows) - 1
    ratio = pn.rounding_ratio(torch.cat([o for o, _ in few]), torch.cat([z for _, z in few]))
    say(f"   {ratio:.4f} of the rounding's error")
    assert ratio < 1.1
