"""GPU checks of the paged cache at the ends of the values' range: the largest
finite ones through the 8-bit format, and what is not finite in V where it is
attended, in tiles with and without masks, against float64 on the CPU."""

import math

import pytest
import torch

from paper_2607_15105_amd import hga
from tests import paged_oracle as po
from tests.test_gpu_paged import BF, F32, _attend_check, _cache, _cfg, _context, _fill_table, _held_rows, _rows, say

pytestmark = pytest.mark.gpu

TOP = 240 * 2.0 ** 120  # the largest value of four significant bits below 2^128


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    hga.lib()


# ---------------------------------------------------------------- the largest finite values in 8 bits

@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F32, 64)])
@pytest.mark.parametrize("layout", ["head", "token"])
def test_the_largest_finite_values_stay_finite(dtype, d, layout):
    """Rows whose largest magnitude lies around 224, 240 and 248 times 2^120 and at
    the type's maximum: held as the values up to TOP are, those over it as TOP."""
    say(f"[write, read] largest values, {dtype}, d {d}, {layout}")
    gen = torch.Generator().manual_seed(41)
    cfg = _cfg(2, 2, d, dtype)
    tops = [torch.finfo(dtype).max, 255 * 2.0 ** 120, 249 * 2.0 ** 120, 248 * 2.0 ** 120, 247 * 2.0 ** 120,
            241 * 2.0 ** 120, TOP, 232 * 2.0 ** 120, 225 * 2.0 ** 120, 224 * 2.0 ** 120, 223 * 2.0 ** 120]
    n = 2 * len(tops)
    x = torch.randn(n, 2, d, generator=gen) * 2.0 ** 118
    for i, v in enumerate(tops):
        x[2 * i, :, 3], x[2 * i + 1, :, 7] = v, -v
        x[2 * i, 1, 20:28] = torch.tensor(tops[:8]).clamp(max=v)  # several of them in one row
    x = x.to(dtype)
    cache = _cache(cfg, 1, 4, 4, 16, True, layout)
    _fill_table(cache, [n], gen)
    hga.cache_write(cfg, cache, x.cuda(), -x.cuda(), _rows([0, n]), _rows([0]))
    out = torch.full((2, n, 2, d), 7.0, dtype=dtype, device="cuda")
    hga.cache_read(cfg, cache, out[0], out[1], _rows([0, n]), _rows([0]))
    torch.cuda.synchronize()
    exact = x.double()
    code, e = po.held(exact.clamp(-TOP, TOP))
    want = code * torch.exp2(e)[..., None]
    assert bool(torch.isfinite(want).all()) and bool((want.abs() <= TOP).all())
    # the promise about them: 2^-4 relative, or 2^(e - 10) where that is more
    assert bool(((want - exact).abs() <= torch.maximum(exact.abs() * 2.0 ** -4, torch.exp2(e - 10)[..., None])).all())
    for sign, got in ((1.0, out[0]), (-1.0, out[1])):
        assert torch.equal(sign * got.double().cpu(), want), float(got.float().abs().max())


@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F32, 64)])
@pytest.mark.parametrize("max_rows", [1, 5, 140])
def test_attention_of_the_largest_finite_values(dtype, d, max_rows):
    """Values of the type's maximum at keys of weight e^-5 beside others, in tiles
    that are masked for some of the rows and not for others."""
    say(f"[attend] largest values, {dtype}, d {d}, max_rows {max_rows}")
    gen = torch.Generator().manual_seed(42)
    cfg = _cfg(4, 2, d, dtype)
    ctx, rows = 300, 140
    cache = _cache(cfg, 1, 20, 20, 16, True, "head")
    _fill_table(cache, [ctx], gen)
    K, V = torch.zeros(ctx, 2, d), torch.randn(ctx, 2, d, generator=gen)
    top = torch.finfo(dtype).max
    for t, h, i, v in ((3, 0, 5, top), (70, 1, 6, -top), (200, 0, 7, top), (201, 1, 8, -top)):
        K[t, h] = -5.0 / math.sqrt(d)
        V[t, h, i] = v
    K, V = K.to(dtype), V.to(dtype)
    hga.cache_write(cfg, cache, K.cuda(), V.cuda(), _rows([0, ctx]), _rows([0]))
    Kd, Vd = (_held_rows(cfg, x.double().clamp(-TOP, TOP), True) for x in (K, V))
    Q = torch.ones(rows, 4, d, dtype=dtype, device="cuda")
    O, _ = _attend_check(cfg, cache, Q, [0, rows], [ctx - rows], [Kd], [Vd], max_rows, what="largest values")
    assert bool(torch.isfinite(O).all()) and float(O.float().abs().max()) > 1e30


# ---------------------------------------------------------------- what is not finite in V, where it is attended

def _attend_not_finite(cfg, cache, Q, begin, Kd, Vd, max_rows, what):
    """One sequence's rows over K, V [L, Hkv, d] in float64, V with infinities and
    NaN. Of an element of O whose attended values are not all finite the result is
    their sum: an infinity, or NaN; the others are held to their bounds."""
    n, Hq, d = Q.shape
    G = Hq // Kd.shape[1]
    O, lse = torch.full_like(Q, 7.0), torch.full((n, Hq), 7.0, device="cuda")
    ws = torch.full((hga.paged_workspace_size(cfg, n, max_rows),), 255, dtype=torch.uint8, device="cuda")
    hga.attend_paged_fwd(cfg, cache, Q, _rows([0, n]), _rows([begin]), O, lse, ws, max_rows)
    torch.cuda.synchronize()
    pos = begin + torch.arange(n)
    fine = torch.isfinite(Vd)
    o, z, bo, bl = po.attend(Q.cpu(), Kd, torch.where(fine, Vd, 0.0), torch.ones(len(Kd), dtype=torch.bool), pos,
                             1 / math.sqrt(d), 2.0 ** -8 if Q.dtype == BF else 2.0 ** -24)
    odd = torch.zeros(n, Hq, d, dtype=torch.float64)
    for t in torch.nonzero((~fine).flatten(1).any(1))[:, 0].tolist():
        x = torch.where(fine[t], 0.0, Vd[t]).repeat_interleave(G, 0)
        odd = odd + torch.where((pos >= t)[:, None, None], x, 0.0)
    got = O.double().cpu()
    some = odd != 0  # NaN too
    assert int(some.sum()) > 0 and bool((~some).any())
    same = (got == odd) | (torch.isnan(got) & torch.isnan(odd))
    wrong = torch.nonzero(some & ~same)
    assert len(wrong) == 0, (what, len(wrong), [(i.tolist(), float(got[tuple(i)]), float(odd[tuple(i)])) for i in wrong[:4]])
    assert bool(((got - o).abs() <= bo)[~some].all()), what
    assert bool(((lse.double().cpu() - z).abs() <= bl).all()), what


@pytest.mark.parametrize("dtype,d,heads", [(BF, 128, (4, 2)), (BF, 64, (8, 2)), (F32, 64, (4, 2))])
@pytest.mark.parametrize("ctx,rows", [(300, 140), (3000, 3), (3000, 9), (9000, 70)])
@pytest.mark.parametrize("expected", ["one", "all"])
def test_infinities_in_attended_values(dtype, d, heads, ctx, rows, expected):
    """Infinities and NaN in V of rows that are held as they are, at the beginning, in
    the middle and among the new rows: the same result whether a tile is masked, and in
    every form."""
    say(f"[attend] infinite values, {dtype}, d {d}, {rows} rows over {ctx}, {expected}")
    gen = torch.Generator().manual_seed(43)
    cfg = _cfg(*heads, d, dtype)
    cache = _cache(cfg, 1, -(-ctx // 32), -(-ctx // 32), 32, False, "token")
    _fill_table(cache, [ctx], gen)
    Kd, Vd = _context(cfg, cache, [ctx], gen, False)
    bad = torch.full((ctx, heads[1], d), math.nan, dtype=torch.float64)  # NaN: as it is
    inf, begin = math.inf, ctx - rows
    for t, h, i, v in ((0, 0, 1, inf), (33, 1, 2, -inf), (ctx // 2, 0, 3, inf), (ctx // 2 + 1, 0, 3, -inf),
                       (ctx // 2 + 1, 1, 4, inf), (begin - 1, 0, 5, -inf), (begin, 1, d - 1, inf),
                       (begin + rows // 2, 0, d - 2, -inf), (ctx - 1, 1, d - 3, inf), (64, 1, 2, -inf)):
        bad[t, h, i] = v
        Vd[0][t, h, i] = v
    Vd[0][40, 1, 9] = math.nan  # one NaN, early
    at = torch.nonzero(~torch.isnan(bad) | torch.isnan(Vd[0]))
    page = cache.page_table[0].cpu()
    for t, h, i in at.tolist():
        cache.v[int(page[t // 32]), t % 32, h, i] = float(Vd[0][t, h, i])
    Q = torch.randn(rows, heads[0], d, generator=gen).to(dtype).cuda()
    _attend_not_finite(cfg, cache, Q, begin, Kd[0], Vd[0], 1 if expected == "one" else rows, "infinities")


@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F32, 64)])
@pytest.mark.parametrize("ctx,rows", [(300, 140), (3000, 3)])
@pytest.mark.parametrize("expected", ["one", "all"])
def test_codes_that_stand_for_infinities(dtype, d, ctx, rows, expected):
    """A pool of the caller's making whose codes and scales stand for 2^128: read
    back and attended as the infinity that it is in float32, whether a tile is masked."""
    say(f"[read, attend] infinite codes, {dtype}, d {d}, {rows} rows over {ctx}, {expected}")
    gen = torch.Generator().manual_seed(44)
    cfg = _cfg(4, 2, d, dtype)
    cache = _cache(cfg, 1, -(-ctx // 32), -(-ctx // 32), 32, True, "head")
    _fill_table(cache, [ctx], gen)
    Kd, Vd = _context(cfg, cache, [ctx], gen, True)
    page, begin = cache.page_table[0].cpu(), ctx - rows
    codes = cache.v.view(torch.uint8)
    for t, h in ((5, 0), (100, 1), (begin - 2, 0), (begin + rows // 2, 1)):
        p, o = int(page[t // 32]), t % 32
        codes[p, o, h] = 0
        cache.v_scale[p, h, o] = 120 + 127
        Vd[0][t, h] = 0.0
        for i, c, v in ((t % 11, 0x78, math.inf), (20 + t % 7, 0xF8, -math.inf), (40, 0x7F, math.nan)):
            codes[p, o, h, i] = c
            Vd[0][t, h, i] = v
    for t, h, i, c, v in ((7, 1, 3, 0x7F, math.nan), (begin + 1, 0, 4, 0xFF, math.nan)):
        codes[int(page[t // 32]), t % 32, h, i] = c
        Vd[0][t, h, i] = v
    out = torch.full((2, ctx, 2, d), 7.0, dtype=dtype, device="cuda")
    hga.cache_read(cfg, cache, out[0], out[1], _rows([0, ctx]), _rows([0]))
    got = out[1].double().cpu()
    assert bool(((got == Vd[0]) | (torch.isnan(got) & torch.isnan(Vd[0]))).all())
    Q = torch.randn(rows, 4, d, generator=gen).to(dtype).cuda()
    _attend_not_finite(cfg, cache, Q, begin, Kd[0], Vd[0], 1 if expected == "one" else rows, "infinite codes")
