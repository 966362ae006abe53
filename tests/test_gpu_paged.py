"""GPU checks of the paged key/value cache: rows written (and quantised), read
back, gathered for the routed path and attended, against float64 on the CPU
(tests/paged_oracle.py, where the tolerances are derived)."""

import math
import sys

import pytest
import torch

from paper_2607_15105_amd import hga
from tests import paged_oracle as po

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


def say(*a):
    print(*a, flush=True)
    sys.stdout.flush()


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    hga.lib()


def _cache(cfg, n_seqs, cap, n_pages, page, e4m3, layout, fill=None):
    """A cache whose pools hold `fill` bytes; layout: head, token, or odd (K and
    V with strides of their own, gaps between rows)."""
    H, d = cfg.n_kv_heads, cfg.head_dim
    dt = torch.float8_e4m3fn if e4m3 else hga._torch_dtype(cfg)

    def pool(order, pad):
        if order == "head":
            t = torch.zeros(n_pages, H, page, d + pad, dtype=torch.uint8 if e4m3 else dt, device="cuda")
        else:
            t = torch.zeros(n_pages, page, H, d + pad, dtype=torch.uint8 if e4m3 else dt, device="cuda")
        if fill is not None:
            t.view(torch.uint8).fill_(fill)
        t = t.view(dt)[..., :d]
        return t.transpose(1, 2) if order == "head" else t

    k = pool("token" if layout == "token" else "head", 16 if layout == "odd" else 0)
    v = pool("head" if layout == "head" else "token", 32 if layout == "odd" else 0)
    table = torch.full((n_seqs, cap), -1, dtype=torch.int32, device="cuda")
    sc = [torch.full((n_pages, H, page), 200 if fill else 0, dtype=torch.uint8, device="cuda") if e4m3 else None
          for _ in range(2)]
    return hga.paged_cache(cfg, k, v, table, *sc)


def _fill_table(cache, lengths, gen, spare=0):
    """Pages for the given lengths, in mixed order."""
    page = cache.desc.page_size
    need = [-(-n // page) for n in lengths]
    order = torch.randperm(cache.desc.n_pages, generator=gen).to(torch.int32)
    at = spare
    for s, m in enumerate(need):
        cache.page_table[s, :m] = order[at:at + m].cuda()
        at += m
    assert at <= cache.desc.n_pages


def _rows(lists):
    return torch.tensor(lists, dtype=torch.int32, device="cuda")


def _cfg(hq, hkv, d, dtype, **kw):
    return hga.make_config(hq, hkv, d, dtype=dtype, **kw)


def _held_rows(cfg, x, e4m3):
    """What rows x are after a cache in 64 bits."""
    if not e4m3:
        return x.double().cpu()
    v, e = po.held(x.cpu())
    return v * torch.exp2(e)[..., None]


# ---------------------------------------------------------------- writing and reading

def _hard_rows(n, H, d, dtype, gen):
    """Rows over the type's whole range: magnitudes from tiny to large, zeros,
    rows whose maximum is exactly 448 * 2^e or one step beyond, ties of the codes,
    NaN and infinities."""
    x = torch.randn(n, H, d, generator=gen)
    lo, hi = (-120, 118)
    x *= torch.exp2(torch.randint(lo, hi, (n, H, 1), generator=gen).float())
    flat = x.view(-1, d)[2 * H:]
    flat[0] = 0.0
    flat[1] = torch.linspace(-448, 448, d)
    flat[1, 0] = 448.0
    flat[2, 0] = 448.0 * 2 ** 5
    flat[2, 1:] = (torch.arange(d - 1).float() % 16 + 16.5) * 2 ** 4  # between two codes
    flat[3] = 1.0
    flat[3, 0] = 450.0 if dtype == BF else 448.0 * (1 + 2.0 ** -23)
    flat[4] = torch.randn(d, generator=gen)
    flat[4, 3], flat[4, 7], flat[4, 8] = math.nan, math.inf, -math.inf
    flat[5] = math.inf
    flat[6] = 2.0 ** -130
    flat[7] = torch.randn(d, generator=gen) * 2.0 ** -20  # far below the row's maximum: steps of 2^(e - 9)
    flat[7, 5] = 1.0
    return x.to(dtype)


@pytest.mark.parametrize("hkv,d,dtype", [(8, 128, BF), (3, 64, BF), (2, 64, F32), (1, 128, BF)])
@pytest.mark.parametrize("layout", ["head", "token", "odd"])
def test_quantised_rows_are_held_as_defined(hkv, d, dtype, layout):
    say(f"[write] {hkv} heads, d {d}, {dtype}, {layout}")
    gen = torch.Generator().manual_seed(5)
    cfg = _cfg(hkv, hkv, d, dtype)
    lengths = [70, 1, 0, 33]
    cache = _cache(cfg, 4, 6, 13, 16, True, layout)
    _fill_table(cache, [n + 16 for n in lengths], gen)
    first = [2, 72, 73, 73, 106]  # two rows before and one after belong to nobody
    x = [_hard_rows(107, hkv, d, dtype, gen) for _ in range(2)]
    K, V = (t.cuda() for t in x)
    begin = [5, 0, 3, 12]
    before = [t.view(torch.uint8).clone() for t in (cache.k, cache.v)]
    hga.cache_write(cfg, cache, K, V, _rows(first), _rows(begin))
    torch.cuda.synchronize()
    written = torch.zeros(13, 16, dtype=torch.bool)
    table = cache.page_table.cpu()
    for pool, scale, rows, old in ((cache.k, cache.k_scale, x[0], before[0]), (cache.v, cache.v_scale, x[1], before[1])):
        val, e = po.held(rows)
        got, sc = pool.float().cpu().double(), scale.cpu()
        for r, s, t in po.positions(first, begin, 107):
            p, o = int(table[s, t // 16]), t % 16
            written[p, o] = True
            same = (got[p, o] == val[r]) | (torch.isnan(got[p, o]) & torch.isnan(val[r]))
            assert bool(same.all()), (r, got[p, o][~same][:4], val[r][~same][:4])
            assert torch.equal(sc[p, :, o].double() - 127, e[r]), r
        rest = (pool.view(torch.uint8).cpu() != old.cpu()).flatten(2).any(-1)
        assert not bool((rest & ~written).any())  # nothing else was touched


@pytest.mark.parametrize("hkv,d,dtype", [(8, 128, BF), (3, 64, BF), (2, 64, F32)])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("page,layout", [(16, "token"), (64, "head"), (128, "odd")])
def test_rows_come_back(hkv, d, dtype, e4m3, page, layout):
    say(f"[read] {hkv} heads, d {d}, {dtype}, e4m3 {e4m3}, pages of {page}, {layout}")
    gen = torch.Generator().manual_seed(6)
    cfg = _cfg(hkv, hkv, d, dtype)
    lengths = [200, 1, 64, 0, 129]
    cache = _cache(cfg, 5, 16, 30, page, e4m3, layout)
    _fill_table(cache, lengths, gen)
    first = [0]
    for n in lengths:
        first.append(first[-1] + n)
    big = torch.randn(first[-1], hkv + 1, d + 8, generator=gen).to(dtype).cuda()
    K, V = big[:, :hkv, :d], big[:, 1:, :d]  # strides of their own, shared memory
    zero = _rows([0] * 5)
    hga.cache_write(cfg, cache, K, V, _rows(first), zero)
    cache.page_table[2, 0] = -1  # a page that is gone
    out = torch.full((2, first[-1] + 3, hkv, d + 8), 7.0, dtype=dtype, device="cuda")
    Ko, Vo = out[0, :, :, :d], out[1, :, :, :d]
    hga.cache_read(cfg, cache, Ko, Vo, _rows(first), zero)
    torch.cuda.synchronize()
    for src, got in ((K, Ko), (V, Vo)):
        want = _held_rows(cfg, src, e4m3)
        want[first[2]:first[2] + min(page, 64)] = 0.0
        assert torch.equal(got[:first[-1]].double().cpu(), want)
    assert bool((out[:, first[-1]:] == 7).all()) and bool((out[..., d:] == 7).all())


def test_positions_outside_the_table_are_dropped_and_read_as_zeros():
    cfg = _cfg(2, 2, 64, BF)
    cache = _cache(cfg, 3, 2, 6, 16, True, "head")
    cache.page_table.copy_(torch.tensor([[0, 1], [2, 99], [-5, 3]]))
    K = torch.ones(60, 2, 64, dtype=BF, device="cuda")
    first, begin = _rows([0, 20, 40, 60]), _rows([-4, 20, 6])
    hga.cache_write(cfg, cache, K, 2 * K, first, begin)
    out = torch.full((2, 60, 2, 64), 7.0, dtype=BF, device="cuda")
    hga.cache_read(cfg, cache, out[0], out[1], first, begin)
    torch.cuda.synchronize()
    there = torch.zeros(60, dtype=torch.bool)
    for r, s, t in po.positions([0, 20, 40, 60], [-4, 20, 6], 60):
        there[r] = 0 <= t < 32 and int(cache.page_table[s, t // 16]) in range(6)
    assert 0 < int(there.sum()) < 60
    for got, v in ((out[0], 1.0), (out[1], 2.0)):
        assert torch.equal(got.cpu().float(), there[:, None, None].float().expand(-1, 2, 64) * v)
    assert not bool(cache.k[4:].float().any())  # pages of nobody


def test_rows_of_many_sequences_find_their_place():
    """More sequences than one look at seq_rows covers, most of them empty."""
    gen = torch.Generator().manual_seed(8)
    cfg = _cfg(1, 1, 64, BF)
    n = 301
    lengths = [int(x) for x in torch.randint(0, 3, (n,), generator=gen)]
    cache = _cache(cfg, n, 1, 2 * n, 16, False, "head")
    _fill_table(cache, [16] * n, gen)
    first = [0]
    for m in lengths:
        first.append(first[-1] + m)
    K = torch.randn(first[-1], 1, 64, generator=gen).to(BF).cuda()
    begin = [int(x) for x in torch.randint(0, 14, (n,), generator=gen)]
    hga.cache_write(cfg, cache, K, -K, _rows(first), _rows(begin))
    torch.cuda.synchronize()
    table = cache.page_table.cpu()
    kp, vp, kc = cache.k.cpu(), cache.v.cpu(), K.cpu()
    for r, s, t in po.positions(first, begin, first[-1]):
        assert torch.equal(kp[int(table[s, 0]), t], kc[r]) and torch.equal(vp[int(table[s, 0]), t], -kc[r])


# ---------------------------------------------------------------- attention

def _attend_check(cfg, cache, Q, first, begin, Kd, Vd, max_rows=None, O=None, what="", only=None):
    """attend_paged_fwd against float64; Kd, Vd: per sequence the held rows of
    positions 0 .. [L, Hkv, d] in float64; `only`: the sequences that are compared
    (all). Returns (O, lse)."""
    n = Q.shape[0]
    O = torch.full_like(Q, 7.0) if O is None else O
    lse = torch.full((n, cfg.n_q_heads), 7.0, device="cuda")
    ws = torch.full((hga.paged_workspace_size(cfg, n, max_rows if max_rows else n),), 255, dtype=torch.uint8,
                    device="cuda")
    hga.attend_paged_fwd(cfg, cache, Q, _rows(first), _rows(begin), O, lse, ws, max_rows)
    torch.cuda.synchronize()
    page, table = cache.desc.page_size, cache.page_table.cpu()
    rounding = 2.0 ** -8 if cfg.dtype == hga.HGA_BF16 else 2.0 ** -24
    scale = cfg.softmax_scale if cfg.softmax_scale > 0 else 1 / math.sqrt(cfg.head_dim)
    mine = torch.zeros(n, dtype=torch.bool)
    worst = 0.0
    for s in range(len(begin)):
        a, b = first[s], min(first[s + 1], n)
        if b <= a:
            continue
        mine[a:b] = True
        if only is not None and s not in only:
            continue
        L = Kd[s].shape[0]
        t = torch.arange(L)
        at = t // page
        ok = (at < table.shape[1])
        entry = table[s][at.clamp(max=table.shape[1] - 1)]
        ok &= (entry >= 0) & (entry < cache.desc.n_pages)
        pos = begin[s] + torch.arange(b - a)
        o, z, bo, bl = po.attend(Q[a:b].cpu(), torch.where(ok[:, None, None], Kd[s], 0.0),
                                 torch.where(ok[:, None, None], Vd[s], 0.0), ok, pos, scale, rounding)
        go, gz = O[a:b].double().cpu(), lse[a:b].double().cpu()
        none = torch.isinf(z)
        assert bool((go[none] == 0).all()) and bool((gz[none] == -math.inf).all()), (what, s)
        eo, ez = (go - o).abs(), (gz - z).abs()
        assert bool((eo <= bo + 1e-30)[~none].all()), (what, s, float((eo / bo.clamp(min=1e-30))[~none].max()))
        assert bool((ez <= bl)[~none].all()), (what, s, float((ez / bl)[~none].max()))
        if bool((~none).any()):
            worst = max(worst, float((eo / bo.clamp(min=1e-30))[~none].max()))
    assert bool((O[~mine.cuda()] == 7).all()) and bool((lse[~mine.cuda()] == 7).all()), what  # of no sequence
    say(f"   {what}: largest error {worst:.3f} of its bound")
    return O, lse


def _context(cfg, cache, lengths, gen, e4m3, garbage=True):
    """Random K/V of every position written into the cache; the held rows."""
    H, d = cfg.n_kv_heads, cfg.head_dim
    dt = hga._torch_dtype(cfg)
    first = [0]
    for n in lengths:
        first.append(first[-1] + n)
    if first[-1] == 0:
        return [torch.zeros(0, H, d, dtype=torch.float64)] * len(lengths), [torch.zeros(0, H, d, dtype=torch.float64)] * len(lengths)
    K = (torch.randn(first[-1], H, d, generator=gen) + 0.5 * torch.randn(1, H, d, generator=gen)).to(dt)
    V = torch.randn(first[-1], H, d, generator=gen).to(dt)
    hga.cache_write(cfg, cache, K.cuda(), V.cuda(), _rows(first), _rows([0] * len(lengths)))
    Kh, Vh = _held_rows(cfg, K, e4m3), _held_rows(cfg, V, e4m3)
    cut = [(first[s], first[s + 1]) for s in range(len(lengths))]
    return [Kh[a:b] for a, b in cut], [Vh[a:b] for a, b in cut]


HEADS = [(8, 2, 128, BF), (8, 1, 64, BF), (3, 3, 128, BF), (4, 2, 64, F32), (16, 8, 128, BF)]


@pytest.mark.parametrize("hq,hkv,d,dtype", HEADS)
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("form", ["decode", "few", "chunks", "mixed"])
def test_rows_attend_their_cached_context(hq, hkv, d, dtype, e4m3, form):
    say(f"[attend] {hq}/{hkv} heads, d {d}, {dtype}, e4m3 {e4m3}, {form}")
    gen = torch.Generator().manual_seed(11)
    cfg = _cfg(hq, hkv, d, dtype)
    ctx, rows = {"decode": ([1, 2, 63, 64, 65, 0, 700, 1025, 16], [1, 1, 1, 1, 1, 0, 1, 1, 1]),
                 "few": ([3, 64, 66, 500, 2, 0], [3, 2, 4, 3, 1, 0]),
                 "chunks": ([300, 64, 777, 129, 0, 1000], [300, 1, 77, 65, 0, 130]),
                 "mixed": ([600, 1, 333, 90, 2000], [290, 1, 1, 2, 1])}[form]
    for page, layout in ((16, "token"), (64, "head"), (256, "odd")):
        cap = max(-(-c // page) for c in ctx) + 1
        cache = _cache(cfg, len(ctx), cap, sum(-(-c // page) for c in ctx) + 2, page, e4m3, layout, fill=0xFF)
        _fill_table(cache, ctx, gen)
        Kd, Vd = _context(cfg, cache, ctx, gen, e4m3)
        first = [1]
        for r in rows:
            first.append(first[-1] + r)
        begin = [c - r for c, r in zip(ctx, rows)]
        n = first[-1] + 2
        Q = torch.randn(n, hq, d, generator=gen).to(dtype).cuda()
        _attend_check(cfg, cache, Q, first, begin, Kd, Vd, max(rows), what=f"pages of {page}, {layout}")


@pytest.mark.parametrize("dtype,d", [(BF, 128), (F32, 64)])
@pytest.mark.parametrize("rows", [1, 100])
def test_long_context_is_split_and_joined(dtype, d, rows):
    say(f"[attend] split {dtype} rows {rows}")
    gen = torch.Generator().manual_seed(12)
    cfg = _cfg(4, 1, d, dtype)
    for ctx in (257, 20011):
        cache = _cache(cfg, 2, -(-ctx // 64), -(-ctx // 64) + 1, 64, False, "head", fill=0xFF)
        _fill_table(cache, [ctx, 1], gen)
        Kd, Vd = _context(cfg, cache, [ctx, 1], gen, False)
        Q = torch.randn(rows + 1, 4, d, generator=gen).to(dtype).cuda()
        first, begin = [0, rows, rows + 1], [ctx - rows, 0]
        O, lse = _attend_check(cfg, cache, Q, first, begin, Kd, Vd, rows, what=f"context {ctx}")
        again, z2 = _attend_check(cfg, cache, Q, first, begin, Kd, Vd, rows, what="again")
        assert torch.equal(O, again) and torch.equal(lse, z2)  # the same bits
        _attend_check(cfg, cache, Q, first, begin, Kd, Vd, 1, what="one row expected")
        _attend_check(cfg, cache, Q, first, begin, Kd, Vd, None, what="nothing expected")


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("dtype,d", [(BF, 128), (F32, 64)])
def test_absent_pages_are_left_out_and_rows_without_keys_are_empty(dtype, d, e4m3):
    say(f"[attend] absent pages {dtype} {e4m3}")
    gen = torch.Generator().manual_seed(13)
    cfg = _cfg(4, 2, d, dtype)
    ctx, rows = [500, 130, 40, 300, 200], [3, 130, 2, 1, 150]
    cache = _cache(cfg, 5, 40, 90, 16, e4m3, "head", fill=0xFF)
    _fill_table(cache, ctx, gen)
    Kd, Vd = _context(cfg, cache, ctx, gen, e4m3)
    cache.page_table[0, 1:20] = -1                # the middle of a context
    cache.page_table[1, 0:3] = 90                 # its beginning: the first 48 rows see nothing
    cache.page_table[2] = -7                      # all of it
    cache.page_table[3, ::2] = 1 << 30
    cache.page_table[4, 4:8] = -1                 # a whole 64-key tile
    first = [0]
    for r in rows:
        first.append(first[-1] + r)
    Q = torch.randn(first[-1], 4, d, generator=gen).to(dtype).cuda()
    begin = [c - r for c, r in zip(ctx, rows)]
    for max_rows in (1, 150):
        _attend_check(cfg, cache, Q, first, begin, Kd, Vd, max_rows, what=f"max_rows {max_rows}")


@pytest.mark.parametrize("max_rows", [1, 200])
def test_positions_before_zero_or_past_the_table(max_rows):
    gen = torch.Generator().manual_seed(14)
    cfg = _cfg(8, 2, 64, BF)
    cache = _cache(cfg, 3, 4, 12, 16, False, "head", fill=0xFF)
    _fill_table(cache, [64, 64, 64], gen)
    Kd, Vd = _context(cfg, cache, [64, 64, 64], gen, False)
    begin, first = [-30, 50, -500], [0, 60, 130, 140]
    grow = lambda x: torch.cat([x, torch.zeros(200, 2, 64, dtype=torch.float64)])
    Q = torch.randn(140, 8, 64, generator=gen).to(BF).cuda()
    _attend_check(cfg, cache, Q, first, begin, [grow(k) for k in Kd], [grow(v) for v in Vd], max_rows, what="outside")


@pytest.mark.parametrize("max_rows", [1, 90])
@pytest.mark.parametrize("dtype,d,e4m3", [(BF, 128, False), (BF, 64, True), (F32, 64, False)])
def test_later_rows_never_enter(dtype, d, e4m3, max_rows):
    """NaN and infinities in the keys and values of later rows of the chunk."""
    say(f"[attend] poisoned later rows {dtype} {e4m3}")
    gen = torch.Generator().manual_seed(15)
    cfg = _cfg(4, 2, d, dtype)
    ctx, rows, cut = 201, 90, 40  # rows from `cut` on are poisoned
    cache = _cache(cfg, 1, 13, 14, 16, e4m3, "head", fill=0xFF)
    _fill_table(cache, [ctx], gen)
    Kd, Vd = _context(cfg, cache, [ctx], gen, e4m3)
    bad = torch.randn(rows - cut, 2, d, generator=gen)
    bad[3, 0, 5], bad[4, 1, 7], bad[7] = math.nan, math.inf, -math.inf
    bad[0, 0, d - 1] = math.nan
    x = bad.to(dtype).cuda()
    Q = torch.randn(rows, 4, d, generator=gen).to(dtype).cuda()
    begin = ctx - rows
    for kv in ("k", "v"):
        K, V = (x, torch.ones_like(x)) if kv == "k" else (torch.ones_like(x), x)
        hga.cache_write(cfg, cache, K, V, _rows([0, rows - cut]), _rows([begin + cut]))
        O = torch.zeros_like(Q)
        lse = torch.zeros(rows, 4, device="cuda")
        ws = torch.empty(hga.paged_workspace_size(cfg, rows, max_rows), dtype=torch.uint8, device="cuda")
        hga.attend_paged_fwd(cfg, cache, Q, _rows([0, rows]), _rows([begin]), O, lse, ws, max_rows)
        torch.cuda.synchronize()
        pos = begin + torch.arange(cut)
        rounding = 2.0 ** -8 if dtype == BF else 2.0 ** -24
        n = begin + cut
        o, z, bo, bl = po.attend(Q[:cut].cpu(), Kd[0][:n], Vd[0][:n], torch.ones(n, dtype=torch.bool), pos,
                                 1 / math.sqrt(d), rounding)
        assert bool(((O[:cut].double().cpu() - o).abs() <= bo).all()) and bool(((lse[:cut].double().cpu() - z).abs() <= bl).all())
        # rows at or after a NaN value see it, in its dimension and head only
        if kv == "v":
            assert bool(torch.isnan(O[cut:, :2, d - 1]).all())
            if not e4m3:
                assert bool(torch.isfinite(O[cut:cut + 3, :, :5].float()).all())
                assert bool((O[cut + 4:cut + 7, 2:, 7] == math.inf).all())


def test_queries_and_outputs_with_strides_and_a_given_scale():
    gen = torch.Generator().manual_seed(16)
    cfg = _cfg(8, 4, 64, BF, softmax_scale=0.4)
    ctx, rows = [150, 90, 2], [40, 1, 1]
    cache = _cache(cfg, 3, 10, 20, 16, False, "odd", fill=0xFF)
    _fill_table(cache, ctx, gen)
    Kd, Vd = _context(cfg, cache, ctx, gen, False)
    first = [0, 40, 41, 42]
    Q = torch.randn(42, 12, 72, generator=gen).to(BF).cuda()[:, 2:10, :64]
    big = torch.full((8, 42, 80), 7.0, dtype=BF, device="cuda")
    O = big.transpose(0, 1)[:, :, :64]
    for max_rows in (1, 40):
        _attend_check(cfg, cache, Q, first, [110, 89, 1], Kd, Vd, max_rows, O=O, what="strided")
    assert bool((big[..., 64:] == 7).all())


@pytest.mark.parametrize("e4m3", [False, True])
def test_pool_offsets_beyond_32_bits(e4m3):
    """Pages whose byte offsets pass 2^32 (and a scale table past 2^31 of the codes)."""
    gen = torch.Generator().manual_seed(17)
    cfg = _cfg(8, 8, 128, BF)
    page, n_pages = 256, (5 << 30) // (256 * 8 * 128 * (1 if e4m3 else 2))
    cache = _cache(cfg, 2, 3, n_pages, page, e4m3, "head")
    cache.page_table.copy_(torch.tensor([[n_pages - 1, 0, n_pages - 2], [n_pages - 3, 1, -1]]))
    ctx = [600, 400]
    Kd, Vd = _context(cfg, cache, ctx, gen, e4m3)
    out = torch.empty(2, 1000, 8, 128, dtype=BF, device="cuda")
    hga.cache_read(cfg, cache, out[0], out[1], _rows([0, 600, 1000]), _rows([0, 0]))
    assert torch.equal(out[0].double().cpu(), torch.cat(Kd)) and torch.equal(out[1].double().cpu(), torch.cat(Vd))
    for rows in ([1, 1], [70, 40]):
        first = [0, rows[0], sum(rows)]
        Q = torch.randn(sum(rows), 8, 128, generator=gen).to(BF).cuda()
        _attend_check(cfg, cache, Q, first, [c - r for c, r in zip(ctx, rows)], Kd, Vd, max(rows), what="far pages")


def test_two_sequences_share_a_prefix():
    gen = torch.Generator().manual_seed(18)
    cfg = _cfg(4, 1, 128, BF)
    cache = _cache(cfg, 2, 6, 12, 16, True, "head", fill=0xFF)
    _fill_table(cache, [90, 0], gen)
    Kd, Vd = _context(cfg, cache, [90, 0], gen, True)
    cache.page_table[1, :3] = cache.page_table[0, :3]
    Q = torch.randn(21, 4, 128, generator=gen).to(BF).cuda()
    _attend_check(cfg, cache, Q, [0, 1, 21], [89, 28], [Kd[0], Kd[0][:48]], [Vd[0], Vd[0][:48]], 20, what="shared")


@pytest.mark.parametrize("rows,e4m3", [(1, False), (1, True), (3, False), (3, True)])
def test_long_shares(rows, e4m3):
    """64 sequences over the same 20,000 cached positions: enough work that a
    workgroup follows one context over hundreds of tiles."""
    say(f"[attend] long shares, {rows} rows, e4m3 {e4m3}")
    gen = torch.Generator().manual_seed(22)
    cfg = _cfg(64, 8, 64, BF)
    ctx, S = 20000, 64
    cache = _cache(cfg, S, 160, 161, 128, e4m3, "head", fill=0xFF)
    _fill_table(cache, [ctx] + [0] * (S - 1), gen)
    Kd, Vd = _context(cfg, cache, [ctx] + [0] * (S - 1), gen, e4m3)
    cache.page_table[1:] = cache.page_table[0]
    cache.page_table[40, 70] = -1
    Q = torch.randn(rows * S, 64, 64, generator=gen).to(BF).cuda()
    begin = [ctx - rows - 37 * s for s in range(S)]
    _attend_check(cfg, cache, Q, [rows * s for s in range(S + 1)], begin, [Kd[0]] * S, [Vd[0]] * S, rows, only=(0, 7, 40, 63))


@pytest.mark.parametrize("max_rows", [1, 3, 9, None])
def test_more_sequences_than_threads(max_rows):
    gen = torch.Generator().manual_seed(23)
    cfg = _cfg(4, 2, 64, BF)
    S = 1100
    rows = [int(x) for x in torch.randint(0, 3, (S,), generator=gen)]
    rows[700], rows[1099] = 9, 9
    ctx = [r + int(x) if r else 0 for r, x in zip(rows, torch.randint(0, 40, (S,), generator=gen))]
    cache = _cache(cfg, S, 4, sum(-(-c // 16) for c in ctx) + 1, 16, False, "token", fill=0xFF)
    _fill_table(cache, ctx, gen)
    Kd, Vd = _context(cfg, cache, ctx, gen, False)
    first = [0]
    for r in rows:
        first.append(first[-1] + r)
    Q = torch.randn(first[-1], 4, 64, generator=gen).to(BF).cuda()
    _attend_check(cfg, cache, Q, first, [c - r for c, r in zip(ctx, rows)], Kd, Vd, max_rows, what=f"{S} sequences")


def test_a_tiny_scale_and_equal_keys():
    """Every p alike: O is the mean of the values, lse the logarithm of their number."""
    gen = torch.Generator().manual_seed(24)
    cfg = _cfg(4, 2, 128, BF, softmax_scale=1e-38)
    cache = _cache(cfg, 1, 10, 10, 16, False, "head", fill=0xFF)
    _fill_table(cache, [150], gen)
    Kd, Vd = _context(cfg, cache, [150], gen, False)
    Q = torch.randn(40, 4, 128, generator=gen).to(BF).cuda()
    for max_rows in (1, 40):
        _attend_check(cfg, cache, Q, [0, 40], [110], Kd, Vd, max_rows)


# ---------------------------------------------------------------- streams, graphs

def test_recorded_calls_and_graphs_that_share_a_workspace():
    """Calls marshalled once, and two captured graphs with one workspace replayed
    one after the other: the direct calls' bits."""
    gen = torch.Generator().manual_seed(25)
    cfg = _cfg(8, 2, 128, BF)
    cache = _cache(cfg, 2, 30, 60, 64, True, "head")
    _fill_table(cache, [1900, 900], gen)
    K, V = (torch.randn(2800, 2, 128, generator=gen).to(BF).cuda() for _ in range(2))
    calls = []
    ws = torch.empty(hga.paged_workspace_size(cfg, 300, 200), dtype=torch.uint8, device="cuda")
    for rows in ([1, 1], [200, 100]):
        Q = torch.randn(sum(rows), 8, 128, generator=gen).to(BF).cuda()
        first, begin = _rows([0, rows[0], sum(rows)]), _rows([1900 - rows[0], 900 - rows[1]])
        calls.append((Q, first, begin, torch.zeros_like(Q), torch.zeros(sum(rows), 8, device="cuda"), max(rows)))

    def attend(i):
        Q, first, begin, O, lse, most = calls[i]
        hga.attend_paged_fwd(cfg, cache, Q, first, begin, O, lse, ws, most)

    first, begin = _rows([0, 1900, 2800]), _rows([0, 0])  # kept: the recorded call has their addresses
    with hga.record() as kept:
        hga.cache_write(cfg, cache, K, V, first, begin)
        attend(0)
        attend(1)
    assert not bool(cache.k.float().any())  # recorded, not made
    for call in kept:
        call()
    torch.cuda.synchronize()
    want = [(c[3].clone(), c[4].clone()) for c in calls]
    assert all(bool(w[0].float().abs().sum() > 0) for w in want)
    side, graphs = torch.cuda.Stream(), [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    for i in range(2):
        with torch.cuda.graph(graphs[i], stream=side):
            attend(i)
    for turn in range(4):
        for c in calls:
            c[3].zero_()
            c[4].zero_()
        ws.fill_(255)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graphs[turn % 2].replay()
            graphs[1 - turn % 2].replay()
        side.synchronize()
        for c, (o, z) in zip(calls, want):
            assert torch.equal(c[3], o) and torch.equal(c[4], z)


def test_captured_steps_follow_the_lengths_on_the_device():
    """One decode step (write, attend) captured once and replayed as the
    contexts grow, on a side stream, with eager work between; two graphs with
    workspaces of their own."""
    gen = torch.Generator().manual_seed(19)
    cfg = _cfg(8, 2, 128, BF)
    S, steps = 5, 6
    start = [0, 63, 500, 14, 100]
    cache = _cache(cfg, S, 10, 52, 64, True, "head", fill=0xFF)
    _fill_table(cache, [640] * S, gen)
    Kd, Vd = _context(cfg, cache, start, gen, True)
    first = _rows(list(range(S + 1)))
    begin = _rows(start)
    K, V = torch.zeros(S, 2, 128, dtype=BF, device="cuda"), torch.zeros(S, 2, 128, dtype=BF, device="cuda")
    Q = torch.zeros(S, 8, 128, dtype=BF, device="cuda")
    O, lse = torch.zeros_like(Q), torch.zeros(S, 8, device="cuda")
    many = torch.randn(40, 8, 128, generator=gen).to(BF).cuda()  # a second graph: 40 rows of sequence 2
    O2, lse2 = torch.zeros_like(many), torch.zeros(40, 8, device="cuda")
    first2, begin2 = _rows([0, 0, 0, 40, 40, 40]), _rows([0, 0, 460, 0, 0])
    ws = torch.empty(hga.paged_workspace_size(cfg, S, 1), dtype=torch.uint8, device="cuda")
    ws2 = torch.empty(hga.paged_workspace_size(cfg, 40), dtype=torch.uint8, device="cuda")

    def step():
        hga.cache_write(cfg, cache, K, V, first, begin)
        hga.attend_paged_fwd(cfg, cache, Q, first, begin, O, lse, ws, 1)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    step()  # every kernel is loaded before the capture
    hga.attend_paged_fwd(cfg, cache, many, first2, begin2, O2, lse2, ws2)
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=side):
        step()
    with torch.cuda.graph(g2, stream=side):
        hga.attend_paged_fwd(cfg, cache, many, first2, begin2, O2, lse2, ws2)
    for i in range(steps):
        x = [torch.randn(S, h, 128, generator=gen).to(BF) for h in (2, 2, 8)]
        for dst, src in zip((K, V, Q), x):
            dst.copy_(src)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            g.replay()
            g2.replay()
        side.synchronize()
        gO, gl, gO2 = O.clone(), lse.clone(), O2.clone()
        Kh, Vh = _held_rows(cfg, x[0], True), _held_rows(cfg, x[1], True)
        Kd = [torch.cat([Kd[s], Kh[s:s + 1]]) for s in range(S)]
        Vd = [torch.cat([Vd[s], Vh[s:s + 1]]) for s in range(S)]
        eO, el = _attend_check(cfg, cache, Q, list(range(S + 1)), [n + i for n in start], Kd, Vd, 1, what=f"step {i}")
        assert torch.equal(gO, eO) and torch.equal(gl, el)
        hga.attend_paged_fwd(cfg, cache, many, first2, begin2, O2, lse2, ws2)
        torch.cuda.synchronize()
        assert torch.equal(gO2, O2)
        begin += 1


# ---------------------------------------------------------------- used together

@pytest.mark.parametrize("e4m3", [False, True])
def test_a_prompt_in_chunks_then_generation(e4m3):
    """Two sequences: their prompts written and attended in chunks, then tokens
    one by one, each compared with the whole context in float64."""
    gen = torch.Generator().manual_seed(20)
    cfg = _cfg(8, 2, 128, BF)
    cache = hga.alloc_paged_cache(cfg, 2, 8, 16, 64, e4m3)
    cache.page_table.copy_(torch.randperm(16, generator=gen).view(2, 8).to(torch.int32))
    done = [0, 0]
    Kd = [torch.zeros(0, 2, 128, dtype=torch.float64)] * 2
    Vd = list(Kd)
    for rows in ([130, 1], [70, 200], [1, 33], [1, 1], [1, 1], [0, 1]):
        first = [0, rows[0], sum(rows)]
        K, V = (torch.randn(first[2], 2, 128, generator=gen).to(BF) for _ in range(2))
        Q = torch.randn(first[2], 8, 128, generator=gen).to(BF).cuda()
        hga.cache_write(cfg, cache, K.cuda(), V.cuda(), _rows(first), _rows(done))
        Kh, Vh = _held_rows(cfg, K, e4m3), _held_rows(cfg, V, e4m3)
        for s in range(2):
            Kd[s] = torch.cat([Kd[s], Kh[first[s]:first[s + 1]]])
            Vd[s] = torch.cat([Vd[s], Vh[first[s]:first[s + 1]]])
        _attend_check(cfg, cache, Q, first, done, Kd, Vd, max(rows), what=f"rows {rows}")
        done = [a + b for a, b in zip(done, rows)]


@pytest.mark.parametrize("hq,hkv,d,dtype,e4m3,page", [(8, 2, 128, BF, True, 64), (8, 2, 128, BF, False, 16),
                                                      (8, 4, 64, BF, True, 256), (2, 1, 64, F32, True, 32)])
def test_routed_path_over_the_cache_equals_the_dense_rows(hq, hkv, d, dtype, e4m3, page):
    """Summaries and routing of a sequence's rows as read back, its routed rows
    gathered from the pages, and attention and its gradient over them: bit for bit
    those of the dense rows."""
    gen = torch.Generator().manual_seed(21)
    cfg = _cfg(hq, hkv, d, dtype, group_size=8, top_chunks=4, top_groups=9, sink_tokens=64, local_tokens=128)
    T, n_q = 1536, 512
    cache = _cache(cfg, 3, T // page + 1, 2 * (T // page), page, e4m3, "head", fill=0xFF)
    _fill_table(cache, [40, T, 0], gen)
    K, V = (torch.randn(T, hkv, d, generator=gen).to(dtype).cuda() for _ in range(2))
    first, begin = _rows([0, 0, T, T]), _rows([0, 0, 0])
    hga.cache_write(cfg, cache, K, V, first, begin)
    hga.cache_read(cfg, cache, K, V, first, begin)  # K, V: as held
    q0 = T - n_q
    Q, dO = (torch.randn(n_q, hq, d, generator=gen).to(dtype).cuda() for _ in range(2))
    cs, gs = hga.alloc_summaries(cfg, T)
    hga.build_summaries(cfg, K, 0, T, cs, gs)
    rb = hga.alloc_route(cfg, q0, n_q)
    hga.route(cfg, Q, q0, cs, gs, rb.sel_chunks, rb.sel_groups, rb.n_sel_groups, rb.workspace)
    cap = hga.gathered_rows(cfg)
    a, b = (torch.full((2, n_q // 64, hkv, cap, d), 7.0, dtype=dtype, device="cuda") for _ in range(2))
    hga.gather_routed(cfg, K, V, q0, n_q, rb.sel_groups, rb.n_sel_groups, a[0], a[1])
    hga.gather_paged(cfg, cache, 1, q0, n_q, rb.sel_groups, rb.n_sel_groups, b[0], b[1])
    assert torch.equal(a, b)
    O, O2 = torch.zeros_like(Q), torch.zeros_like(Q)
    lse, lse2 = torch.zeros(n_q, hq, device="cuda"), torch.zeros(n_q, hq, device="cuda")
    hga.attend_fwd(cfg, Q, K, V, q0, rb.sel_groups, rb.n_sel_groups, O, lse)
    hga.attend_gathered_fwd(cfg, Q, b[0], b[1], q0, rb.n_sel_groups, O2, lse2)
    assert torch.equal(O, O2) and torch.equal(lse, lse2)
    grads = [[torch.zeros(n_q, h, d, device="cuda") for h in (hq, hkv, hkv)] for _ in range(2)]
    ws = torch.empty(hga.workspace_size(cfg, hga.OP_BWD, q0, n_q, q0), dtype=torch.uint8, device="cuda")
    hga.attend_bwd(cfg, Q, K, V, O, dO, lse, q0, q0, rb.sel_groups, rb.n_sel_groups, *grads[0], ws)
    hga.attend_gathered_bwd(cfg, Q, b[0], b[1], K[q0:], V[q0:], q0, O2, dO, lse2, q0, q0, rb.sel_groups,
                            rb.n_sel_groups, *grads[1], ws)
    assert all(torch.equal(x, y) for x, y in zip(*grads))
    # a page that is gone: its rows are zeros, the others stay
    gone = q0 // page
    cache.page_table[1, gone] = -1
    hga.gather_paged(cfg, cache, 1, q0, n_q, rb.sel_groups, rb.n_sel_groups, b[0], b[1])
    K[gone * page:gone * page + page] = 0
    V[gone * page:gone * page + page] = 0
    hga.gather_routed(cfg, K, V, q0, n_q, rb.sel_groups, rb.n_sel_groups, a[0], a[1])
    assert torch.equal(a, b)


# ---------------------------------------------------------------- the ends of the ranges

@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("first", [[0, 0, 0], [40, 40, 40], [17, 17, 17]])
def test_a_batch_without_rows_changes_nothing(first, e4m3):
    cfg = _cfg(4, 2, 64, BF)
    cache = _cache(cfg, 2, 4, 8, 16, e4m3, "head", fill=0x11)
    cache.page_table.copy_(torch.arange(8).view(2, 4))
    before = [t.view(torch.uint8).clone() for t in (cache.k, cache.v)]
    x = torch.ones(40, 2, 64, dtype=BF, device="cuda")
    rows, begin = _rows(first), _rows([3, 9])
    hga.cache_write(cfg, cache, x, x, rows, begin)
    assert all(torch.equal(t.view(torch.uint8), b) for t, b in zip((cache.k, cache.v), before))
    out = torch.full((2, 40, 2, 64), 7.0, dtype=BF, device="cuda")
    hga.cache_read(cfg, cache, out[0], out[1], rows, begin)
    O, lse = torch.full((40, 4, 64), 7.0, dtype=BF, device="cuda"), torch.full((40, 4), 7.0, device="cuda")
    for max_rows in (1, 16, 40):
        ws = torch.full((hga.paged_workspace_size(cfg, 40, max_rows),), 255, dtype=torch.uint8, device="cuda")
        hga.attend_paged_fwd(cfg, cache, O, rows, begin, O, lse, ws, max_rows)
    assert bool((out == 7).all()) and bool((O == 7).all()) and bool((lse == 7).all())


def test_more_rows_than_a_launch_has():
    """2^26 rows and some, of which only the last belong to sequences."""
    cfg = _cfg(1, 1, 64, BF)
    n = (1 << 26) + 7
    say(f"[write, read] {n} rows")
    cache = _cache(cfg, 2, 2, 4, 16, False, "head")
    cache.page_table.copy_(torch.arange(4).view(2, 2))
    a, b = (torch.empty(n, 1, 64, dtype=BF, device="cuda") for _ in range(2))
    gen = torch.Generator().manual_seed(31)
    tail = torch.randn(8, 1, 64, generator=gen).to(BF).cuda()
    a[n - 8:], b[n - 8:], a[:4], b[:4] = tail, -tail, 5.0, 5.0
    first, begin = _rows([n - 5, n - 2, n]), _rows([0, 15])
    hga.cache_write(cfg, cache, a, b, first, begin)
    k, v = cache.k.cpu(), cache.v.cpu()
    at = [(0, 0), (0, 1), (0, 2), (2, 15), (3, 0)]  # page, slot
    want = torch.zeros_like(k)
    for (p, t), row in zip(at, tail[3:].cpu()):
        want[p, t] = row
    assert torch.equal(k, want) and torch.equal(v, -want)
    a[n - 8:], b[n - 8:] = 7.0, 7.0
    hga.cache_read(cfg, cache, a, b, first, begin)
    assert torch.equal(a[n - 5:], tail[3:]) and torch.equal(b[n - 5:], -tail[3:])
    assert bool((a[n - 8:n - 5] == 7).all()) and bool((a[:4] == 5).all()) and bool((b[:4] == 5).all())


def test_codes_held_as_bytes_are_the_same_cache():
    """A pool of uint8 and one of float8_e4m3fn: the same bytes and results."""
    gen = torch.Generator().manual_seed(32)
    cfg = _cfg(4, 2, 128, BF)
    one = _cache(cfg, 1, 6, 6, 16, True, "token")
    _fill_table(one, [90], gen)
    two = hga.paged_cache(cfg, one.k.view(torch.uint8).clone(), one.v.view(torch.uint8).clone(), one.page_table,
                          one.k_scale.clone(), one.v_scale.clone())
    Q, K = torch.randn(90, 4, 128, generator=gen).to(BF).cuda(), torch.randn(90, 2, 128, generator=gen).to(BF).cuda()
    got = []
    for cache in (one, two):
        hga.cache_write(cfg, cache, K, K, _rows([0, 90]), _rows([0]))
        O, lse = torch.empty_like(Q), torch.empty(90, 4, device="cuda")
        ws = torch.empty(hga.paged_workspace_size(cfg, 90), dtype=torch.uint8, device="cuda")
        hga.attend_paged_fwd(cfg, cache, Q, _rows([0, 90]), _rows([0]), O, lse, ws)
        got.append((cache.k.view(torch.uint8), cache.v.view(torch.uint8), cache.k_scale, cache.v_scale, O, lse))
    assert all(torch.equal(x, y) for x, y in zip(*got))


@pytest.mark.parametrize("rows", [3, 70])
@pytest.mark.parametrize("e4m3", [False, True])
def test_the_largest_pages(rows, e4m3):
    gen = torch.Generator().manual_seed(33)
    cfg = _cfg(2, 1, 64, BF)
    cache = _cache(cfg, 1, 2, 3, 65536, e4m3, "head", fill=0xFF)
    cache.page_table.copy_(torch.tensor([[2, 0]]))
    ctx = 65536 + 201
    Kd, Vd = _context(cfg, cache, [ctx], gen, e4m3)
    Q = torch.randn(rows, 2, 64, generator=gen).to(BF).cuda()
    _attend_check(cfg, cache, Q, [0, rows], [ctx - rows], Kd, Vd, rows, what="large pages")


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("dtype,d", [(BF, 64), (F32, 64)])
@pytest.mark.parametrize("rows", [20, 50, 330])
def test_chunks_of_every_size_with_absent_pages_and_poisoned_rows(rows, dtype, d, e4m3):
    """A chunk, a row beside it and an idle sequence; a fifth of the pages absent,
    NaN in keys and values behind each row."""
    say(f"[attend] chunk of {rows}, {dtype} {e4m3}")
    gen = torch.Generator().manual_seed(34)
    cfg = _cfg(4, 2, d, dtype)
    n = [rows, 1, 0]
    ctx = [rows + 411, 130, 0]
    cache = _cache(cfg, 3, 60, 80, 16, e4m3, "token", fill=0xFF)
    _fill_table(cache, ctx, gen)
    Kd, Vd = _context(cfg, cache, ctx, gen, e4m3)
    cache.page_table[0, 3:9] = -1
    cache.page_table[1, 1] = 1000
    cut = rows - 7  # rows behind `cut` of the chunk are poisoned
    x = torch.ones(7, 2, d)
    x[2], x[5, 0, 3] = math.nan, math.nan
    x = x.to(dtype).cuda()
    hga.cache_write(cfg, cache, x, x, _rows([0, 7, 7, 7]), _rows([ctx[0] - 7, 0, 0]))
    Q = torch.randn(rows + 1, 4, d, generator=gen).to(dtype).cuda()
    first, begin = [0, rows, rows + 1, rows + 1], [ctx[0] - rows, ctx[1] - 1, 0]
    for max_rows in (1, rows):
        O, lse = torch.zeros_like(Q), torch.zeros(rows + 1, 4, device="cuda")
        ws = torch.empty(hga.paged_workspace_size(cfg, rows + 1, max_rows), dtype=torch.uint8, device="cuda")
        hga.attend_paged_fwd(cfg, cache, Q, _rows(first), _rows(begin), O, lse, ws, max_rows)
        torch.cuda.synchronize()
        table = cache.page_table.cpu()
        for s, a, b in ((0, 0, cut), (1, rows, rows + 1)):
            L = ctx[s] - (7 if s == 0 else 0)
            entry = table[s][torch.arange(L) // 16]
            ok = (entry >= 0) & (entry < 80)
            pos = begin[s] + torch.arange(b - a)
            o, z, bo, bl = po.attend(Q[a:b].cpu(), torch.where(ok[:, None, None], Kd[s][:L], 0.0),
                                     torch.where(ok[:, None, None], Vd[s][:L], 0.0), ok, pos, 1 / math.sqrt(d),
                                     2.0 ** -8 if dtype == BF else 2.0 ** -24)
            assert bool(((O[a:b].double().cpu() - o).abs() <= bo).all()), (max_rows, s)
            assert bool(((lse[a:b].double().cpu() - z).abs() <= bl).all()), (max_rows, s)
        assert bool(torch.isnan(O[cut + 2:rows]).all())  # every later row attends the NaN


@pytest.mark.parametrize("hq,hkv,d,dtype", [(11, 11, 128, BF), (34, 17, 64, BF), (13, 13, 64, F32)])
@pytest.mark.parametrize("e4m3", [False, True])
def test_many_odd_heads(hq, hkv, d, dtype, e4m3):
    gen = torch.Generator().manual_seed(35)
    cfg = _cfg(hq, hkv, d, dtype)
    ctx, rows = [140, 37], [33, 1]
    cache = _cache(cfg, 2, 5, 13, 32, e4m3, "token", fill=0xFF)
    _fill_table(cache, ctx, gen)
    Kd, Vd = _context(cfg, cache, ctx, gen, e4m3)
    out = torch.empty(2, 177, hkv, d, dtype=dtype, device="cuda")
    hga.cache_read(cfg, cache, out[0], out[1], _rows([0, 140, 177]), _rows([0, 0]))
    assert torch.equal(out[0].double().cpu(), torch.cat(Kd)) and torch.equal(out[1].double().cpu(), torch.cat(Vd))
    Q = torch.randn(34, hq, d, generator=gen).to(dtype).cuda()
    for max_rows in (1, 33):
        _attend_check(cfg, cache, Q, [0, 33, 34], [107, 36], Kd, Vd, max_rows, what=f"{hkv} kv heads")
