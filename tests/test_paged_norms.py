"""That the checks of tests/paged_norms.py accept what the kernels compute, and
reject results with a small part of a long context wrong: mistakes planted in the
reference, on the CPU."""

import math

import pytest
import torch

from tests import paged_norms as pn

BF, F32 = torch.bfloat16, torch.float32


def _inputs(ctx, rows, hq, hkv, d, dtype, seed=1):
    gen = torch.Generator().manual_seed(seed)
    K = (torch.randn(ctx, hkv, d, generator=gen) + 0.5 * torch.randn(1, hkv, d, generator=gen)).to(dtype)
    V = torch.randn(ctx, hkv, d, generator=gen).to(dtype)
    Q = torch.randn(rows, hq, d, generator=gen).to(dtype)
    return Q, K, V, torch.ones(ctx, dtype=torch.bool), ctx - rows + torch.arange(rows)


def _like_the_kernel(Q, K, V, ok, pos, bits, drop=None):
    """Attention in float32 with P of `bits` significant bits before P.V (24: as it is;
    the sum of P is not rounded), keys `drop` left out."""
    n, Hq, d = Q.shape
    G = Hq // K.shape[1]
    see = (torch.arange(K.shape[0])[None, :] <= pos[:, None]) & ok[None, :]
    if drop is not None:
        see[:, drop] = False
    O, lse = torch.zeros(n, Hq, d), torch.zeros(n, Hq)
    for h in range(Hq):
        s = (Q[:, h].float() @ K[:, h // G].float().T / math.sqrt(d)).masked_fill(~see, -math.inf)
        m = s.amax(-1, keepdim=True)
        p = torch.exp(s - m)
        l = p.sum(-1, keepdim=True)
        lse[:, h] = (m + l.log())[:, 0]
        if bits < 24:
            f, e = torch.frexp(p)
            p = torch.ldexp(torch.round(f * 2.0 ** bits) / 2.0 ** bits, e)
        O[:, h] = p @ V[:, h // G].float() / l
    return O.to(Q.dtype), lse


SIZES = [(64, 3, 4, 1, 128, BF), (700, 5, 8, 2, 64, BF), (1025, 70, 4, 2, 128, BF), (20011, 1, 4, 1, 128, BF),
         (20011, 3, 4, 1, 64, F32), (65737, 3, 2, 1, 64, BF)]


@pytest.mark.parametrize("ctx,rows,hq,hkv,d,dtype", SIZES)
def test_right_results_pass(ctx, rows, hq, hkv, d, dtype):
    x = _inputs(ctx, rows, hq, hkv, d, dtype)
    ref = pn.reference(*x, 1 / math.sqrt(d))
    for bits in ((24,) if dtype == F32 else (8, 16)):
        assert max(pn.excess(*_like_the_kernel(*x, bits), ref, dtype == BF, bits > 8)) <= 1, bits


def _other_values(V, at, n):
    V = V.clone()
    V[at:at + n] = V[at + n:at + 2 * n].clone()
    return V


@pytest.mark.parametrize("ctx,rows,hq,hkv,d,dtype", [s for s in SIZES if s[0] > 10000])
def test_a_wrong_tile_of_a_long_context_is_seen(ctx, rows, hq, hkv, d, dtype):
    """A tile of 64 keys with another tile's values, or with none; a page look-up of 256
    keys that is one off."""
    Q, K, V, ok, pos = _inputs(ctx, rows, hq, hkv, d, dtype)
    ref = pn.reference(Q, K, V, ok, pos, 1 / math.sqrt(d))
    bits = 24 if dtype == F32 else 8
    for at, n in ((64, 64), (ctx // 2 // 64 * 64, 64), (4096, 256)):
        none = V.clone()
        none[at:at + n] = 0
        for wrong in (_other_values(V, at, n), none):
            eo, ez = pn.excess(*_like_the_kernel(Q, K, wrong, ok, pos, bits), ref, dtype == BF, False)
            assert eo > 1, (at, n, eo)


@pytest.mark.parametrize("ctx,rows,hq,hkv,d,dtype", [s for s in SIZES if s[0] > 10000])
def test_dropped_keys_of_a_long_context_are_seen(ctx, rows, hq, hkv, d, dtype):
    """16 keys by their part of the sum, 8e-4 of it at 20,011 and 2.4e-4 at 65,737, where
    lse is held to about 7e-5 and 1e-4 (S about 12: 4 (138 + 149) u; 9 with d = 64: 4 (74 +
    264) u). One key of 20,011, 5e-5, would be too few."""
    Q, K, V, ok, pos = _inputs(ctx, rows, hq, hkv, d, dtype)
    ref = pn.reference(Q, K, V, ok, pos, 1 / math.sqrt(d))
    for n in (16, 32):
        drop = slice(ctx // 3, ctx // 3 + n)
        eo, ez = pn.excess(*_like_the_kernel(Q, K, V, ok, pos, 24 if dtype == F32 else 8, drop), ref, dtype == BF, False)
        assert ez > 1, (n, ez)


@pytest.mark.parametrize("ctx,rows,hq,hkv,d,dtype", [s for s in SIZES if s[5] == BF])
def test_a_weight_of_too_few_bits_is_seen(ctx, rows, hq, hkv, d, dtype):
    """Over some rows: P as one bf16 value where it should be a pair, and P of five
    significant bits where it should be one."""
    x = _inputs(ctx, max(rows, 12 if ctx > 10000 else 24), hq, hkv, d, dtype, seed=2)
    ref = pn.reference(*x, 1 / math.sqrt(d))
    assert pn.rounding_ratio(_like_the_kernel(*x, 16)[0], ref[0]) < 1.1
    assert pn.rounding_ratio(_like_the_kernel(*x, 8)[0], ref[0]) > 1.1
    assert pn.excess(*_like_the_kernel(*x, 5), ref, True, False)[0] > 1
