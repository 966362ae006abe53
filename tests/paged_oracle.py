"""The paged cache and its attention in float64 on the CPU, from their
definitions, and the bounds that the kernels' results are held to.

A row x is held in 8 bits as code * 2^e: e the least integer >= -100 with
max |x_j| <= 448 * 2^e over the finite elements, codes in e4m3 (steps of 2^-3
relative to the leading bit, least step 2^-9), ties to even; what is not
finite is NaN.
"""

import math

import torch


def held(x):
    """(values of the codes, exponents) of rows x [..., d]."""
    x = x.double()
    fine = torch.isfinite(x)
    a = torch.where(fine, x, 0.0).abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(a.clamp(min=2.0 ** -300) / 448.0)).clamp(min=-100.0)
    y = torch.where(fine, x, 0.0) / torch.exp2(e)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    code = torch.round(y / step) * step  # torch.round: ties to even
    return torch.where(fine, code, math.nan), e[..., 0]


def positions(seq_rows, q_begin, n_rows):
    """[(row, sequence, position)] of a batch."""
    out = []
    for s in range(len(q_begin)):
        for r in range(seq_rows[s], min(seq_rows[s + 1], n_rows)):
            out.append((r, s, q_begin[s] + r - seq_rows[s]))
    return out


def attend(Q, K, V, ok, pos, scale, rounding):
    """Attention of rows Q [n, Hq, d] at positions pos over K, V [L, Hkv, d]
    (float64) where ok [L], in float64: (O, lse, bound of O, bound of lse).

    The bounds. `rounding` is half a step of the output type (bf16 2^-8, float32
    2^-24). A score sums d products in float32, exact ones for bf16: d + 4
    roundings (the products' of float32, the scale, the shift by the maximum
    among them) of at most u = 2^-24 of the sum of magnitudes, so p is off by
    2 * delta, delta = (d + 4) u max sum |q k| scale, and by 2^-21 of exp2 and
    the factors that rescale it. l and O are sums of n terms: n u each, of
    l and of A = sum p |v|. bf16: p itself is rounded, which moves O by another
    2^-8 A; then O is rounded."""
    u = 2.0 ** -24
    n, Hq, d = Q.shape
    G = Hq // K.shape[1]
    t = torch.arange(K.shape[0])
    see = (t[None, :] <= pos[:, None]) & ok[None, :]
    O, lse = torch.zeros(n, Hq, d, dtype=torch.float64), torch.full((n, Hq), -math.inf, dtype=torch.float64)
    bo, bl = torch.zeros_like(O), torch.zeros_like(lse)
    for h in range(Hq):
        k, v, q = K[:, h // G].double(), V[:, h // G].double(), Q[:, h].double()
        score = (q @ k.T * scale).masked_fill(~see, -math.inf)
        size = (q.abs() @ k.abs().T * scale).masked_fill(~see, 0.0)
        z = torch.logsumexp(score, -1)
        p = torch.exp(score - torch.where(torch.isfinite(z), z, 0.0)[:, None])
        delta = (d + 4) * u * size.amax(-1)
        terms = see.sum(-1) * u
        vz = torch.where(see.any(0)[:, None], v, 0.0)
        O[:, h], lse[:, h] = p @ vz, z
        A = p @ vz.abs()
        rel = 2 * delta + 2 * terms + 2.0 ** -20
        if rounding > 2.0 ** -20:
            rel = rel + rounding
        bo[:, h] = rel[:, None] * A * (1 + rounding) + rounding * O[:, h].abs()
        bl[:, h] = delta + terms + 2.0 ** -20 + 4 * u * torch.where(torch.isfinite(z), z, 0.0).abs()
    return O, lse, bo, bl
