"""Attention over the paged cache held to what its error should be, rather than to
what it could be.

The element bounds of tests/paged_oracle.py are worst cases: over n keys they grow
with sum p |v|, some sqrt(n) times |O|, and would let a wrong tile of a long
context pass. Here a row's error is a vector whose parts are independent: a
rounding of each weight moves O by a random walk over the keys, whose length is
W = sqrt(sum p^2 |v|^2) times the rounding, about |O| times it.

Bounds, with u = 2^-24, for a row over n keys, S the largest sum |q k| * scale:
  f32   = 4 (sqrt(d + 4) S + sqrt(n) + 8) u: roundings of a score's d products
          and of the scale, of the sums over n keys, and of exp2 and the joining;
          each at most u, added as a random walk, four times its length;
  |O - O64| <= r |O64| + w W + f32 (|O64| + W)   (2-norms of a row and head)
          r: half a step of the output type (bf16 2^-8, float32 2^-24);
          w: the rounding of P. 0 for float32 inputs; 1.5 * 2^-16 where P is a
          pair of bf16 values, 1.5 * 2^-8 where it is one (1.5: few keys of like
          weight, whose values are not quite at right angles);
  |lse - lse64| <= f32 + 4 u |lse64|.
Where P is a pair, the rounding of O is all that is left: over many rows the
error is that of O64 rounded to bf16, which is known, and 1.1 of it is allowed (P
as one bf16 value makes 1.4 of it)."""

import math

import torch

U = 2.0 ** -24


def reference(Q, K, V, ok, pos, scale):
    """Rows Q [n, Hq, d] at positions pos over K, V [L, Hkv, d] where ok [L], in
    float64: (O, lse, W, S, keys), W and S [n, Hq], keys [n]."""
    n, Hq, d = Q.shape
    G = Hq // K.shape[1]
    see = (torch.arange(K.shape[0])[None, :] <= pos[:, None]) & ok[None, :]
    O = torch.zeros(n, Hq, d, dtype=torch.float64)
    lse, W, S = (torch.zeros(n, Hq, dtype=torch.float64) for _ in range(3))
    for h in range(Hq):
        k, v, q = K[:, h // G].double(), V[:, h // G].double(), Q[:, h].double()
        score = (q @ k.T * scale).masked_fill(~see, -math.inf)
        S[:, h] = (q.abs() @ k.abs().T * scale).masked_fill(~see, 0.0).amax(-1)
        lse[:, h] = torch.logsumexp(score, -1)
        p = torch.exp(score - lse[:, h].clamp(min=-1e300)[:, None])
        O[:, h] = p @ v
        W[:, h] = (p * p @ (v * v).sum(-1, keepdim=True))[:, 0].sqrt()
    return O, lse, W, S, see.sum(-1)


def excess(O, lse, ref, bf16, pair):
    """The largest errors of O and of lse in parts of their bounds: at most 1 is right."""
    O64, z, W, S, keys = ref
    d = O64.shape[-1]
    f32 = 4 * (math.sqrt(d + 4) * S + keys.double().sqrt()[:, None] + 8) * U
    size = O64.norm(dim=-1)
    w = 0.0 if not bf16 else 1.5 * (2.0 ** -16 if pair else 2.0 ** -8)
    bound = (2.0 ** -8 if bf16 else U) * size + w * W + f32 * (size + W)
    eo = (O.double() - O64).norm(dim=-1) / bound.clamp(min=1e-300)
    ez = (lse.double() - z).abs() / (f32 + 4 * U * z.abs())
    some = keys > 0
    return float(eo[some].max()), float(ez[some].max())


def rounding_ratio(O, O64):
    """The error of a bf16 result over all rows in parts of that of O64 rounded to bf16."""
    return float((O.double() - O64).norm() / (O64.to(torch.bfloat16).double() - O64).norm())
