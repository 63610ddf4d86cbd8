"""Oracle for attention with a window, sinks and draft trees over a bf16 cache, and for the steps of a draft tree.

TEST INFRASTRUCTURE ONLY.  Only the tests may import this module; the product
path never does, and this module imports nothing from the product path.

Attention is fp64 and unrounded, on torch tensors of any device.  The tree's steps are plain Python over lists.
Pins: tests/test_oracle_kv_attn.py (closed forms and counted cases; none is "parity unpinned").
"""
from __future__ import annotations

import math

import torch

NO_SLOT = 1 << 40


def seen_from(pos, slots, window: int, sinks: int):
    """Which slots a query at each of `pos` sees: bool [len(pos)][len(slots)] (slots stand at their own positions)."""
    p, s = pos[:, None], slots[None]
    seen = s <= p
    if window > 0:
        seen = seen & ((s > p - window) | (s < sinks))
    return seen


def attend(q, k, v, seen, add=None, w_eps: float = 2.0 ** -16):
    """softmax(q . k / sqrt(d) + add) v of rows q [m][d] over keys k, v [n][d] (fp64), seen bool [m][n], add [n] or None.
    A row that sees nothing (or only -inf) is 0.  Returns out [m][d], tol [m][d], spread [m][d]:

    tol bounds the error of a computation with exact products summed in fp32 and weights rounded by w_eps, without
    the rounding of the result:
      a score is off by at most e = (d + 16) 2^-23 max_j (|q| . |k_j|) / sqrt(d) + 2^-21 max_j |z_j| (an addition is off by
      at most 2^-23 whatever its order; scaling, mask and the exponential's argument take a few operations);
      with every score off by at most e, a weight is off by a factor within exp(2 e), and so
      |error| <= sum_j w_j |v_j| (expm1(2 e) + w_eps + (n / 16 + 96) 2^-24 + 2^-14) + |out| w_eps + 2^-24 max|v|,
      the |out| w_eps where the sum that divides is of the rounded weights (sum_j w_j d_j (v_j - out), |d_j| <= w_eps),
      the last terms for the sums over n keys, of which a matrix instruction does 16 and more at a time, the
      exponential, the joining of parts and weights below fp32's range.
    spread is the standard deviation of the error that the weights' rounding alone makes, if the roundings are independent and
    spread evenly over +-w_eps: w_eps / sqrt(3) sqrt(sum_j w_j^2 v_j^2 + out^2 sum_j w_j^2) at most."""
    d, n = q.shape[-1], k.shape[0]
    kk = torch.where(seen.any(0)[:, None], k, 0.0)           # (keys that no row sees may be NaN)
    vv = torch.where(seen.any(0)[:, None], v, 0.0)
    z = q @ kk.T.contiguous() / math.sqrt(d)
    if add is not None:
        z = z + torch.where(seen.any(0), add, 0.0)[None]
    z = z.masked_fill(~seen, -math.inf)
    top = z.amax(-1, keepdim=True)
    p = torch.exp(z - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    w = p / torch.where(total == 0, 1.0, total)
    reach = (q.abs() @ kk.abs().T.contiguous() / math.sqrt(d)).masked_fill(~(z > -math.inf), 0.0).amax(-1)
    e = (d + 16) * 2.0 ** -23 * reach + 2.0 ** -21 * z.masked_fill(z == -math.inf, 0.0).abs().amax(-1)
    tol = (w @ vv.abs()) * (torch.expm1(2 * e) + w_eps + (n / 16 + 96) * 2.0 ** -24 + 2.0 ** -14)[:, None] + 2.0 ** -24 * vv.abs().amax()
    out = w @ vv
    return out, tol + out.abs() * w_eps, w_eps / math.sqrt(3) * torch.sqrt(w ** 2 @ vv ** 2 + out ** 2 * (w ** 2).sum(-1, keepdim=True))


# ------------------------------------------------------------- draft trees

def ancestors(parents, i):
    """Node i and the nodes above it, upwards; parents[i] outside 0 .. i - 1 is none."""
    chain = [i]
    while 0 <= parents[chain[-1]] < chain[-1]:
        chain.append(parents[chain[-1]])
    return chain


def plan(parents, ctx: int, window: int, sinks: int):
    """Positions [N] and sets of the nodes that each node sees."""
    chains = [ancestors(parents, i) for i in range(len(parents))]
    pos = [max(ctx, 0) + len(c) - 1 for c in chains]
    return pos, [{a for a in c if window == 0 or pos[a] > pos[i] - window or pos[a] < sinks} for i, c in enumerate(chains)]


def words(sets, N: int):
    """The sets as words of 64 bits, as signed integers."""
    out = []
    for s in sets:
        row = [sum(1 << (a % 64) for a in s if a // 64 == w) for w in range((N + 63) // 64)]
        out.append([x - (1 << 64) if x >> 63 else x for x in row])
    return out


def accept(parents, tokens, picks):
    """The path's nodes, and the pick of the last one."""
    path = [0]
    while True:
        below = [c for c in range(len(parents)) if 0 <= parents[c] < c and parents[c] == path[-1] and tokens[c] == picks[path[-1]]]
        if not below:
            return path, picks[path[-1]]
        path.append(below[0])
