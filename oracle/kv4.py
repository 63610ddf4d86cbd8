"""CPU oracle for the key/value cache held in 4 bits.

TEST INFRASTRUCTURE ONLY.  Only the tests may import this module; the product
path never does, and this module imports nothing from the product path.

Per token and kv head the dims are cut into groups of 32.  Of a group's values
x, taken as fp16:  lo = min x,  s = fp16((max x - lo) / 15),
c = min(15, floor((x - lo) / s + 1/2)) (0 where s = 0); the value held is
lo + s c.  A group with a value that has no fp16 value is NaN throughout.

Everything is fp64 and unrounded, except where the definition rounds.  fp64
holds the differences and borders exactly: fp16 values are multiples of 2^-24
below 2^16 (41 bits), a border (k + 1/2) s has 16 bits.

Pins: tests/test_oracle_kv4.py checks each function against rational
arithmetic and closed forms; none is "parity unpinned".
"""
from __future__ import annotations

import numpy as np

from oracle import layer as _layer

F64 = np.float64
GROUP = 32


def quantise(x):
    """codes, s, lo of values [..][d]: uint8 [..][d], fp64 [..][d / 32] twice."""
    x = np.asarray(x, dtype=F64)
    with np.errstate(over="ignore", invalid="ignore"):
        x = x.astype(np.float16).astype(F64)
    g = x.reshape(x.shape[:-1] + (-1, GROUP))
    bad = ~np.isfinite(g).all(-1)
    g = np.where(bad[..., None], 0.0, g)
    lo, hi = g.min(-1), g.max(-1)
    s = ((hi - lo) / 15).astype(np.float16).astype(F64)
    t = g - lo[..., None]
    with np.errstate(divide="ignore", invalid="ignore"):
        c = np.where(s[..., None] > 0, np.floor(t / s[..., None] + 0.5), 0.0)
    c = np.minimum(c, 15).astype(np.uint8)
    nan = np.where(bad, np.nan, 0.0)
    return c.reshape(x.shape), s + nan, lo + nan


def values(codes, s, lo) -> np.ndarray:
    g = codes.astype(F64).reshape(codes.shape[:-1] + (-1, GROUP))
    return (lo[..., None] + s[..., None] * g).reshape(codes.shape)


def held(x) -> np.ndarray:
    """The values a cache holds of x."""
    return values(*quantise(x))


def attend(q, k, v, seen, add=None, key_eps: float = 0.0):
    """Attention of q [nq][d] over keys / values k, v [nkv][n][d] (fp64),
    seen [n] bool, add [n] (the mask's values) or None; the scores are scaled by
    d^-1/2.  Returns out [nq][d] and a bound on the error of a computation in
    which the scores' sums are fp32, every key is off by at most key_eps
    relative to its group's largest magnitude, and weights and values are each
    rounded to fp16; without the rounding of the result:

      a score is off by at most e = (key_eps + (d + 16) 2^-24) 3 sum|q| max|k| / sqrt(d)
      (3: s, lo and code are multiplied apart, each part at most 2 max|k|, in
      sum) plus 2^-21 max|score| (its scaling, the exponential's argument);
      weights are then off by a factor within exp(2 e), and
      |out error| <= sum_j w_j |v_j| (exp(2 e) - 1 + 2^-11 + 2^-11 + 2^-14) + 2^-24 (1 + max|v|)
      (2^-14: the exponential and the fp32 sums of the weights)."""
    nq, d = q.shape
    nkv, n, _ = k.shape
    r = nq // nkv
    out, tol = np.zeros((nq, d)), np.zeros((nq, d))
    if not np.any(seen):
        return out, tol
    for h in range(nq):
        kk, vv = k[h // r][seen], v[h // r][seen]
        z = kk @ q[h] / np.sqrt(d)
        e = (key_eps + (d + 16) * 2.0 ** -24) * 3 * np.abs(q[h]).sum() * np.abs(kk).max() / np.sqrt(d)
        e += 2.0 ** -21 * np.abs(z).max()
        if add is not None:
            z = z + add[seen]
        p = np.exp(z - z.max())
        w = p / p.sum()
        out[h] = w @ vv
        tol[h] = (w @ np.abs(vv)) * (np.expm1(2 * e) + 2.0 ** -10 + 2.0 ** -14) + 2.0 ** -24 * (1 + np.abs(vv).max())
    return out, tol


def fp16_operands(x):
    """Values held, as the prefill kernel multiplies them: lo + s c rounded once to fp16 (still fp64)."""
    return np.asarray(x, dtype=F64).astype(np.float16).astype(F64)


def attend_heads(q, k, v, first, kparts=None, vparts=None, w_eps=2.0 ** -11, drop=None):
    """Causal attention of all queries, head by head: q [T][nq][d], k, v [nkv][n][d] torch fp64 tensors, the very
    operands that a computation multiplies (fp16_operands for the prefill kernel); query t sees keys 0 .. first + t.
    kparts, vparts: where a key or value is multiplied in parts (scale times code, offset), the sum of the parts'
    magnitudes; w_eps: the rounding of a weight; drop(t0, t1) for a planted mistake: [t1 - t0][n] bool, keys left out.
    Yields (head, out [T][d], tol [T][d]); tol bounds the error of fp32 sums of exact products, before the result is
    rounded:

      A score's d products are exact in fp32 and summed there; with an addition off by at most 2^-23, in whatever
      order, and a few operations on the sum, the argument of the exponential is off by at most
          e = (d + 16) 2^-23 max_j (|q| . |k_j|) / sqrt(d) + 2^-21 max_j |z_j|.
      Scores off by at most e either way change the weight w_j by a factor 1 + f, |f| <= (1 - w_j) expm1(2 e): with
      every other score moved against it w' / w = 1 / (w + (1 - w) exp(-+2 e)), for which that holds.
      Rounded to 2^-11 (w_eps), or, in fp16's subnormals, by at most 2^-25 of the largest weight's unit, and never by
      more than itself.  n additions to the output and to the weights' sum in fp32, of which a matrix instruction does
      16 and more at a time: (n / 2 + 96) 2^-24.  2^-20: the exponential, the final division, the joining of parts."""
    import torch
    T, nq, d = q.shape
    nkv, n, _ = k.shape
    r = nq // nkv
    kparts = k.abs() if kparts is None else kparts
    vparts = v.abs() if vparts is None else vparts
    seen = torch.arange(n, device=q.device)[None] <= torch.arange(T, device=q.device)[:, None] + first
    if drop is not None:
        seen = seen & ~drop
    scale = float(d) ** -0.5
    for h in range(nq):
        qh, kh = q[:, h].contiguous(), k[h // r].t().contiguous()
        z = (qh @ kh) * scale
        z = torch.where(seen, z, -torch.inf)
        zmax = z.amax(-1, keepdim=True)
        mag = (qh.abs() @ kparts[h // r].t().contiguous()) * scale
        e = (d + 16) * 2.0 ** -23 * torch.where(seen, mag, 0.0).amax(-1, keepdim=True)
        e += 2.0 ** -21 * torch.where(seen, z.abs(), 0.0).amax(-1, keepdim=True)
        p = torch.exp(z - zmax)
        total = p.sum(-1, keepdim=True)
        w = p / total
        out = w @ v[h // r]
        rel = (1 - w) * torch.expm1(2 * e.clamp(max=50)) + (w_eps + (n / 2 + 96) * 2.0 ** -24 + 2.0 ** -20)
        tol = (w * rel) @ vparts[h // r] + (p.clamp(max=2.0 ** -25) / total) @ vparts[h // r]
        yield h, out, tol


def probing_queries(rng, k, nq, T, first):
    """Queries [T][nq][d] whose outputs show every key: rows (query, head) of a kv head in order, every other one near
    one key of a stage of 64 after another (its first, last or some key), of the rest each fourth near the last key seen,
    the first one hidden, key 0, and nowhere in particular.  "Near" a key: six times its difference from the
    keys' mean, which puts nearly all the weight on it.  k [nkv][n][d]."""
    nkv, n, d = k.shape
    r = nq // nkv
    mean = k.mean(1)
    q = np.empty((T, nq, d))
    for g in range(nkv):
        for i in range(T * r):
            t, h = divmod(i, r)
            last, kind = first + t, i % 8
            if kind % 2 == 0:
                st = (i // 2) % (last // 64 + 1)
                j = min(last, 64 * st + (0, 63, int(rng.integers(64)))[(i // 2 + i // 512) % 3])
            else:
                j = {1: last, 3: min(last + 1, n - 1), 5: 0, 7: -1}[kind]
            q[t, g * r + h] = rng.standard_normal(d) if j < 0 else 6.0 * (k[g, j] - mean[g])
    return _layer.round_bf16(q)


def block(w: dict, cfg, x, pos, k_hist=None, v_hist=None, bias=None, rows=None, W=None):
    """oracle.layer.block for a layer whose cache is held in 4 bits: the new
    keys and values (bf16 after RoPE, as they are formed there) enter the cache,
    and every key and value that the attention sees, the call's own among them,
    is what the cache holds.  k_hist, v_hist: the values held, [nkv][L][d].
    Returns y and the values held of the new k, v [T][nkv][d]."""
    nq, d = cfg.n_heads, cfg.head_dim
    W = _layer.dequant_layer(w, cfg) if W is None else W
    x = np.asarray(x, dtype=F64)
    T = x.shape[0]
    sel = np.arange(T) if rows is None else np.asarray(rows)
    xn = _layer.round_bf16(_layer.rmsnorm(x, _layer.bf16_to_f64(w["attn_norm"]), cfg.rms_eps))
    cos, sin = _layer.rope_cos_sin(pos, d, cfg.rope_base)
    q = _layer.round_bf16(_layer.rope((xn[sel] @ W["q"]).reshape(len(sel), nq, d), cos[sel], sin[sel]))
    k = held(_layer.round_bf16(_layer.rope((xn @ W["k"]).reshape(T, -1, d), cos, sin)))
    v = held(_layer.round_bf16((xn @ W["v"]).reshape(T, -1, d)))
    L = 0 if k_hist is None else k_hist.shape[1]
    k_all = k if not L else np.concatenate([k_hist.transpose(1, 0, 2), k])
    v_all = v if not L else np.concatenate([v_hist.transpose(1, 0, 2), v])
    b = None if bias is None else np.asarray(bias, dtype=F64)[sel]
    a = _layer.round_bf16(_layer.attention(q, k_all, v_all, L + sel, b).reshape(len(sel), nq * d))
    h = x[sel] + a @ W["o"]
    hn = _layer.round_bf16(_layer.rmsnorm(h, _layer.bf16_to_f64(w["mlp_norm"]), cfg.rms_eps))
    g = _layer.round_bf16(_layer.silu(hn @ W["gate"]) * (hn @ W["up"]))
    return h + g @ W["down"], k, v
