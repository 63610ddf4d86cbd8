"""Prefill attention over the 4-bit cache, every query of a call, in every way in which the work is dealt out (row tiles
whole, in parts with their states merged, as a line that the blocks cut into equal runs, as rows of the decode
kernel), with queries that look at every stage of keys and at the causal border.  The bound is that of
oracle.kv4.attend_heads for the operands that the kernel multiplies, plus the rounding of the output (2^-8);
tests/test_oracle_kv4_probing.py shows which mistakes pass it."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import kv4 as O
from oracle.layer import round_bf16
from paper_2607_15865_amd import binding, synth
from gpu_helpers import log

pytestmark = pytest.mark.gpu

# form, heads, kv heads, head dim, queries, history
CASES = [
    ("runs", 22, 11, 64, 2447, 498), ("runs", 35, 5, 64, 1492, 387), ("runs", 15, 15, 64, 2255, 989),
    ("runs", 77, 11, 64, 404, 1031), ("runs", 32, 8, 128, 700, 4000), ("runs", 25, 5, 128, 1997, 536),
    ("runs", 48, 16, 128, 1383, 841), ("runs", 32, 4, 128, 700, 4000),
    ("parts", 1, 1, 128, 594, 290), ("parts", 14, 2, 64, 511, 700), ("parts", 5, 5, 64, 73, 2842),
    ("parts", 56, 8, 128, 65, 1000), ("parts", 7, 1, 128, 900, 4000), ("parts", 32, 16, 128, 31, 1055),
    ("parts", 64, 64, 64, 9, 2100), ("parts", 24, 8, 64, 401, 31),
    ("whole", 48, 12, 64, 292, 0), ("whole", 33, 11, 128, 225, 0), ("whole", 64, 8, 128, 1500, 1), ("whole", 40, 8, 64, 2049, 63),
    ("rows", 8, 2, 128, 33, 300), ("rows", 14, 2, 64, 61, 250), ("rows", 7, 1, 128, 5, 4000), ("rows", 32, 8, 128, 1, 2100),
    ("rows", 16, 8, 64, 4, 70000), ("rows", 16, 8, 128, 1, 70001), ("rows", 28, 4, 128, 2, 70002)]
BIG = [("runs", 60, 12, 128, 530, 1911), ("parts", 32, 16, 128, 120, 213), ("rows", 8, 2, 128, 70, 263)]


def form_of(nq, nkv, d, T, hist):
    single, chunk, blocks, merge = (ctypes.c_int() for _ in range(4))
    binding._lib.w4_kv4_prefill_plan(T, hist, nkv, nq // nkv, d, *(ctypes.byref(x) for x in (single, chunk, blocks, merge)))
    return "rows" if single.value else "runs" if not chunk.value else "parts" if merge.value else "whole"


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).cuda().to(torch.bfloat16)


def f64(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float64)).cuda()


def values(rng, shape, scale=1.0):
    x = rng.standard_normal(shape) + (rng.random(shape[-1]) < 0.06) * rng.standard_normal(shape[-1]) * 5
    return round_bf16(np.clip(x * scale, -65280, 65280))


def cache_of(nq, nkv, d, k, v, max_seq):
    """k, v [n][nkv][d] in row 1 of a cache of two, everything else NaN."""
    cfg = synth.replace(synth.CONFIGS["llama8b"], n_heads=nq, n_kv_heads=nkv, head_dim=d, max_seq=max_seq)
    c = binding.KV4Cache(cfg, 2)
    c.k.fill_(0xFF), c.v.fill_(0xFF)
    both = [torch.stack([torch.full_like(dev(x), float("nan")), dev(x)]) for x in (k, v)]
    c.append(*both, [0, 0])
    return c


def prefill(c, q, hist):
    out = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
    c.attn_prefill(dev(q), hist, out, row=1)
    torch.cuda.synchronize()
    return out.double()


def operands(x, form):
    """What a value is multiplied as, [nkv][n][d], and the magnitudes of its parts."""
    codes, s, lo = O.quantise(np.swapaxes(x, 0, 1))
    held = O.values(codes, s, lo)
    if form != "rows":
        return f64(O.fp16_operands(held)), None
    return f64(held), f64(O.values(codes, s, np.abs(lo)))


def check_all(got, q, k, v, hist, form, what, skip=None):
    """Every element; skip [T][nq][d] bool: not compared."""
    (ko, kp), (vo, vp) = operands(k, form), operands(v, form)
    worst = 0.0
    pair = form == "rows"                                    # weights times scales as pairs of fp16: 2^-20, and 2^-24 a key
    for h, out, tol in O.attend_heads(f64(q), ko, vo, hist, kp, vp, w_eps=2.0 ** -20 if pair else 2.0 ** -11):
        lim = (tol + (k.shape[0] * 2.0 ** -24 if pair else 0.0)) * 1.01 + out.abs() * 2.0 ** -8
        err = (got[:, h] - out).abs()
        if skip is not None:
            err = torch.where(torch.from_numpy(skip[:, h]).cuda(), 0.0, err)
        assert torch.isfinite(err).all(), f"{what} head {h}"
        bad = (err > lim).nonzero()
        assert bad.numel() == 0, f"{what} head {h}: {bad.shape[0]} elements, first (query, dim) {bad[0].tolist()}"
        worst = max(worst, float((err / lim.clamp(min=1e-300)).max()))
    log(f"  {what}: {worst:.3f} of the bound")


@pytest.mark.parametrize("form,nq,nkv,d,T,hist", CASES)
def test_every_query(form, nq, nkv, d, T, hist):
    log(f"{form} heads {nq}/{nkv} d {d} T {T} hist {hist}")
    assert form_of(nq, nkv, d, T, hist) == form
    rng = np.random.default_rng(T + nq)
    n = hist + T
    k, v = values(rng, (n, nkv, d)), values(rng, (n, nkv, d))
    q = O.probing_queries(rng, np.swapaxes(O.held(k), 0, 1), nq, T, hist)
    c = cache_of(nq, nkv, d, k, v, n + 3)
    got = prefill(c, q, hist)
    check_all(got, q, k, v, hist, form, "all queries")


@pytest.mark.parametrize("qscale,vscale", [(1e-6, 1.0), (1.0, 300.0), (1e4, 1.0), (30.0, 15000.0), (1.0, 1e-4)])
@pytest.mark.parametrize("form,nq,nkv,d,T,hist", BIG)
def test_ranges(form, nq, nkv, d, T, hist, qscale, vscale):
    """Scores from equal to one that wins by far, values over fp16's range."""
    log(f"{form} heads {nq}/{nkv} d {d} T {T} hist {hist} q {qscale} v {vscale}")
    assert form_of(nq, nkv, d, T, hist) == form
    rng = np.random.default_rng(40)
    n = hist + T
    k, v = values(rng, (n, nkv, d)), values(rng, (n, nkv, d), vscale)
    q = round_bf16(O.probing_queries(rng, np.swapaxes(O.held(k), 0, 1), nq, T, hist) * qscale)
    check_all(prefill(cache_of(nq, nkv, d, k, v, n), q, hist), q, k, v, hist, form, "all queries")


@pytest.mark.parametrize("form,nq,nkv,d,T,hist", [CASES[1], CASES[4], CASES[7], CASES[9], CASES[18]])
def test_nan_reaches_exactly_the_rows_that_see_it(form, nq, nkv, d, T, hist):
    """NaN values (their group's dims) and keys (all dims) of single tokens, at the borders of tiles and stages and
    between: the queries from that token on, of that kv head; all other elements within the bound."""
    log(f"{form} heads {nq}/{nkv} d {d} T {T} hist {hist}")
    assert form_of(nq, nkv, d, T, hist) == form
    rng = np.random.default_rng(50)
    n, r = hist + T, nq // nkv
    k, v = values(rng, (n, nkv, d)), values(rng, (n, nkv, d))
    want = np.zeros((T, nq, d), bool)
    border = (hist + T // 2) // 64 * 64
    for i, j in enumerate((border - 1, border, border + 31, border + 32, n - 1, hist + T // 3)):
        g, dim = i % nkv, (37 * i + 5) % d
        v[j, g, dim] = np.inf if i % 2 else np.nan
        want[max(j - hist, 0):, g * r:(g + 1) * r, dim // 32 * 32:dim // 32 * 32 + 32] = True
    j, g = hist + T * 3 // 4, nkv - 1
    k[j, g, 1] = np.nan
    want[j - hist:, g * r:(g + 1) * r] = True
    c = cache_of(nq, nkv, d, k, v, n + 64)
    q = round_bf16(rng.standard_normal((T, nq, d)))
    got = prefill(c, q, hist)
    assert np.array_equal(torch.isnan(got).cpu().numpy(), want)
    for x in (k, v):
        x[~np.isfinite(x)] = 0.0
    # (the other 31 dims of a group with a NaN were held as NaN: no element compared sees them)
    check_all(got, q, k, v, hist, form, "the others", skip=want)


def test_forms_agree_at_their_borders():
    """One query after another as calls of the decode kernel's rows and of the prefill kernel: each within the bound of
    its operands."""
    nq, nkv, d, T, hist = 32, 16, 128, 120, 300
    rng = np.random.default_rng(60)
    n = hist + T
    k, v = values(rng, (n, nkv, d)), values(rng, (n, nkv, d))
    q = O.probing_queries(rng, np.swapaxes(O.held(k), 0, 1), nq, T, hist)
    c = cache_of(nq, nkv, d, k, v, n)
    forms = set()
    for at, m in ((0, T), (0, 1), (1, 8), (9, 40), (49, 71)):
        form = form_of(nq, nkv, d, m, hist + at)
        forms.add(form)
        got = prefill(c, q[at:at + m], hist + at)
        check_all(got, q[at:at + m], k[:hist + at + m], v[:hist + at + m], hist + at, form, f"queries {at} .. {at + m - 1}")
    assert {"rows", "parts"} <= forms


@pytest.mark.parametrize("nq,nkv,d", [(8, 2, 128), (14, 2, 64), (7, 1, 128)])
@pytest.mark.parametrize("qscale", [30.0, 1e4])
def test_decode_with_large_queries(nq, nkv, d, qscale):
    """The decode kernel where one key wins, by the same bound (the keys as they are held, in parts)."""
    log(f"decode heads {nq}/{nkv} d {d} q {qscale}")
    rng = np.random.default_rng(70)
    ctx = [699, 77, 0]
    n = max(ctx) + 1
    cfg = synth.replace(synth.CONFIGS["llama8b"], n_heads=nq, n_kv_heads=nkv, head_dim=d, max_seq=n)
    c = binding.KV4Cache(cfg, 3)
    k, v = values(rng, (3, n, nkv, d)), values(rng, (3, n, nkv, d))
    c.append(dev(k), dev(v), [0, 0, 0])
    q = round_bf16(np.concatenate([O.probing_queries(rng, np.swapaxes(O.held(k[b]), 0, 1), nq, 1, ctx[b]) for b in range(3)]) * qscale)
    out = torch.empty((3, nq, d), dtype=torch.bfloat16, device="cuda")
    c.attn_decode(dev(q), torch.tensor(ctx, dtype=torch.int32, device="cuda"), n - 1, out)
    torch.cuda.synchronize()
    for b in range(3):
        m = ctx[b] + 1
        check_all(out[b:b + 1].double(), q[b:b + 1], k[b, :m], v[b, :m], ctx[b], "rows", f"row {b}")
