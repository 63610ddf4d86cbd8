"""The 4-bit key/value cache on the GPU against its fp64 oracle (oracle/kv4.py).

Written and read back: bit for bit (the codes are those of exact arithmetic,
the values are rounded once).  Attention: element by element within the
bound that the oracle derives for fp32 sums and fp16 operands, plus the
rounding of the output (2^-8 relative).
"""
import numpy as np
import pytest
import torch

from oracle import kv4 as O
from oracle.layer import round_bf16
from paper_2607_15865_amd import binding, synth
from gpu_helpers import log

pytestmark = pytest.mark.gpu

HEADS = [(14, 2, 64), (8, 8, 64), (16, 2, 64), (1, 1, 128), (8, 2, 128), (7, 1, 128), (16, 2, 128), (9, 3, 128)]


def config(nq, nkv, d, max_seq):
    return synth.replace(synth.CONFIGS["llama8b"], n_heads=nq, n_kv_heads=nkv, head_dim=d, max_seq=max_seq)


def bf16_values(rng, shape, scale=1.0):
    """Values with a few far channels, as float32 that are bf16 numbers."""
    x = rng.standard_normal(shape) + (rng.random(shape[-1]) < 0.06) * rng.standard_normal(shape[-1]) * 5
    return round_bf16(x * scale).astype(np.float32)


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda().to(torch.bfloat16)


def host(t):
    return t.float().cpu().numpy().astype(np.float64)


def expected_read(x):
    """bf16 of the fp32 of lo + s c (one fma, one rounding)."""
    h = O.held(x).astype(np.float32).astype(np.float64)
    return np.where(np.isnan(h), np.nan, round_bf16(np.nan_to_num(h)))


def new_cache(cfg, batch, fill=None):
    c = binding.KV4Cache(cfg, batch)
    for t in (c.k, c.v):
        t.fill_(0xFF if fill is None else fill)              # (0xFFFF: an fp16 NaN)
    return c


def read(c, slots, T):
    shape = (len(slots), T, c.desc.n_kv_heads, c.desc.head_dim)
    k, v = (torch.full(shape, 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    c.read(slots, T, k, v)
    torch.cuda.synchronize()
    return host(k), host(v)


# ------------------------------------------------------------- write and read

@pytest.mark.parametrize("nkv,d", [(2, 64), (1, 128), (3, 128)])
@pytest.mark.parametrize("slots,T", [([0], 1), ([31], 1), ([5], 8), ([0], 32), ([7, 40, 0], 33), ([30, 1], 100), ([0], 257)])
def test_append_read_round_trip(nkv, d, slots, T):
    log(f"round trip nkv {nkv} d {d} slots {slots} T {T}")
    rng = np.random.default_rng(T + d)
    c = new_cache(config(nkv, nkv, d, 300), len(slots) + 1)
    k, v = (bf16_values(rng, (len(slots), T, nkv, d), s) for s in (1.0, 0.3))
    c.append(dev(k), dev(v), slots)
    gk, gv = read(c, slots, T)
    assert np.array_equal(gk, expected_read(k)) and np.array_equal(gv, expected_read(v))


@pytest.mark.parametrize("d", [64, 128])
def test_append_leaves_other_slots_alone(d):
    """Every byte of a cache filled at random, then one run: the slots around it, the other sequence and the padding
    keep their values (by slot through the reader; the bytes that changed belong to the run)."""
    cfg = config(2, 2, d, 90)
    rng = np.random.default_rng(3)
    c = new_cache(cfg, 2)
    k, v = (bf16_values(rng, (2, 90, 2, d)) for _ in range(2))
    c.append(dev(k), dev(v), [0, 0])
    for start, T in ((0, 1), (17, 1), (31, 2), (40, 9), (89, 1), (60, 30)):
        before = [t.clone() for t in (c.k, c.v)]
        kn, vn = (bf16_values(rng, (1, T, 2, d)) for _ in range(2))
        c.append(dev(kn), dev(vn), [start])
        k[0, start:start + T], v[0, start:start + T] = kn[0], vn[0]
        gk, gv = read(c, [0, 0], 90)
        assert np.array_equal(gk, expected_read(k)) and np.array_equal(gv, expected_read(v)), (start, T)
        for a, b in zip(before, (c.k, c.v)):
            assert int((a != b).sum()) <= T * 2 * (d // 32) * 20 + T * 2 * d // 2
            assert torch.equal(a[c.desc.stride_b:], b[c.desc.stride_b:])


def test_append_in_pieces_equals_append_at_once():
    cfg = config(8, 2, 128, 130)
    rng = np.random.default_rng(4)
    k, v = (dev(bf16_values(rng, (1, 130, 2, 128))) for _ in range(2))
    whole, pieces, steps = (new_cache(cfg, 1, 0) for _ in range(3))
    whole.append(k, v, [0])
    at = 0
    for n in (1, 2, 29, 5, 64, 29):
        pieces.append(k[:, at:at + n].contiguous(), v[:, at:at + n].contiguous(), [at])
        at += n
    for i in range(130):
        steps.append_step(k[:, i].contiguous(), v[:, i].contiguous(), torch.tensor([i], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    for other in (pieces, steps):
        assert torch.equal(whole.k, other.k) and torch.equal(whole.v, other.v)


def test_append_step_skips_slots_outside():
    cfg = config(2, 2, 64, 40)
    rng = np.random.default_rng(5)
    c = new_cache(cfg, 4, 0x11)
    before = [t.clone() for t in (c.k, c.v)]
    k, v = (bf16_values(rng, (4, 1, 2, 64)) for _ in range(2))
    c.append_step(dev(k), dev(v), torch.tensor([-1, 39, 40, 2 ** 31 - 1], dtype=torch.int32, device="cuda"))
    gk, gv = read(c, [0, 39, 0, 0], 1)
    assert np.array_equal(gk[1], expected_read(k)[1]) and np.array_equal(gv[1], expected_read(v)[1])
    n = c.desc.stride_b
    for a, b in zip(before, (c.k, c.v)):
        for row in (0, 2, 3):
            assert torch.equal(a[row * n:(row + 1) * n], b[row * n:(row + 1) * n])


@pytest.mark.parametrize("kind", ["ties", "constant", "tiny", "subnormal", "wide", "huge", "largest", "zeros"])
def test_codes_next_to_borders(kind):
    """Values on and next to the borders between codes, over fp16's whole range, bit for bit."""
    rng = np.random.default_rng(6)
    n, d = 64, 128
    if kind == "ties":                                       # s = 2^e, many values exactly half way
        x = rng.integers(0, 31, (n, d)) / 2.0
        x[:, ::32], x[:, 1::32] = 0.0, 15.0
        x = x * 2.0 ** rng.integers(-8, 8, (n, 1)) - 2.0 ** rng.integers(-3, 3, (n, 1))
    elif kind == "constant":
        x = np.repeat(rng.standard_normal((n, d // 32)), 32, axis=1)
    elif kind == "tiny":
        x = rng.standard_normal((n, d)) * 2.0 ** -16
    elif kind == "subnormal":
        x = rng.standard_normal((n, d)) * 2.0 ** -22
    elif kind == "wide":                                     # differences of more than 24 bits
        x = rng.choice([-3.0, 4.5, 12.0], (n, d)) + 0.0
        x[:, 2::3] = rng.standard_normal(x[:, 2::3].shape) * 2.0 ** -23
    elif kind == "huge":
        x = rng.standard_normal((n, d)) * 15000
    elif kind == "largest":
        x = rng.choice([-65280.0, 65280.0, 1.0, 32000.0], (n, d))
    else:
        x = np.where(rng.random((n, d)) < 0.5, 0.0, -0.0)
    x = round_bf16(np.clip(x, -65280, 65280)).astype(np.float32).reshape(1, n, 1, d)
    c = new_cache(config(1, 1, d, n), 1)
    c.append(dev(x), dev(-x), [0])
    gk, gv = read(c, [0], n)
    assert np.array_equal(gk, expected_read(x)) and np.array_equal(gv, expected_read(-x))


def test_groups_without_fp16_values_read_back_as_nan():
    x = np.ones((1, 40, 1, 128), dtype=np.float32)
    x[0, 3, 0, 33], x[0, 9, 0, 127], x[0, 20, 0, 0], x[0, 33, 0, 64] = np.nan, np.inf, -np.inf, 65536.0
    c = new_cache(config(1, 1, 128, 40), 1, 0)
    c.append(dev(x), dev(x), [0])
    for got in read(c, [0], 40):
        ref = expected_read(x)
        assert np.isnan(ref).sum() == 4 * 32
        assert np.array_equal(got, ref, equal_nan=True)


# ------------------------------------------------------------------ attention

def check(got, ref, tol, what):
    """got within the oracle's bound and the rounding to bf16."""
    lim = tol * 1.01 + np.abs(ref) * 2.0 ** -8
    err = np.abs(got - ref)
    worst = float(np.max(np.where(err == 0, 0.0, err / np.maximum(lim, 1e-300))))     # (a bound of 0 asks for 0)
    log(f"  {what}: {worst:.3f} of the bound")
    assert np.isfinite(got).all(), what
    assert worst <= 1.0, f"{what}: {worst} of the bound"


def filled(nq, nkv, d, B, n, seed=0, max_seq=None, kscale=1.0):
    rng = np.random.default_rng(seed)
    c = new_cache(config(nq, nkv, d, max_seq or n), B)
    k, v = bf16_values(rng, (B, n, nkv, d), kscale), bf16_values(rng, (B, n, nkv, d))
    c.append(dev(k), dev(v), [0] * B)
    kh, vh = (np.ascontiguousarray(np.swapaxes(O.held(x), 1, 2)) for x in (k, v))    # [B][nkv][n][d]
    return c, kh, vh, rng


def decode(c, q, ctx, max_ctx=None, mask=None):
    out = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
    c.attn_decode(dev(q), torch.tensor(ctx, dtype=torch.int32, device="cuda"), max(ctx) if max_ctx is None else max_ctx, out,
                  attn_mask=None if mask is None else torch.from_numpy(mask).cuda())
    torch.cuda.synchronize()
    return host(out)


def check_decode(c, kh, vh, q, ctx, got, mask, what):
    for b, n in enumerate(ctx):
        seen, add = np.arange(kh.shape[2]) <= n, None
        if mask is not None:
            add = mask[b, :kh.shape[2]].astype(np.float64)
            seen &= add != -np.inf
        ref, tol = O.attend(q[b].astype(np.float64), kh[b], vh[b], seen, add)
        check(got[b], ref, tol, f"{what} row {b} ctx {n}")


@pytest.mark.parametrize("nq,nkv,d", HEADS)
@pytest.mark.parametrize("ctx", [[0], [1, 30, 31], [32, 0, 33, 62, -1, 64], [255, 256, 7], [1030]])
def test_decode_attention(nq, nkv, d, ctx):
    log(f"decode heads {nq}/{nkv} d {d} ctx {ctx}")
    c, kh, vh, rng = filled(nq, nkv, d, len(ctx), max(ctx) + 1, seed=len(ctx))
    q = bf16_values(rng, (len(ctx), nq, d))
    got = decode(c, q, ctx)
    check_decode(c, kh, vh, q, ctx, got, None, "decode")
    for b, n in enumerate(ctx):
        if n < 0:
            assert not got[b].any()


@pytest.mark.parametrize("nq,nkv,d,B,ctx", [(32, 8, 128, 1, 2048), (28, 4, 128, 3, 4097), (14, 2, 64, 2, 5000),
                                            (8, 1, 128, 1, 16385), (4, 4, 64, 40, 300)])
def test_decode_attention_long(nq, nkv, d, B, ctx):
    log(f"decode heads {nq}/{nkv} d {d} B {B} ctx {ctx}")
    rng = np.random.default_rng(9)
    lens = [ctx] + [int(rng.integers(0, ctx + 1)) for _ in range(B - 1)]
    c, kh, vh, rng = filled(nq, nkv, d, B, ctx + 1, seed=7)
    q = bf16_values(rng, (B, nq, d))
    check_decode(c, kh, vh, q, lens, decode(c, q, lens), None, "decode")


@pytest.mark.parametrize("nq,nkv,d", [(14, 2, 64), (8, 2, 128), (7, 1, 128)])
@pytest.mark.parametrize("kind", ["left", "random", "bias", "most", "lowest"])
def test_decode_mask(nq, nkv, d, kind):
    """Additive masks; hidden slots hold NaN and garbage."""
    log(f"mask {kind} heads {nq}/{nkv} d {d}")
    B, n, cap = 4, 700, 705
    c, kh, vh, rng = filled(nq, nkv, d, B, n, seed=11, max_seq=cap)
    ctx = [699, 300, 31, 500]
    mask = np.zeros((B, cap), dtype=np.float32)
    if kind == "left":
        for b in range(B):
            mask[b, :ctx[b] * b // 4] = -np.inf
    elif kind == "random":
        mask[rng.random((B, cap)) < 0.5] = -np.inf
    elif kind == "bias":
        mask[:] = rng.standard_normal((B, cap)) * 3
        mask[:, ::7] = -np.inf
    elif kind == "most":                                     # one slot left, in the last tile; none in row 3
        mask[:] = -np.inf
        for b in range(3):
            mask[b, ctx[b] - 1] = 0.5
    else:                                                    # the lowest finite value: equal weights where nothing else is seen
        mask[:] = np.finfo(np.float32).min
        mask[0, 5], mask[1, 299] = 0.0, -2.0
    # garbage in hidden slots: NaN keys and values (also codes), beyond ctx as well
    hidden = [(b, j) for b in range(B) for j in range(0, cap, 3) if mask[b, j] == -np.inf or j > ctx[b]]
    for b, j in hidden[:60]:
        junk = torch.full((1, 1, nkv, d), float("nan"), dtype=torch.bfloat16, device="cuda")
        one = binding.kv4_desc(1, nkv, cap, d, c.desc.stride_b, c.desc.stride_h, c.desc.stride_b)
        binding.check(binding.kv4_append(one, c.k.data_ptr() + b * c.desc.stride_b, c.v.data_ptr() + b * c.desc.stride_b,
                                         junk, junk, 1, 1, [j]))
    q = bf16_values(rng, (B, nq, d))
    got = decode(c, q, ctx, mask=mask)
    check_decode(c, kh, vh, q, ctx, got, mask, kind)
    if kind == "most":
        assert not got[3].any()


@pytest.mark.parametrize("kscale,qscale", [(30.0, 1.0), (1e-3, 1.0), (1.0, 1e4), (1.0, 1e-6), (100.0, 1e30), (2000.0, 30.0)])
def test_decode_range_of_scores(kscale, qscale):
    """Scores from nearly equal to one that wins by far; queries far outside fp16's range."""
    log(f"scores k {kscale} q {qscale}")
    c, kh, vh, rng = filled(8, 2, 128, 2, 200, seed=13, kscale=kscale)
    q = round_bf16(bf16_values(rng, (2, 8, 128)) * qscale).astype(np.float32)
    ctx = [199, 77]
    got = decode(c, q, ctx)
    if qscale < 1e20:
        check_decode(c, kh, vh, q, ctx, got, None, "range")
    else:                                                    # one key wins (its lead passes 2^7 in every head)
        for b in range(2):
            for h in range(8):
                z = kh[b, h // 4, :ctx[b] + 1] @ q[b, h].astype(np.float64)
                assert np.array_equal(got[b, h], round_bf16(vh[b, h // 4, int(z.argmax())].astype(np.float32)))


@pytest.mark.parametrize("vscale", [1e-5, 0.01, 300.0, 15000.0])
def test_decode_range_of_values(vscale):
    """Values from fp16's smallest to its largest, a peaked and a flat softmax: the fp16 operands keep their precision."""
    rng = np.random.default_rng(14)
    for kscale in (0.1, 3.0):
        c = new_cache(config(8, 2, 128, 3000), 1)
        k = bf16_values(rng, (1, 3000, 2, 128), kscale)
        v = np.clip(bf16_values(rng, (1, 3000, 2, 128), vscale), -65280, 65280)
        v[0, 2500:] = np.clip(v[0, 2500:] * 4, -65280, 65280)          # the largest come last
        v = round_bf16(v).astype(np.float32)
        c.append(dev(k), dev(v), [0])
        kh, vh = (np.swapaxes(O.held(x), 1, 2) for x in (k, v))
        q = bf16_values(rng, (1, 8, 128))
        check_decode(c, kh, vh, q, [2999], decode(c, q, [2999]), None, f"values {vscale} keys {kscale}")


def test_nan_spreads_to_its_heads_only():
    """A NaN key that is seen makes its kv head's outputs NaN, a NaN query its own head's; no others."""
    c, kh, vh, rng = filled(8, 4, 64, 1, 50, seed=15)
    q = bf16_values(rng, (1, 8, 64))
    bad = bf16_values(rng, (1, 1, 4, 64))
    bad[0, 0, 1, 3] = np.nan
    c.append(dev(bad), dev(bf16_values(rng, (1, 1, 4, 64))), [20])
    q[0, 7, 5] = np.nan
    got = decode(c, q, [49])
    assert np.isnan(got[0, [2, 3, 7]]).all() and np.isfinite(got[0, [0, 1, 4, 5, 6]]).all()


def prefill(c, q, hist, row=0):
    out = torch.full(q.shape, float("nan"), dtype=torch.bfloat16, device="cuda")
    c.attn_prefill(dev(q), hist, out, row=row)
    torch.cuda.synchronize()
    return host(out)


@pytest.mark.parametrize("nq,nkv,d", HEADS)
@pytest.mark.parametrize("T,hist", [(1, 0), (2, 0), (31, 1), (32, 32), (33, 0), (64, 100), (5, 400), (130, 31)])
def test_prefill_attention(nq, nkv, d, T, hist):
    log(f"prefill heads {nq}/{nkv} d {d} T {T} hist {hist}")
    n = hist + T
    c, kh, vh, rng = filled(nq, nkv, d, 2, n, seed=T, max_seq=n + 3)
    q = bf16_values(rng, (T, nq, d))
    got = prefill(c, q, hist, row=1)
    for t in sorted({0, 1, T // 2, T - 2, T - 1} & set(range(T))):
        ref, tol = O.attend(q[t].astype(np.float64), kh[1], vh[1], np.arange(n) <= hist + t, key_eps=2.0 ** -11)
        check(got[t], ref, tol, f"query {t}")


@pytest.mark.parametrize("nq,nkv,d,T,hist", [(8, 2, 128, 700, 0), (7, 1, 128, 300, 3001), (14, 2, 64, 257, 2000),
                                             (4, 1, 128, 64, 4000), (8, 1, 128, 1, 5000)])
def test_prefill_attention_long(nq, nkv, d, T, hist):
    log(f"prefill heads {nq}/{nkv} d {d} T {T} hist {hist}")
    n = hist + T
    c, kh, vh, rng = filled(nq, nkv, d, 1, n, seed=T)
    q = bf16_values(rng, (T, nq, d))
    got = prefill(c, q, hist)
    assert np.isfinite(got).all()
    for t in sorted({0, T // 3, T // 2, max(T - 2, 0), T - 1}):
        ref, tol = O.attend(q[t].astype(np.float64), kh[0], vh[0], np.arange(n) <= hist + t, key_eps=2.0 ** -11)
        check(got[t], ref, tol, f"query {t}")


@pytest.mark.parametrize("qscale,vscale", [(1e-6, 1.0), (30.0, 1.0), (1e4, 300.0), (1.0, 15000.0), (1.0, 1e-4)])
def test_prefill_ranges(qscale, vscale):
    rng = np.random.default_rng(16)
    n, T = 333, 70
    c = new_cache(config(8, 2, 128, n), 1)
    k = bf16_values(rng, (1, n, 2, 128))
    v = round_bf16(np.clip(bf16_values(rng, (1, n, 2, 128), vscale), -65280, 65280)).astype(np.float32)
    c.append(dev(k), dev(v), [0])
    kh, vh = (np.swapaxes(O.held(x), 1, 2) for x in (k, v))
    q = round_bf16(bf16_values(rng, (T, 8, 128)) * qscale).astype(np.float32)
    got = prefill(c, q, n - T)
    for t in (0, 13, T - 1):
        ref, tol = O.attend(q[t].astype(np.float64), kh[0], vh[0], np.arange(n) <= n - T + t, key_eps=2.0 ** -11)
        check(got[t], ref, tol, f"query {t}")


def test_prefill_ignores_what_lies_behind():
    """Slots after the last query hold NaN."""
    c, kh, vh, rng = filled(8, 2, 128, 1, 100, seed=17, max_seq=160)
    junk = torch.full((1, 60, 2, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    c.append(junk, junk, [100])
    q = bf16_values(rng, (9, 8, 128))
    got = prefill(c, q, 91)
    for t in range(9):
        ref, tol = O.attend(q[t].astype(np.float64), kh[0], vh[0], np.arange(100) <= 91 + t, key_eps=2.0 ** -11)
        check(got[t], ref, tol, f"query {t}")


# --------------------------------------------------------- as they are used

def test_run_of_them_together():
    """A prompt, a second chunk, then single tokens: every call over what the ones before wrote; the steps agree with
    a prefill of the same tokens."""
    nq, nkv, d, T0, T1, steps = 8, 2, 128, 70, 45, 20
    n = T0 + T1 + steps
    rng = np.random.default_rng(18)
    c = new_cache(config(nq, nkv, d, n), 2)
    k, v, q = bf16_values(rng, (2, n, nkv, d)), bf16_values(rng, (2, n, nkv, d)), bf16_values(rng, (2, n, nq, d))
    kh, vh = (np.swapaxes(O.held(x), 1, 2) for x in (k, v))
    got = np.full((2, n, nq, d), np.nan)
    for b in range(2):
        one = binding.kv4_desc(1, nkv, n, d, c.desc.stride_b, c.desc.stride_h, c.desc.stride_b)
        for at, T in ((0, T0), (T0, T1)):
            binding.check(binding.kv4_append(one, c.k.data_ptr() + b * c.desc.stride_b, c.v.data_ptr() + b * c.desc.stride_b,
                                             dev(k[b, at:at + T]), dev(v[b, at:at + T]), 1, T, [at]))
            got[b, at:at + T] = prefill(c, q[b, at:at + T], at, row=b)
    for i in range(T0 + T1, n):
        ctx = torch.tensor([i, i], dtype=torch.int32, device="cuda")
        c.append_step(dev(k[:, i]), dev(v[:, i]), ctx)
        out = torch.empty((2, nq, d), dtype=torch.bfloat16, device="cuda")
        c.attn_decode(dev(q[:, i]), ctx, i, out)
        got[:, i] = host(out)
    for b in range(2):
        for t in (0, 31, T0 - 1, T0, T0 + T1 - 1, T0 + T1, n - 1):
            ref, tol = O.attend(q[b, t].astype(np.float64), kh[b], vh[b], np.arange(n) <= t, key_eps=2.0 ** -11)
            check(got[b, t], ref, tol, f"row {b} token {t}")
        late = prefill(c, q[b, T0 + T1:], T0 + T1, row=b)
        for t in range(steps):
            _, tol = O.attend(q[b, T0 + T1 + t].astype(np.float64), kh[b], vh[b], np.arange(n) <= T0 + T1 + t, key_eps=2.0 ** -11)
            a, z = got[b, T0 + T1 + t], late[t]
            assert (np.abs(a - z) <= 2 * tol * 1.01 + 2.0 ** -7 * np.abs(a)).all()


@pytest.mark.parametrize("ctx_cap", [127, 4095])
def test_captured_steps_replay(ctx_cap):
    """A captured step (append and attention) replayed with other keys, contexts and queries, eager work and other
    captures in between: every replay equals the eager result bit for bit."""
    nq, nkv, d, B = 8, 2, 128, 3
    cfg = config(nq, nkv, d, ctx_cap + 1)
    rng = np.random.default_rng(19)
    a, e = new_cache(cfg, B, 0), new_cache(cfg, B, 0)
    hist = [dev(bf16_values(rng, (B, ctx_cap - 20, nkv, d))) for _ in range(2)]
    for c in (a, e):
        c.append(*hist, [0] * B)
    k, v, q = (torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in ((B, nkv, d), (B, nkv, d), (B, nq, d)))
    ctx = torch.zeros(B, dtype=torch.int32, device="cuda")
    out, ref = torch.zeros_like(q), torch.zeros_like(q)

    def step(c, o):
        c.append_step(k, v, ctx)
        c.attn_decode(q, ctx, ctx_cap, o)

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step(a, out)
        step(e, ref)
    side.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(a, out)
        graphs.append(g)
    for i in range(6):
        for t, shape in ((k, (B, nkv, d)), (v, (B, nkv, d)), (q, (B, nq, d))):
            t.copy_(dev(bf16_values(rng, shape)))
        ctx.copy_(torch.tensor([ctx_cap - 15 + i, i * 7, 60 + i], dtype=torch.int32))
        graphs[i % 2].replay()
        step(e, ref)
        torch.cuda.synchronize()
        assert torch.equal(out, ref), i
        assert torch.equal(a.k, e.k) and torch.equal(a.v, e.v)


def test_prefill_captured():
    c, kh, vh, rng = filled(8, 2, 128, 1, 900, seed=20)
    q = dev(bf16_values(rng, (200, 8, 128)))
    out, ref = torch.zeros_like(q), torch.zeros_like(q)
    c.attn_prefill(q, 700, ref)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.attn_prefill(q, 700, out)
    for _ in range(4):
        q.copy_(dev(bf16_values(rng, (200, 8, 128))))
        g.replay()
        c.attn_prefill(q, 700, ref)
        torch.cuda.synchronize()
        assert torch.equal(out, ref)


def test_two_streams_at_once():
    """Two caches on two streams, calls interleaved, against the same calls one after the other."""
    rng = np.random.default_rng(21)
    ref, got = [], []
    sets = []
    for i in range(2):
        c, _, _, _ = filled(8, 2, 128, 2, 3000, seed=30 + i)
        sets.append((c, dev(bf16_values(rng, (2, 8, 128))), torch.tensor([2999, 1200], dtype=torch.int32, device="cuda"),
                     dev(bf16_values(rng, (100, 8, 128)))))
    for c, q, ctx, qp in sets:
        o, op = torch.empty_like(q), torch.empty_like(qp)
        c.attn_decode(q, ctx, 2999, o)
        c.attn_prefill(qp, 2900, op)
        torch.cuda.synchronize()
        ref.append((o, op))
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        outs = []
        for (c, q, ctx, qp), s in zip(sets, streams):
            o, op = torch.zeros_like(q), torch.zeros_like(qp)
            s.wait_stream(torch.cuda.current_stream())
            c.attn_decode(q, ctx, 2999, o, stream=s)
            c.attn_prefill(qp, 2900, op, stream=s)
            outs.append((o, op))
        torch.cuda.synchronize()
        got.append(outs)
    for outs in got:
        for (o, op), (r, rp) in zip(outs, ref):
            assert torch.equal(o, r) and torch.equal(op, rp)


def test_offsets_beyond_32_bits():
    """Strides of a cache of more than 4 GiB: the last sequence and head lie past 2^32 bytes."""
    nq, nkv, d, n = 8, 2, 128, 200
    rc, de = binding.kv4_layout(config(nq, nkv, d, n), 2)
    assert rc == 0
    de.stride_h = (5 << 29) + 16                              # 2.5 GiB between heads, 5 GiB between rows
    de.stride_b = 2 * de.stride_h
    size = 3 * de.stride_h + 7 * 32 * 80
    kc, vc = (torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(2))
    rng = np.random.default_rng(22)
    k, v, q = bf16_values(rng, (2, n, nkv, d)), bf16_values(rng, (2, n, nkv, d)), bf16_values(rng, (2, nq, d))
    binding.check(binding.kv4_append(de, kc, vc, dev(k), dev(v), 2, n, [0, 0]))
    ko, vo = (torch.zeros((2, n, nkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    binding.check(binding.kv4_read(de, kc, vc, 2, n, [0, 0], ko, vo))
    assert np.array_equal(host(ko), expected_read(k)) and np.array_equal(host(vo), expected_read(v))
    ws = torch.empty(max(binding.kv4_attn_workspace_size(de, nq, 2, 2, 1, n - 1),
                         binding.kv4_attn_workspace_size(de, nq, 1, 1, 2, n - 2)), dtype=torch.uint8, device="cuda")
    out = torch.empty((2, nq, d), dtype=torch.bfloat16, device="cuda")
    ctx = torch.tensor([n - 1, n - 1], dtype=torch.int32, device="cuda")
    binding.check(binding.kv4_attn_decode(de, dev(q), ctx, n - 1, None, 2, nq, kc, vc, out, ws, ws.numel()))
    kh, vh = (np.swapaxes(O.held(x), 1, 2) for x in (k, v))
    for b in range(2):
        ref, tol = O.attend(q[b].astype(np.float64), kh[b], vh[b], np.ones(n, bool))
        check(host(out)[b], ref, tol, f"row {b}")
    op = torch.empty((2, nq, d), dtype=torch.bfloat16, device="cuda")
    binding.check(binding.kv4_attn_prefill(de, dev(q), 2, n - 2, nq, kc.data_ptr() + de.stride_b, vc.data_ptr() + de.stride_b,
                                           op, ws, ws.numel()))
    for t in range(2):
        ref, tol = O.attend(q[t].astype(np.float64), kh[1], vh[1], np.arange(n) <= n - 2 + t, key_eps=2.0 ** -11)
        check(host(op)[t], ref, tol, f"query {t}")


def test_more_rows_than_one_launch_takes():
    """Batches above the 64 rows whose slots go with one launch."""
    B = 150
    rng = np.random.default_rng(23)
    c = new_cache(config(2, 2, 64, 40), B)
    slots = [int(rng.integers(0, 37)) for _ in range(B)]
    k, v = (bf16_values(rng, (B, 4, 2, 64)) for _ in range(2))
    c.append(dev(k), dev(v), slots)
    gk, gv = read(c, slots, 4)
    assert np.array_equal(gk, expected_read(k)) and np.array_equal(gv, expected_read(v))


def test_class_refuses_what_does_not_fit():
    c, _, _, rng = filled(8, 2, 128, 2, 50, seed=24)
    k = dev(bf16_values(rng, (2, 3, 2, 128)))
    q = dev(bf16_values(rng, (2, 8, 128)))
    ctx = torch.tensor([4, 5], dtype=torch.int32, device="cuda")
    for bad in (k.float(), k[:, :, :, :64], k.transpose(1, 2).contiguous().transpose(1, 2), k.cpu()):
        with pytest.raises(ValueError):
            c.append(k, bad, [0, 0])
    with pytest.raises(ValueError):
        c.append(k, k, [0])
    with pytest.raises(binding.W4Error):
        c.append(k, k, [0, 48])
    with pytest.raises(ValueError):
        c.append_step(k[:, 0].contiguous(), k[:, 0].contiguous(), ctx.long())
    with pytest.raises(ValueError):
        c.attn_decode(q[:, :4].contiguous(), ctx, 5, torch.empty_like(q))
    with pytest.raises(ValueError):
        c.attn_decode(q, ctx, 5, torch.empty_like(q), attn_mask=torch.zeros(2, 49, device="cuda"))
    with pytest.raises(binding.W4Error):
        c.attn_decode(q, ctx, 50, torch.empty_like(q))
    with pytest.raises(binding.W4Error):
        c.attn_decode(q, ctx, 5, q)
    with pytest.raises(ValueError):
        c.attn_prefill(q, 4, torch.empty_like(q), row=2)
    with pytest.raises(binding.W4Error):
        c.attn_prefill(q, 49, torch.empty_like(q))


def test_prefill_nan_values_reach_the_rows_that_see_them():
    """NaN values (and a NaN key) of some tokens: rows before them are untouched, rows from them on are NaN in the
    group (for a key: in all dims) of its kv head; with and without a history."""
    nq, nkv, d, n = 8, 2, 128, 210
    for T in (210, 90):
        rng = np.random.default_rng(25)
        k, v = bf16_values(rng, (1, n, nkv, d)), bf16_values(rng, (1, n, nkv, d))
        v[0, 150, 0, 40], v[0, 190, 1, 127], k[0, 200, 1, 3] = np.nan, np.inf, np.nan
        c = new_cache(config(nq, nkv, d, n), 1)
        c.append(dev(k), dev(v), [0])
        q = bf16_values(rng, (T, nq, d))
        got = prefill(c, q, n - T)
        want = np.zeros(got.shape, bool)
        t0 = n - T
        want[150 - t0:, :4, 32:64] = True
        want[190 - t0:, 4:, 96:128] = True
        want[200 - t0:, 4:, :] = True
        assert np.array_equal(np.isnan(got), want), T
        for x in (k, v):
            x[~np.isfinite(x)] = 0.0
        kh, vh = (np.swapaxes(O.held(x), 1, 2) for x in (k, v))
        for t in (149 - t0, 150 - t0, T - 1):
            ref, tol = O.attend(q[t].astype(np.float64), kh[0], vh[0], np.arange(n) <= t0 + t, key_eps=2.0 ** -11)
            ok = ~want[t]
            # (the other dims of a group with a NaN were quantised with it: not compared)
            if ok.any():
                check(np.where(ok, got[t], ref), ref, tol, f"query {t}")


# ------------------------------------------------- prefills of many queries
#
# A prefill of few queries or keys runs as rows of the decode kernel (T kv heads ceil(keys / 32) head_dim up to 2^21);
# these are beyond, in every way of dealing out the work: whole row tiles, parts of them, equal runs.

@pytest.mark.parametrize("nq,nkv,d,T,hist", [
    (64, 64, 64, 129, 0), (64, 64, 64, 33, 500), (64, 64, 64, 2, 8200), (32, 16, 128, 100, 333), (32, 16, 128, 257, 0),
    (32, 16, 128, 31, 1055), (56, 8, 128, 65, 1000), (56, 8, 128, 300, 0), (14, 2, 64, 511, 700), (24, 8, 64, 401, 31),
    (8, 1, 128, 1025, 0), (7, 1, 128, 900, 4000), (64, 8, 128, 1500, 1), (40, 8, 64, 2049, 63)])
def test_prefill_many_queries(nq, nkv, d, T, hist):
    log(f"prefill heads {nq}/{nkv} d {d} T {T} hist {hist}")
    n = hist + T
    assert T * nkv * -(-n // 32) * d > 2 ** 21
    c, kh, vh, rng = filled(nq, nkv, d, 1, n, seed=T, max_seq=n + 5)
    q = bf16_values(rng, (T, nq, d))
    got = prefill(c, q, hist)
    assert np.isfinite(got).all()
    for t in sorted({0, 1, T // 3, T // 2, T - 2, T - 1}):
        ref, tol = O.attend(q[t].astype(np.float64), kh[0], vh[0], np.arange(n) <= hist + t, key_eps=2.0 ** -11)
        check(got[t], ref, tol, f"query {t}")


def test_prefill_forms_agree_at_their_border():
    """The same queries as one call of the prefill kernel and as calls of a few each, which the decode kernel takes."""
    nq, nkv, d, T, hist = 32, 16, 128, 120, 300
    c, kh, vh, rng = filled(nq, nkv, d, 1, hist + T, seed=30)
    q = bf16_values(rng, (T, nq, d))
    whole = prefill(c, q, hist)
    for at, n in ((0, 1), (1, 8), (9, 40), (49, 71)):
        part = prefill(c, q[at:at + n], hist + at)
        for t in {0, n // 2, n - 1}:
            _, tol = O.attend(q[at + t].astype(np.float64), kh[0], vh[0], np.arange(hist + T) <= hist + at + t, key_eps=2.0 ** -11)
            a, z = part[t], whole[at + t]
            assert (np.abs(a - z) <= 2 * tol * 1.01 + 2.0 ** -7 * np.abs(a)).all()


@pytest.mark.parametrize("qscale,vscale", [(1e-6, 1.0), (30.0, 1.0), (1e4, 300.0), (1.0, 15000.0), (1.0, 1e-4)])
def test_prefill_many_ranges(qscale, vscale):
    rng = np.random.default_rng(31)
    n, T, nkv = 333, 120, 16
    c = new_cache(config(32, nkv, 128, n), 1)
    k = bf16_values(rng, (1, n, nkv, 128))
    v = round_bf16(np.clip(bf16_values(rng, (1, n, nkv, 128), vscale), -65280, 65280)).astype(np.float32)
    c.append(dev(k), dev(v), [0])
    kh, vh = (np.swapaxes(O.held(x), 1, 2) for x in (k, v))
    q = round_bf16(bf16_values(rng, (T, 32, 128)) * qscale).astype(np.float32)
    got = prefill(c, q, n - T)
    for t in (0, 13, T - 1):
        ref, tol = O.attend(q[t].astype(np.float64), kh[0], vh[0], np.arange(n) <= n - T + t, key_eps=2.0 ** -11)
        check(got[t], ref, tol, f"query {t}")


@pytest.mark.parametrize("T,n", [(210, 210), (90, 400)])
def test_prefill_many_nan_values_reach_the_rows_that_see_them(T, n):
    """As for few queries; slots after the last query hold NaN, too."""
    nq, nkv, d = 32, 16, 128
    t0 = n - T
    rng = np.random.default_rng(32)
    k, v = bf16_values(rng, (1, n, nkv, d)), bf16_values(rng, (1, n, nkv, d))
    at = [n - 60, n - 20, n - 10]
    v[0, at[0], 0, 40], v[0, at[1], 9, 127], k[0, at[2], 9, 3] = np.nan, np.inf, np.nan
    c = new_cache(config(nq, nkv, d, n + 70), 1)
    c.append(dev(k), dev(v), [0])
    junk = torch.full((1, 70, nkv, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    c.append(junk, junk, [n])
    q = bf16_values(rng, (T, nq, d))
    got = prefill(c, q, t0)
    want = np.zeros(got.shape, bool)
    want[at[0] - t0:, 0:2, 32:64] = True
    want[at[1] - t0:, 18:20, 96:128] = True
    want[at[2] - t0:, 18:20, :] = True
    assert np.array_equal(np.isnan(got), want)
    for x in (k, v):
        x[~np.isfinite(x)] = 0.0
    kh, vh = (np.swapaxes(O.held(x), 1, 2) for x in (k, v))
    for t in (0, at[0] - t0 - 1, at[0] - t0, T - 1):
        ref, tol = O.attend(q[t].astype(np.float64), kh[0], vh[0], np.arange(n) <= t0 + t, key_eps=2.0 ** -11)
        check(np.where(want[t], ref, got[t]), ref, tol, f"query {t}")


def test_prefill_many_captured_on_another_stream():
    nq, nkv, d, n, T = 32, 16, 128, 900, 200
    c, kh, vh, rng = filled(nq, nkv, d, 1, n, seed=33)
    q = dev(bf16_values(rng, (T, nq, d)))
    out, ref = torch.zeros_like(q), torch.zeros_like(q)
    c.attn_prefill(q, n - T, ref)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.attn_prefill(q, n - T, out)
    side = torch.cuda.Stream()
    for _ in range(4):
        q.copy_(dev(bf16_values(rng, (T, nq, d))))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            g.replay()
        side.synchronize()
        c.attn_prefill(q, n - T, ref)
        torch.cuda.synchronize()
        assert torch.equal(out, ref)


def test_class_refuses_integers_beyond_32_bits():
    c, _, _, rng = filled(8, 2, 128, 2, 50, seed=34)
    k = dev(bf16_values(rng, (2, 3, 2, 128)))
    q = dev(bf16_values(rng, (2, 8, 128)))
    ctx = torch.tensor([4, 5], dtype=torch.int32, device="cuda")
    for call in (lambda: c.append(k, k, [0, 2 ** 32]), lambda: c.read([2 ** 32, 0], 3, torch.empty_like(k), torch.empty_like(k)),
                 lambda: c.attn_decode(q, ctx, 2 ** 32 + 5, torch.empty_like(q)),
                 lambda: c.attn_prefill(q, 2 ** 32 + 4, torch.empty_like(q))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(AttributeError):
        c.k = c.v


def test_captured_on_forks():
    """Two calls on two streams of one capture, a third behind them, each with a workspace: replays equal the eager calls."""
    nq, nkv, d, n = 8, 2, 128, 3000
    c, _, _, rng = filled(nq, nkv, d, 2, n, seed=35)
    qs = [dev(bf16_values(rng, (2, nq, d))) for _ in range(3)]
    outs, refs = ([torch.zeros_like(qs[0]) for _ in range(3)] for _ in range(2))
    ctx = torch.tensor([n - 1, 1700], dtype=torch.int32, device="cuda")
    for q, ref in zip(qs, refs):
        c.attn_decode(q, ctx, n - 1, ref)
    side = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        main = torch.cuda.current_stream()
        side.wait_stream(main)
        c.attn_decode(qs[0], ctx, n - 1, outs[0], stream=side)
        c.attn_decode(qs[1], ctx, n - 1, outs[1])
        c.attn_decode(qs[2], ctx, n - 1, outs[2])
        main.wait_stream(side)
    for _ in range(4):
        for q in qs:
            q.copy_(dev(bf16_values(rng, (2, nq, d))))
        g.replay()
        for q, ref in zip(qs, refs):
            c.attn_decode(q, ctx, n - 1, ref)
        torch.cuda.synchronize()
        for out, ref in zip(outs, refs):
            assert torch.equal(out, ref)
