"""Attention with a window, sinks and draft trees over the bf16 cache on the GPU, against its fp64 oracle
(oracle/kv_attn.py): element by element within the bound that the oracle derives plus the rounding of the output
(2^-8 of the value, and of the value's own error), and over each case's whole error within three standard deviations of what
the roundings can make where they are independent.  Weights are rounded to bf16 (2^-8) at most."""
import pytest
import torch

from oracle import kv_attn as O
from paper_2607_15865_amd import binding, synth
from gpu_helpers import log

pytestmark = pytest.mark.gpu

HEADS = [(14, 2, 64), (1, 1, 128), (8, 8, 64), (32, 8, 128), (28, 4, 128), (7, 1, 128), (40, 2, 64), (64, 1, 128), (17, 1, 64), (12, 6, 128)]
WINDOWS = [(0, 0), (1, 0), (1, 1), (7, 3), (64, 4), (100, 70), (33, 0), (1000, 5)]
W_EPS = 2.0 ** -8


def config(nq, nkv, d, max_seq):
    return synth.replace(synth.CONFIGS["llama8b"], n_heads=nq, n_kv_heads=nkv, head_dim=d, max_seq=max_seq)


def randn(g, *shape, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(torch.bfloat16)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def filled(g, nq, nkv, d, max_seq, batch, strides=False):
    """A KVCache with values in every slot; with strides, a token-major view inside larger buffers."""
    cfg = config(nq, nkv, d, max_seq)
    if strides:
        big = [randn(g, batch, max_seq, nkv + 1, d + 8) for _ in range(2)]
        k, v = (x[:, :, :nkv, :d].transpose(1, 2) for x in big)
    else:
        k, v = (randn(g, batch, nkv, max_seq, d) for _ in range(2))
    k += (torch.randn((nkv, 1, d), generator=g, device="cuda") * (torch.rand((nkv, 1, d), generator=g, device="cuda") < 0.06) * 3).to(k.dtype)
    return binding.KVCache(cfg, batch, k, v)


def check(got, q, k, v, seen, add=None, what=""):
    """got, q [m][nq][d] against the oracle over keys, values [nkv][n][d]; seen [m][n]."""
    m, nq, d = q.shape
    r = nq // k.shape[0]
    err2 = var = 0.0
    for h in range(nq):
        out, tol, spread = O.attend(q[:, h].double(), k[h // r].double(), v[h // r].double(), seen, add, W_EPS)
        err = (got[:, h].double() - out).abs()
        bound = tol + (out.abs() + tol) * 2.0 ** -8 + 2.0 ** -133
        assert torch.isfinite(got[:, h]).all(), f"{what}: head {h} is not finite"
        worst = (err / bound).max().item()
        assert worst <= 1, f"{what}: head {h}, error {worst} of its bound"
        empty = ~(seen & (True if add is None else (add != -float('inf'))[None])).any(1)
        assert torch.all(got[empty, h] == 0), f"{what}: an empty row of head {h} is not 0"
        err2 += (err ** 2).sum().item()
        var += (spread ** 2 + (out * 2.0 ** -8) ** 2 / 3).sum().item()
    if q.numel() >= 2048:                    # (the mean square of thousands of errors)
        assert err2 <= 9 * var + 1e-12, f"{what}: errors of {err2 ** 0.5}, {var ** 0.5} expected at most"


def run_decode(c, q, ctx, window, sinks, mask=None, max_ctx=None, stream=None):
    out = torch.full_like(q, 7.0)
    dev = torch.tensor(ctx, dtype=torch.int32, device="cuda")
    c.attn_decode(q, dev, max(ctx) if max_ctx is None else max_ctx, out, window=window, sinks=sinks, attn_mask=mask, stream=stream)
    torch.cuda.synchronize()
    return out


def check_decode(c, q, out, ctx, window, sinks, mask=None):
    for b, n in enumerate(ctx):
        if n < 0:
            assert torch.all(out[b] == 0)
            continue
        seen = O.seen_from(torch.tensor([n], device="cuda"), torch.arange(n + 1, device="cuda"), window, sinks)
        check(out[b:b + 1], q[b:b + 1], c.k[b, :, :n + 1], c.v[b, :, :n + 1], seen, None if mask is None else mask[b, :n + 1].double(),
              f"decode row {b} ctx {n} window {window} sinks {sinks}")


# ------------------------------------------------------------- single queries

@pytest.mark.parametrize("window,sinks", WINDOWS)
@pytest.mark.parametrize("nq,nkv,d", HEADS)
def test_decode(nq, nkv, d, window, sinks):
    log(f"decode heads {nq} {nkv} {d} window {window} sinks {sinks}")
    g = gen(nq * d + window)
    ctx = [0, 1, 31, 32, 63, 64, -1, 300, 517]
    c = filled(g, nq, nkv, d, 600, len(ctx))
    q = randn(g, len(ctx), nq, d)
    check_decode(c, q, run_decode(c, q, ctx, window, sinks), ctx, window, sinks)


@pytest.mark.parametrize("ctx", [[5000], [40000], [9000, 5, 8191, -1, 8192, 700, 4095], [2000] * 33])
@pytest.mark.parametrize("window,sinks", [(0, 0), (4096, 4), (1500, 0)])
@pytest.mark.parametrize("nq,nkv,d", [(14, 2, 64), (32, 8, 128), (28, 4, 128)])
def test_decode_long(nq, nkv, d, window, sinks, ctx):
    log(f"decode heads {nq} {nkv} {d} window {window} sinks {sinks} ctx {ctx[:3]}")
    g = gen(max(ctx) + d)
    c = filled(g, nq, nkv, d, max(ctx) + 3, len(ctx))
    q = randn(g, len(ctx), nq, d)
    check_decode(c, q, run_decode(c, q, ctx, window, sinks, max_ctx=max(ctx) + 2), ctx, window, sinks)


@pytest.mark.parametrize("scale", [1e-3, 8.0, 60.0])
def test_decode_flat_and_sharp_scores(scale):
    g = gen(3)
    c = filled(g, 8, 2, 128, 900, 2)
    q = randn(g, 2, 8, 128, scale=scale)
    check_decode(c, q, run_decode(c, q, [880, 450], 512, 4), [880, 450], 512, 4)


@pytest.mark.parametrize("window,sinks", [(0, 0), (200, 4), (200, 300)])
@pytest.mark.parametrize("nq,nkv,d", [(14, 2, 64), (32, 8, 128), (40, 2, 128), (64, 1, 128), (45, 1, 64)])
def test_decode_mask(nq, nkv, d, window, sinks):
    """Additive masks: padded on the left, scattered, nothing left, finite values; what is hidden holds NaN."""
    log(f"mask heads {nq} {nkv} {d} window {window} sinks {sinks}")
    g = gen(17 + d + window)
    ctx = [400, 777, 777, 90, 777]
    c = filled(g, nq, nkv, d, 1000, 5)
    mask = torch.zeros((5, 1000), device="cuda")
    mask[0, :150] = -float("inf")
    mask[1, torch.rand(1000, generator=g, device="cuda") < 0.5] = -float("inf")
    mask[2] = -float("inf")
    mask[3] = torch.randn(1000, generator=g, device="cuda") * 3
    mask[4, 700:] = -float("inf")
    q = randn(g, 5, nq, d)
    want = run_decode(c, q, ctx, window, sinks, mask)
    check_decode(c, q, want, ctx, window, sinks, mask)
    hidden = (mask == -float("inf"))[:, None, :, None]
    for t, bad in ((c.k, float("nan")), (c.v, float("nan")), (c.v, float("inf"))):
        t.masked_fill_(hidden, bad)
        assert torch.equal(run_decode(c, q, ctx, window, sinks, mask), want)


def test_decode_mask_of_the_lowest_value():
    """The lowest float added to every score leaves them equal (the scores vanish in it): the mean of the values; added to
    some, it hides them as -inf does."""
    g = gen(5)
    c = filled(g, 8, 2, 64, 300, 2)
    q = randn(g, 2, 8, 64)
    low = torch.finfo(torch.float32).min
    mask = torch.zeros((2, 300), device="cuda")
    mask[0] = low
    mask[1, :100] = low
    out = run_decode(c, q, [200, 200], 0, 0, mask)
    mean = c.v[0, :, :201].double().mean(1).repeat_interleave(4, 0)
    assert torch.allclose(out[0].double(), mean, rtol=2.0 ** -7, atol=2.0 ** -8 * 2 / 201 ** 0.5)
    mask[1, :100] = -float("inf")
    assert torch.equal(run_decode(c, q, [200, 200], 0, 0, mask)[1], out[1])


@pytest.mark.parametrize("nq,nkv,d", [(14, 2, 64), (32, 8, 128), (64, 1, 128)])
def test_decode_unseen_slots_may_hold_anything(nq, nkv, d):
    """NaN and infinities behind the context, before the window, and in other sequences."""
    g = gen(23 + d)
    ctx, window, sinks = [310, 100, 449], 100, 3
    c = filled(g, nq, nkv, d, 450, 3)
    q = randn(g, 3, nq, d)
    want = run_decode(c, q, ctx, window, sinks)
    check_decode(c, q, want, ctx, window, sinks)
    for bad in (float("nan"), float("inf")):
        for b, n in enumerate(ctx):
            unseen = ~O.seen_from(torch.tensor([n], device="cuda"), torch.arange(450, device="cuda"), window, sinks)[0]
            for t in (c.k, c.v):
                t[b, :, unseen] = bad
        assert torch.equal(run_decode(c, q, ctx, window, sinks), want)


def test_decode_visible_nan_and_infinity_come_through():
    g = gen(2)
    c = filled(g, 4, 2, 64, 100, 1)
    q = randn(g, 1, 4, 64)
    c.v[0, 0, 50, 7] = float("nan")
    c.v[0, 1, 60, 9] = float("inf")
    out = run_decode(c, q, [80], 0, 0)
    assert torch.isnan(out[0, :2, 7]).all() and not torch.isfinite(out[0, 2:, 9]).any()


def test_strided_caches():
    g = gen(31)
    c = filled(g, 14, 2, 64, 333, 3, strides=True)
    assert not c.k.is_contiguous() and c.desc.stride_s == 3 * 72
    q, ctx = randn(g, 3, 14, 64), [332, 17, 200]
    check_decode(c, q, run_decode(c, q, ctx, 90, 4), ctx, 90, 4)
    q = randn(g, 150, 14, 64)
    check_prefill(c, q, run_prefill(c, q, 100, 64, 4, row=1), 100, 64, 4, row=1)


def test_append_of_more_sequences_than_a_launch_takes():
    g = gen(19)
    c = filled(g, 4, 2, 64, 40, 150)
    want = [c.k.clone(), c.v.clone()]
    new, slots = [randn(g, 130, 3, 2, 64) for _ in range(2)], [(7 * b) % 38 for b in range(130)]
    c.append(*new, slots)
    torch.cuda.synchronize()
    for t, w, x in zip((c.k, c.v), want, new):
        for b, s in enumerate(slots):
            w[b, :, s:s + 3] = x[b].transpose(0, 1)
        assert torch.equal(t, w)
    with pytest.raises(binding.W4Error):
        c.append(*new, slots[:-1] + [38])
    with pytest.raises(ValueError):
        c.append(*new, slots[:-1])
    torch.cuda.synchronize()
    assert torch.equal(c.k, want[0]) and torch.equal(c.v, want[1])


def test_offsets_beyond_32_bits():
    """A window at the end of a cache of 2^24 slots and more: element and byte offsets beyond 2^31 and 2^32."""
    n = (1 << 24) + 4000
    g = gen(41)
    cfg = config(8, 1, 128, n)
    k, v = (torch.empty((1, 1, n, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for t in (k, v):
        t[:, :, :64] = randn(g, 1, 1, 64, 128)
        t[:, :, -6000:] = randn(g, 1, 1, 6000, 128)
    c = binding.KVCache(cfg, 1, k, v)
    ctx, window, sinks = n - 301, 700, 5
    slots = torch.cat([torch.arange(sinks), torch.arange(ctx - 2000, n)]).cuda()
    kk, vv = k[0][:, slots], v[0][:, slots]

    def expect(out, q, pos, extra=None):
        seen = O.seen_from(pos, slots, window, sinks)
        check(out, q, kk, vv, seen if extra is None else seen & extra, None, "far slots")

    q = randn(g, 1, 8, 128)
    expect(run_decode(c, q, [ctx], window, sinks), q, torch.tensor([ctx], device="cuda"))
    q = randn(g, 300, 8, 128)
    expect(run_prefill(c, q, ctx, window, sinks), q, torch.arange(ctx, ctx + 300, device="cuda"))
    tree = binding.DraftTree(1, 70)
    q = randn(g, 1, 70, 8, 128)
    parents = torch.arange(-1, 69, dtype=torch.int32, device="cuda")[None].contiguous()
    out = run_tree(c, tree, q, parents, [ctx], window, sinks)
    expect(out[0], q[0], torch.arange(ctx, ctx + 70, device="cuda"))


# ------------------------------------------------------------- queries of one sequence

def run_prefill(c, q, hist, window, sinks, row=0, stream=None):
    out = torch.full_like(q, 7.0)
    c.attn_prefill(q, hist, out, window=window, sinks=sinks, row=row, stream=stream)
    torch.cuda.synchronize()
    return out


def check_prefill(c, q, out, hist, window, sinks, row=0):
    T = q.shape[0]
    seen = O.seen_from(torch.arange(hist, hist + T, device="cuda"), torch.arange(hist + T, device="cuda"), window, sinks)
    check(out, q, c.k[row, :, :hist + T], c.v[row, :, :hist + T], seen, None, f"prefill T {T} hist {hist} window {window} sinks {sinks}")


@pytest.mark.parametrize("window,sinks", WINDOWS)
@pytest.mark.parametrize("T,hist", [(1, 0), (2, 0), (5, 77), (33, 0), (64, 64), (65, 190), (130, 3), (257, 500)])
@pytest.mark.parametrize("nq,nkv,d", [(14, 2, 64), (32, 8, 128), (7, 1, 128), (1, 1, 64)])
def test_prefill(nq, nkv, d, T, hist, window, sinks):
    log(f"prefill heads {nq} {nkv} {d} T {T} hist {hist} window {window} sinks {sinks}")
    g = gen(T * 31 + hist + d)
    c = filled(g, nq, nkv, d, hist + T + 5, 2)
    q = randn(g, T, nq, d)
    check_prefill(c, q, run_prefill(c, q, hist, window, sinks, row=1), hist, window, sinks, row=1)


@pytest.mark.parametrize("window,sinks", [(0, 0), (1024, 4), (4096, 0), (130, 500)])
@pytest.mark.parametrize("nq,nkv,d,T,hist", [(14, 2, 64, 1500, 700), (32, 8, 128, 600, 5000), (28, 4, 128, 2011, 1001), (6, 1, 64, 40, 9000),
                                             (28, 4, 128, 20, 7000), (40, 2, 128, 333, 1200), (4, 4, 128, 3000, 0), (14, 2, 64, 6000, 100),
                                             (14, 2, 64, 500, 500)])
def test_prefill_long(nq, nkv, d, T, hist, window, sinks):
    log(f"prefill heads {nq} {nkv} {d} T {T} hist {hist} window {window} sinks {sinks}")
    g = gen(T + hist + d + window)
    c = filled(g, nq, nkv, d, hist + T, 1)
    q = randn(g, T, nq, d)
    check_prefill(c, q, run_prefill(c, q, hist, window, sinks), hist, window, sinks)


@pytest.mark.parametrize("scale", [1e-3, 8.0, 60.0])
def test_prefill_flat_and_sharp_scores(scale):
    g = gen(4)
    c = filled(g, 8, 2, 128, 900, 1)
    q = randn(g, 500, 8, 128, scale=scale)
    check_prefill(c, q, run_prefill(c, q, 400, 256, 4), 400, 256, 4)


@pytest.mark.parametrize("nq,nkv,d,T,hist,window,sinks", [(14, 2, 64, 300, 100, 0, 0), (32, 8, 128, 200, 300, 70, 3), (28, 4, 128, 12, 500, 200, 0),
                                                          (28, 4, 128, 700, 0, 130, 4), (28, 4, 128, 2011, 101, 300, 4), (14, 2, 64, 1500, 300, 0, 0),
                                                          (14, 2, 64, 1500, 300, 130, 500), (14, 2, 64, 500, 500, 0, 0)])
def test_prefill_unseen_slots_may_hold_anything(nq, nkv, d, T, hist, window, sinks):
    """A NaN or infinity in a key or value reaches the rows that see its slot and no others, which keep their bits."""
    log(f"prefill NaN heads {nq} {nkv} {d} T {T} hist {hist} window {window}")
    g = gen(T + hist)
    n = hist + T
    c = filled(g, nq, nkv, d, n + 40, 1)
    q = randn(g, T, nq, d)
    want = run_prefill(c, q, hist, window, sinks)
    check_prefill(c, q, want, hist, window, sinks)
    pos = torch.arange(hist, n, device="cuda")
    for slots in ([n - 1], [hist + T // 2, hist + T // 2 + 1], [hist // 2, n, n + 39], [0]):
        for which, bad in (("k", float("nan")), ("v", float("nan")), ("v", float("inf")), ("v", -float("inf"))):
            t = getattr(c, which)
            keep = t.clone()
            t[0, :, slots, 3] = bad
            out = run_prefill(c, q, hist, window, sinks)
            t.copy_(keep)
            sees = O.seen_from(pos, torch.tensor(slots, device="cuda"), window, sinks).any(1)
            assert torch.equal(out[~sees], want[~sees]), (slots, which, bad)
            if which == "v":
                assert not torch.isfinite(out[sees][..., 3]).any(), (slots, bad)
            else:
                assert torch.isnan(out[sees]).all(), slots


# ------------------------------------------------------------- drafted tokens

def random_tree(g, B, N, kind):
    if kind == "chain":
        p = torch.arange(-1, N - 1)
        return p.to(torch.int32).repeat(B, 1).cuda()
    if kind == "star":
        p = torch.zeros(N)
        p[0] = -1
        return p.to(torch.int32).repeat(B, 1).cuda()
    p = (torch.rand((B, N), generator=g, device="cuda") * torch.arange(N, device="cuda")).floor()
    p[:, 0] = -1
    if kind == "forest":                     # some roots more, and parents that are none
        p[:, N // 3] = -5
        p[:, N // 2] = N + 3
        p[:, 0] = 2 ** 31 - 1
    return p.to(torch.int32)


def run_tree(c, tree, q, parents, ctx, window, sinks, max_ctx=None, stream=None):
    out = torch.full_like(q, 7.0)
    dev = torch.tensor(ctx, dtype=torch.int32, device="cuda")
    tree.plan(parents, dev, window=window, sinks=sinks, stream=stream)
    c.attn_tree(q, tree, dev, max(ctx) if max_ctx is None else max_ctx, out, stream=stream)
    torch.cuda.synchronize()
    return out


def tree_seen(parents, n, window, sinks):
    """Which slots the nodes of one sequence see, [N][n + N]."""
    N = len(parents)
    pos, sets = O.plan(parents, n, window, sinks)
    seen = torch.zeros((N, n + N), dtype=torch.bool)
    seen[:, :n] = O.seen_from(torch.tensor(pos), torch.arange(n), window, sinks)
    for i, s in enumerate(sets):
        for a in s:
            seen[i, n + a] = True
    return seen.cuda()


def check_tree(c, q, out, parents, ctx, window, sinks):
    for b, n in enumerate(ctx):
        if n < 0:
            assert torch.all(out[b] == 0)
            continue
        end = n + q.shape[1]
        check(out[b], q[b], c.k[b, :, :end], c.v[b, :, :end], tree_seen(parents[b].tolist(), n, window, sinks), None,
              f"tree row {b} ctx {n} window {window} sinks {sinks}")


@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (3, 2), (20, 0), (64, 70), (300, 4)])
@pytest.mark.parametrize("N,kind", [(1, "random"), (2, "chain"), (7, "random"), (16, "star"), (33, "forest"), (64, "random"), (65, "chain"),
                                    (129, "forest"), (256, "random"), (256, "chain")])
@pytest.mark.parametrize("nq,nkv,d", [(14, 2, 64), (32, 8, 128), (7, 1, 128)])
def test_tree(nq, nkv, d, N, kind, window, sinks):
    log(f"tree heads {nq} {nkv} {d} N {N} {kind} window {window} sinks {sinks}")
    g = gen(N * 3 + window + d)
    ctx = [0, 1, 200, -1, 341]
    c = filled(g, nq, nkv, d, 341 + N, len(ctx))
    q = randn(g, len(ctx), N, nq, d)
    parents = random_tree(g, len(ctx), N, kind)
    tree = binding.DraftTree(len(ctx), N)
    check_tree(c, q, run_tree(c, tree, q, parents, ctx, window, sinks), parents, ctx, window, sinks)


@pytest.mark.parametrize("nq,nkv,d,B,N,ctx", [(14, 2, 64, 1, 9, 9000), (32, 8, 128, 2, 64, 7000), (28, 4, 128, 3, 100, 5003), (32, 8, 128, 17, 5, 1500),
                                              (40, 2, 128, 1, 200, 3001), (28, 4, 128, 1, 2, 30000)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (2048, 4)])
def test_tree_long(nq, nkv, d, B, N, ctx, window, sinks):
    log(f"tree heads {nq} {nkv} {d} B {B} N {N} ctx {ctx} window {window}")
    g = gen(N + ctx + window)
    lens = [ctx - b * ctx // (2 * B) for b in range(B)]
    c = filled(g, nq, nkv, d, ctx + N + 9, B)
    q = randn(g, B, N, nq, d)
    parents = random_tree(g, B, N, "random")
    check_tree(c, q, run_tree(c, binding.DraftTree(B, N), q, parents, lens, window, sinks, max_ctx=ctx + 9), parents, lens, window, sinks)


@pytest.mark.parametrize("nq,nkv,d,N", [(14, 2, 64, 8), (32, 8, 128, 40), (28, 4, 128, 100), (32, 8, 128, 2), (32, 8, 128, 256), (28, 4, 128, 256)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (90, 3)])
def test_tree_unseen_slots_may_hold_anything(nq, nkv, d, N, window, sinks):
    """A value that is not finite in a node's or a context's slot reaches the nodes that see it and no others."""
    log(f"tree NaN heads {nq} {nkv} {d} N {N} window {window}")
    g = gen(N + window)
    n = 250
    c = filled(g, nq, nkv, d, n + N + 30, 1)
    q, parents, tree = randn(g, 1, N, nq, d), random_tree(g, 1, N, "random"), binding.DraftTree(1, N)
    want = run_tree(c, tree, q, parents, [n], window, sinks)
    check_tree(c, q, want, parents, [n], window, sinks)
    seen = tree_seen(parents[0].tolist(), n, window, sinks)
    for slots in ([n + N - 1], [n + N // 2], [n], [n + N, n + N + 29], [3], [n - 89, n - 90, n - 91]):
        for which, bad in (("k", float("nan")), ("v", float("nan")), ("v", float("inf"))):
            t = getattr(c, which)
            keep = t.clone()
            t[0, :, slots, 5] = bad
            out = run_tree(c, tree, q, parents, [n], window, sinks)
            t.copy_(keep)
            inside = [s for s in slots if s < n + N]
            sees = seen[:, inside].any(1) if inside else torch.zeros(N, dtype=torch.bool, device="cuda")
            assert torch.equal(out[0][~sees], want[0][~sees]), (slots, which)
            if which == "v":
                assert not torch.isfinite(out[0][sees][..., 5]).any(), slots


def test_tree_with_masks_of_the_callers_own():
    """Masks that no tree makes: a node that sees only others, one that sees nothing of the drafts; without a context it is
    empty.  Bits beyond N are not nodes."""
    g = gen(77)
    cfg_n, N = 120, 70
    c = filled(g, 14, 2, 64, cfg_n + N, 2)
    q = randn(g, 2, N, 14, 64)
    bits = torch.rand((2, N, 128), generator=g, device="cuda") < 0.3
    bits[:, 5] = False
    bits[:, 6, :N] = False
    bits[:, 6, 3] = True
    words = (bits.long().view(2, N, 2, 64) << torch.arange(64, device="cuda")).sum(-1).contiguous()
    ctx = [cfg_n, 0]
    dev = torch.tensor(ctx, dtype=torch.int32, device="cuda")
    out, ws = torch.full_like(q, 7.0), torch.empty(1 << 26, dtype=torch.uint8, device="cuda")
    binding.check(binding.kv_attn_tree(c.desc, q, dev, cfg_n, words, None, 0, 0, 2, N, 14, c.k, c.v, out, ws, ws.numel()))
    torch.cuda.synchronize()
    for b, n in enumerate(ctx):
        seen = torch.ones((N, n + N), dtype=torch.bool, device="cuda")
        seen[:, n:] = bits[b, :, :N]
        check(out[b], q[b], c.k[b, :, :n + N], c.v[b, :, :n + N], seen, None, "own masks")
    assert torch.all(out[1, 5] == 0)


@pytest.mark.parametrize("N", [3, 70])
def test_tree_positions_that_no_tree_has(N):
    """A position outside ctx .. ctx + N - 1 counts as the nearest of these."""
    g = gen(78 + N)
    n, window, sinks = 300, 90, 3
    c = filled(g, 14, 2, 64, n + N, 1)
    q = randn(g, 1, N, 14, 64)
    far = torch.randint(n - 2 * N, n + 3 * N, (1, N), generator=g, device="cuda").int()
    far[0, 0], far[0, 1], far[0, 2] = 2 ** 31 - 1, -2 ** 31, n + N
    words = torch.zeros((1, N, (N + 63) // 64), dtype=torch.int64, device="cuda")        # (no node sees another, or itself)
    dev = torch.tensor([n], dtype=torch.int32, device="cuda")
    out, ws = torch.full_like(q, 7.0), torch.empty(1 << 26, dtype=torch.uint8, device="cuda")
    binding.check(binding.kv_attn_tree(c.desc, q, dev, n, words, far, window, sinks, 1, N, 14, c.k, c.v, out, ws, ws.numel()))
    torch.cuda.synchronize()
    seen = O.seen_from(far[0].clamp(n, n + N - 1), torch.arange(n, device="cuda"), window, sinks)
    check(out[0], q[0], c.k[0, :, :n], c.v[0, :, :n], seen, None, f"positions of {N} nodes")


def test_a_chain_is_a_prefill_and_single_steps():
    """The same tokens as a chain of drafts, as a prefill behind the same context and one by one: the same values up to the
    roundings (all three within the oracle's bound)."""
    g = gen(9)
    n, N, window, sinks = 500, 24, 300, 4
    c = filled(g, 28, 4, 128, n + N, 1)
    q = randn(g, 1, N, 28, 128)
    tree = binding.DraftTree(1, N)
    parents = random_tree(g, 1, N, "chain")
    check_tree(c, q, run_tree(c, tree, q, parents, [n], window, sinks), parents, [n], window, sinks)
    check_prefill(c, q[0], run_prefill(c, q[0], n, window, sinks), n, window, sinks)
    for t in range(N):
        check_decode(c, q[:, t], run_decode(c, q[:, t].contiguous(), [n + t], window, sinks), [n + t], window, sinks)


# ------------------------------------------------------------- the calls

def test_refused_tensors():
    g = gen(1)
    c = filled(g, 14, 2, 64, 100, 2)
    q, out, ctx = randn(g, 2, 14, 64), torch.empty((2, 14, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    tree = binding.DraftTree(2, 3)
    qt = randn(g, 2, 3, 14, 64)
    for bad in (dict(q=q.float()), dict(q=q[:, :7]), dict(q=q.transpose(0, 1)), dict(out=out[:1]), dict(ctx=ctx.long()), dict(ctx=ctx[:1]),
                dict(q=q.cpu()), dict(mask=torch.zeros((2, 99), device="cuda")), dict(mask=torch.zeros((2, 100), device="cuda").half()),
                dict(window=2 ** 31), dict(sinks=2 ** 32), dict(max_ctx=2 ** 32 + 5)):
        a = dict(dict(q=q, out=out, ctx=ctx, mask=None, window=0, sinks=0, max_ctx=5), **bad)
        with pytest.raises(ValueError):
            c.attn_decode(a["q"], a["ctx"], a["max_ctx"], a["out"], window=a["window"], sinks=a["sinks"], attn_mask=a["mask"])
    with pytest.raises(binding.W4Error):
        c.attn_decode(q, ctx, 100, out)
    with pytest.raises(binding.W4Error):
        c.attn_decode(q, ctx, 5, q)
    with pytest.raises(ValueError):
        c.attn_tree(qt, tree, ctx, 5, torch.empty_like(qt))        # (no plan yet)
    with pytest.raises(ValueError):
        tree.plan(torch.zeros((2, 4), dtype=torch.int32, device="cuda"), ctx)
    tree.plan(torch.zeros((2, 3), dtype=torch.int32, device="cuda"), ctx)
    with pytest.raises(ValueError):
        c.attn_tree(qt[:, :2], tree, ctx, 5, torch.empty_like(qt))
    with pytest.raises(ValueError):
        c.attn_prefill(q, 0, out, row=2)
    with pytest.raises(ValueError):
        tree.keep([], ctx)
    with pytest.raises(ValueError):
        tree.keep([c, filled(g, 14, 2, 64, 101, 2)], ctx)
    with pytest.raises(binding.W4Error):
        tree.keep([c, c], ctx)
    for n in (0, 257):
        with pytest.raises(ValueError):
            binding.DraftTree(1, n)
    cfg = config(14, 2, 64, 100)
    for k in (torch.empty((2, 2, 100, 64), device="cuda"), torch.empty((2, 2, 99, 64), device="cuda", dtype=torch.bfloat16),
              torch.empty((2, 2, 100, 64), dtype=torch.bfloat16), torch.empty((2, 2, 64, 100), device="cuda", dtype=torch.bfloat16).transpose(2, 3)):
        with pytest.raises(ValueError):
            binding.KVCache(cfg, 2, k, k.clone())
    with pytest.raises(ValueError):
        binding.KVCache(cfg, 2, c.k)


def test_outputs_and_workspaces_keep_to_their_sizes():
    """Nothing is written before or behind an output, and nothing behind the workspace that a call asked for."""
    g = gen(8)
    c = filled(g, 28, 4, 128, 5000, 3)
    parents, tree = random_tree(g, 3, 37, "random"), binding.DraftTree(3, 37)
    ctx = torch.tensor([4900, 20, 2000], dtype=torch.int32, device="cuda")
    tree.plan(parents, ctx, window=2000, sinks=4)
    for stage, rows, T, hist in ((2, (3,), 1, 4900), (1, (300,), 300, 4000), (1, (3,), 3, 4000), (3, (3, 37), 37, 4900)):
        q = randn(g, *rows, 28, 128)
        big = torch.full((q.numel() + 512,), 7.0, dtype=torch.bfloat16, device="cuda")
        n = binding.kv_attn_workspace_size(c.desc, 28, stage, 3, T, hist)
        ws = torch.full((n + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
        out = big[256:256 + q.numel()]
        if stage == 2:
            rc = binding.kv_attn_decode(c.desc, q, ctx, hist, 2000, 4, None, 3, 28, c.k, c.v, out, ws, n)
        elif stage == 1:
            rc = binding.kv_attn_prefill(c.desc, q, T, hist, 2000, 4, 28, c.k, c.v, out, ws, n)
        else:
            rc = binding.kv_attn_tree(c.desc, q, ctx, hist, tree.mask, tree.pos, 2000, 4, 3, T, 28, c.k, c.v, out, ws, n)
        binding.check(rc)
        torch.cuda.synchronize()
        assert torch.all(big[:256] == 7) and torch.all(big[256 + q.numel():] == 7) and torch.all(ws[n:] == 0xA5), stage


def test_results_do_not_change_from_call_to_call():
    g = gen(6)
    c = filled(g, 32, 8, 128, 6000, 4)
    q, ctx = randn(g, 4, 32, 128), [5900, 3000, 10, 4444]
    first = run_decode(c, q, ctx, 0, 0)
    qp = randn(g, 700, 32, 128)
    prefill = run_prefill(c, qp, 5000, 3000, 4)
    parents, tree, qt = random_tree(g, 4, 60, "random"), binding.DraftTree(4, 60), randn(g, 4, 60, 32, 128)
    drafted = run_tree(c, tree, qt, parents, ctx, 0, 0)
    for _ in range(5):
        assert torch.equal(run_decode(c, q, ctx, 0, 0), first)
        assert torch.equal(run_prefill(c, qp, 5000, 3000, 4), prefill)
        assert torch.equal(run_tree(c, tree, qt, parents, ctx, 0, 0), drafted)


def test_streams_with_calls_in_flight():
    """Two streams at once, each with its own workspace, and a stream that is not the current one."""
    g = gen(12)
    c = filled(g, 28, 4, 128, 9000, 4)
    q, ctx = randn(g, 4, 28, 128), torch.tensor([8900, 7000, 8000, 1], dtype=torch.int32, device="cuda")
    qp = randn(g, 400, 28, 128)
    want = run_decode(c, q, ctx.tolist(), 0, 0)
    wantp = run_prefill(c, qp, 8000, 0, 0)
    s = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(3):
        outs = [torch.empty_like(q) for _ in range(4)]
        outp = [torch.empty_like(qp) for _ in range(4)]
        torch.cuda.synchronize()
        for i in range(4):
            c.attn_decode(q, ctx, 8900, outs[i], stream=s[i % 2])
            c.attn_prefill(qp, 8000, outp[i], stream=s[i % 2].cuda_stream)
        torch.cuda.synchronize()
        assert all(torch.equal(o, want) for o in outs) and all(torch.equal(o, wantp) for o in outp)


def test_captured_and_replayed():
    """Decode, prefill and a whole draft step in one graph, replayed with other inputs and eager calls in between."""
    g = gen(14)
    c, N = filled(g, 28, 4, 128, 4000, 2), 20
    q, qp, qt = randn(g, 2, 28, 128), randn(g, 300, 28, 128), randn(g, 2, N, 28, 128)
    ctx = torch.tensor([3500, 2000], dtype=torch.int32, device="cuda")
    parents, tree = random_tree(g, 2, N, "random"), binding.DraftTree(2, N)
    outs = [torch.empty_like(t) for t in (q, qp, qt)]
    eager = [torch.empty_like(t) for t in (q, qp, qt)]
    mine = binding.DraftTree(2, N)

    def calls(tree, outs):
        tree.plan(parents, ctx, window=1000, sinks=4)
        c.attn_decode(q, ctx, 3500, outs[0], window=1000, sinks=4)
        c.attn_prefill(qp, 3000, outs[1], window=1000, sinks=4)
        c.attn_tree(qt, tree, ctx, 3500, outs[2])

    calls(mine, eager)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(tree, outs)
    for step in range(4):
        for t in (q, qp, qt):
            t.copy_(randn(g, *t.shape))
        ctx.copy_(torch.tensor([3500 - 700 * step, 100 + 900 * step], dtype=torch.int32))
        parents.copy_(random_tree(g, 2, N, "random"))
        for t in outs:
            t.fill_(7.0)
        graph.replay()
        calls(mine, eager)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, eager)) and torch.equal(tree.mask, mine.mask) and torch.equal(tree.pos, mine.pos)
