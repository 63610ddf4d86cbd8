"""The calls of attention with a window and of draft trees on the host, no GPU needed: every refusal, which comes before any
launch (dummy pointers: nothing may be read or written), and the workspace sizes."""
import ctypes
import os

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2607_15865_amd", "libw4layer.so")

if not os.path.exists(LIB):
    from paper_2607_15865_amd import build as _b
    _b.build()

from paper_2607_15865_amd import binding as B  # noqa: E402
from paper_2607_15865_amd import synth  # noqa: E402

P = 4096                      # an aligned dummy pointer
BIG = 2 ** 31 - 1
CFG = synth.replace(synth.CONFIGS["llama8b"], max_seq=1000)


def desc(rows=3, cfg=CFG, **kw):
    rc, d = B.kv_layout(cfg, rows)
    assert rc == 0
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def decode(d=None, q=P, c=P, ctx=10, window=5, sinks=2, mask=None, b=2, nq=32, k=P, v=P, out=2 * P, ws=P, n=1 << 40):
    return B.kv_attn_decode(d or desc(), q, c, ctx, window, sinks, mask, b, nq, k, v, out, ws, n, stream=0)


def prefill(d=None, q=P, t=7, ctx=10, window=5, sinks=2, nq=32, k=P, v=P, out=2 * P, ws=P, n=1 << 40):
    return B.kv_attn_prefill(d or desc(), q, t, ctx, window, sinks, nq, k, v, out, ws, n, stream=0)


def tree(d=None, q=P, c=P, ctx=10, mask=P, pos=P, window=5, sinks=2, b=2, t=7, nq=32, k=P, v=P, out=2 * P, ws=P, n=1 << 40):
    return B.kv_attn_tree(d or desc(), q, c, ctx, mask, pos, window, sinks, b, t, nq, k, v, out, ws, n, stream=0)


def append(d=None, k=P, v=2 * P, x=P, y=P, b=2, t=4, c=P):
    return B.kv_append_step(d or desc(), k, v, x, y, b, t, c, stream=0)


def keep(d=None, ks=(P, 2 * P), vs=(3 * P, 4 * P), count=None, c=P, path=P, n=P, b=2, t=4):
    return B.kv_tree_keep(d or desc(), list(ks), list(vs), len(ks) if count is None else count, c, path, n, b, t, stream=0)


BAD_DESC = [dict(batch=0), dict(n_kv_heads=0), dict(max_seq=0), dict(stride_s=120), dict(stride_s=132), dict(stride_h=64),
            dict(stride_h=128004), dict(stride_b=8 * 128000 + 4), dict(stride_s=136), dict(stride_b=0), dict(bytes=0),
            dict(bytes=3 * 8 * 128000 * 2 - 2), dict(bytes=2 ** 63), dict(batch=4), dict(stride_b=2 ** 62)]


@pytest.mark.parametrize("call", [decode, prefill, tree, append, keep])
def test_descriptors(call):
    for kw in BAD_DESC:
        assert call(desc(**kw)) == B.W4_EINVAL, kw
    assert call(desc(head_dim=96)) == B.W4_EUNSUPPORTED
    assert call(desc(max_seq=2 ** 27 + 1)) == B.W4_EUNSUPPORTED


@pytest.mark.parametrize("call,names", [(decode, ("q", "c", "k", "v", "out", "ws")), (prefill, ("q", "k", "v", "out", "ws")),
                                        (tree, ("q", "c", "mask", "k", "v", "out", "ws")), (append, ("k", "v", "x", "y", "c")),
                                        (keep, ("c", "path", "n"))])
def test_null_and_unaligned_pointers(call, names):
    for name in names:
        assert call(**{name: 0}) == B.W4_EINVAL, name
    for name in set(names) & {"q", "k", "v", "out", "ws", "x", "y"}:
        assert call(**{name: P + 8}) == B.W4_EINVAL, name


@pytest.mark.parametrize("call", [decode, prefill, tree])
def test_attention_refusals(call):
    assert call(window=-1) == B.W4_EINVAL and call(sinks=-1) == B.W4_EINVAL and call(ctx=-1) == B.W4_EINVAL
    assert call(nq=0) == B.W4_EINVAL and call(nq=12) == B.W4_EUNSUPPORTED and call(nq=8 * 65) == B.W4_EUNSUPPORTED
    assert call(out=P) == B.W4_EINVAL and "alias" in B.layer_last_error()
    assert call(n=0) == B.W4_EWORKSPACE
    new = 1 if call is decode else 7
    assert call(ctx=1001 - new) == B.W4_ECAPACITY and call(ctx=BIG) == B.W4_ECAPACITY
    if call is not prefill:
        assert call(b=0) == B.W4_EINVAL and call(b=4) == B.W4_ECAPACITY
    if call is not decode:
        assert call(t=0) == B.W4_EINVAL and call(t=-1) == B.W4_EINVAL
        assert call(t=BIG) in (B.W4_ECAPACITY, B.W4_EUNSUPPORTED)
    if call is prefill:                      # (more queries times heads than a launch takes)
        big = synth.replace(CFG, max_seq=1 << 27)
        assert call(desc(1, big), t=1 << 21, n=0) == B.W4_EWORKSPACE and call(desc(1, big), t=(1 << 21) + 1) == B.W4_ECAPACITY
    if call is tree:
        big = synth.replace(CFG, max_seq=1000)
        assert call(desc(40000, big), b=32768, t=256, nq=128, n=0) == B.W4_EWORKSPACE
        assert call(desc(40000, big), b=32769, t=256, nq=128) == B.W4_ECAPACITY
        assert call(mask=P + 4) == B.W4_EINVAL
        assert call(t=257) == B.W4_EUNSUPPORTED
        assert call(pos=0) == B.W4_EINVAL and "positions" in B.layer_last_error()


@pytest.mark.parametrize("call", [decode, tree])
def test_more_pairs_than_a_launch_takes(call):
    """2^21 sequences times kv heads."""
    d = desc(1 << 16, synth.replace(CFG, n_kv_heads=64, n_heads=64, max_seq=300))
    assert call(d, b=1 << 15, nq=64, n=0) == B.W4_EWORKSPACE
    assert call(d, b=(1 << 15) + 1, nq=64) == B.W4_ECAPACITY and "kv heads" in B.layer_last_error()


@pytest.mark.parametrize("stage", [0, 1, 2, 3])
def test_workspace_sizes(stage):
    d = desc(rows=64)

    def size(b=2, t=9, ctx=500, nq=32, d=d):
        return B.kv_attn_workspace_size(d, nq, stage, b, t, ctx)

    assert size() > 0 and size(ctx=0) > 0
    assert size(ctx=-1) == 0 and size(nq=33) == 0 and size(d=desc(head_dim=32)) == 0
    if stage >= 2:
        assert size(b=0) == 0 and size(b=65) == 0
    if stage != 2:
        assert size(t=0) == 0
    if stage == 3:
        assert size(t=257) == 0
    before = 0
    for ctx in (0, 1, 63, 64, 65, 100, 700, 990, 100000, BIG):       # (beyond the cache: the size of the most that fits)
        assert size(ctx=ctx) >= before
        before = size(ctx=ctx)
    for grow in ("b", "t"):
        before = 0
        for x in (1, 2, 3, 4, 7, 8, 16, 17, 31, 64):
            assert size(**{grow: x}) >= before, (grow, x)
            before = size(**{grow: x})
    assert B.kv_attn_workspace_size(d, 32, 4, 1, 1, 1) == 0 and B.kv_attn_workspace_size(d, 32, -1, 1, 1, 1) == 0


def test_append_step_refusals():
    assert append(b=0) == B.W4_EINVAL and append(t=0) == B.W4_EINVAL and append(b=4) == B.W4_ECAPACITY
    assert append(v=P) == B.W4_EINVAL and "alias" in B.layer_last_error()


def test_keep_refusals():
    assert keep(b=0) == B.W4_EINVAL and keep(b=4) == B.W4_ECAPACITY
    assert keep(t=0) == B.W4_EINVAL and keep(t=257) == B.W4_EUNSUPPORTED
    assert keep(count=0) == B.W4_EINVAL and keep(count=1025) == B.W4_ECAPACITY
    assert keep(ks=(P, P)) == B.W4_EINVAL and keep(vs=(3 * P, P)) == B.W4_EINVAL and "twice" in B.layer_last_error()
    assert keep(ks=(P, 0)) == B.W4_EINVAL and keep(vs=(3 * P, 4 * P + 8)) == B.W4_EINVAL


def test_tree_refusals():
    def plan(par=P, c=P, b=2, n=5, window=0, sinks=0, mask=P, pos=P):
        return B.tree_plan(par, c, b, n, window, sinks, mask, pos, stream=0)

    def accept(par=P, tok=P, pick=P, b=2, n=5, path=P, count=P, nxt=P):
        return B.tree_accept(par, tok, pick, b, n, path, count, nxt, stream=0)

    for name in ("par", "c", "mask", "pos"):
        assert plan(**{name: 0}) == B.W4_EINVAL
    for name in ("par", "tok", "pick", "path", "count", "nxt"):
        assert accept(**{name: 0}) == B.W4_EINVAL
    for call in (plan, accept):
        assert call(b=0) == B.W4_EINVAL and call(n=0) == B.W4_EINVAL and call(n=257) == B.W4_EUNSUPPORTED
        assert call(b=65536) == B.W4_ECAPACITY
    assert plan(mask=P + 4) == B.W4_EINVAL
    assert plan(window=-1) == B.W4_EINVAL and plan(sinks=-1) == B.W4_EINVAL


def test_descriptor_of_token_major_caches_is_taken():
    """[batch][max_seq][n_kv_heads][head_dim]: the calls get past the checks of the descriptor (and stop at the workspace)."""
    d = desc(stride_b=1000 * 8 * 128, stride_s=8 * 128, stride_h=128)
    assert decode(d, n=0) == B.W4_EWORKSPACE
    assert ctypes.sizeof(B.kv_desc) == 48
