"""The 4-bit cache's calls on the host, no GPU needed: layout arithmetic and every refusal, which come before any
launch (dummy pointers: nothing may be read or written)."""
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
CFG = synth.replace(synth.CONFIGS["llama8b"], max_seq=1000)


def desc(rows=3, cfg=CFG, **kw):
    rc, d = B.kv4_layout(cfg, rows)
    assert rc == 0
    for k, v in kw.items():
        setattr(d, k, v)
    return d


def test_layout():
    d = desc()
    assert (d.batch, d.n_kv_heads, d.max_seq, d.head_dim) == (3, 8, 1000, 128)
    assert d.stride_h == 32 * 32 * 80 and d.stride_b == 8 * d.stride_h and d.bytes == 3 * d.stride_b
    rc, d = B.kv4_layout(synth.replace(synth.CONFIGS["tiny"], max_seq=32), 1)
    assert rc == 0 and d.stride_h == 32 * 40
    assert B.kv4_layout(CFG, 0)[0] == B.W4_EINVAL
    assert B.kv4_layout(synth.replace(CFG, head_dim=96), 1)[0] == B.W4_EUNSUPPORTED
    assert B.kv4_layout(synth.replace(CFG, n_kv_heads=0), 1)[0] == B.W4_EINVAL


@pytest.mark.parametrize("call", ["append", "read"])
def test_store_refusals(call):
    def go(d=None, k=P, v=P, x=P, y=P, b=2, t=4, slots=(0, 0)):
        d = d or desc()
        if call == "append":
            return B.kv4_append(d, k, v, x, y, b, t, list(slots), stream=0)
        return B.kv4_read(d, k, v, b, t, list(slots), x, y, stream=0)

    for name in ("k", "v", "x", "y"):
        assert go(**{name: 0}) == B.W4_EINVAL
        assert go(**{name: P + 8}) == B.W4_EINVAL, name
    assert go(b=0) == B.W4_EINVAL and go(t=0) == B.W4_EINVAL
    assert go(b=4, slots=(0,) * 4) == B.W4_ECAPACITY
    assert go(slots=(0, 997)) == B.W4_ECAPACITY and "997..1000" in B.layer_last_error()
    assert go(slots=(-1, 0)) == B.W4_ECAPACITY
    assert go(t=2 ** 31 - 1, slots=(1, 1)) == B.W4_ECAPACITY
    assert go(desc(head_dim=96)) == B.W4_EUNSUPPORTED
    for kw in (dict(stride_h=32 * 32 * 80 - 16), dict(stride_h=32 * 32 * 80 + 8), dict(stride_b=16), dict(batch=0),
               dict(max_seq=0), dict(n_kv_heads=0)):
        assert go(desc(**kw)) == B.W4_EINVAL, kw


def test_append_step_refusals():
    def go(d=None, k=P, v=P, x=P, y=P, b=2, c=P):
        return B.kv4_append_step(d or desc(), k, v, x, y, b, c, stream=0)

    for name in ("k", "v", "x", "y", "c"):
        assert go(**{name: 0}) == B.W4_EINVAL
    assert go(x=P + 2) == B.W4_EINVAL
    assert go(b=0) == B.W4_EINVAL and go(b=4) == B.W4_ECAPACITY
    assert go(desc(head_dim=32)) == B.W4_EUNSUPPORTED


def test_decode_refusals():
    def go(d=None, q=P, c=P, ctx=10, mask=None, b=2, nq=32, k=P, v=P, out=2 * P, ws=P, n=1 << 40):
        return B.kv4_attn_decode(d or desc(), q, c, ctx, mask, b, nq, k, v, out, ws, n, stream=0)

    for name in ("q", "c", "k", "v", "out", "ws"):
        assert go(**{name: 0}) == B.W4_EINVAL
    for name in ("q", "k", "v", "out", "ws"):
        assert go(**{name: 3 * P + 8}) == B.W4_EINVAL, name
    assert go(out=P) == B.W4_EINVAL and "alias" in B.layer_last_error()
    assert go(b=0) == B.W4_EINVAL and go(b=4) == B.W4_ECAPACITY
    assert go(ctx=-1) == B.W4_EINVAL and go(ctx=1000) == B.W4_ECAPACITY
    assert go(nq=0) == B.W4_EINVAL and go(nq=12) == B.W4_EUNSUPPORTED and go(nq=72) == B.W4_EUNSUPPORTED
    assert go(n=B.kv4_attn_workspace_size(desc(), 32, 2, 2, 1, 10) - 1) == B.W4_EWORKSPACE


def test_prefill_refusals():
    def go(d=None, q=P, t=5, hist=10, nq=32, k=P, v=P, out=2 * P, ws=P, n=1 << 40):
        return B.kv4_attn_prefill(d or desc(), q, t, hist, nq, k, v, out, ws, n, stream=0)

    for name in ("q", "k", "v", "out", "ws"):
        assert go(**{name: 0}) == B.W4_EINVAL
        assert go(**{name: 3 * P + 8}) == B.W4_EINVAL, name
    assert go(out=P) == B.W4_EINVAL
    assert go(t=0) == B.W4_EINVAL and go(hist=-1) == B.W4_EINVAL
    assert go(t=991) == B.W4_ECAPACITY and go(t=2 ** 31 - 1, hist=2 ** 31 - 1) == B.W4_ECAPACITY
    assert go(nq=20) == B.W4_EUNSUPPORTED and go(nq=0) == B.W4_EINVAL
    assert go(n=B.kv4_attn_workspace_size(desc(), 32, 1, 1, 5, 10) - 1) == B.W4_EWORKSPACE


def test_workspace_size():
    ws = lambda stage, b, t, ctx, nq=32: B.kv4_attn_workspace_size(desc(), nq, stage, b, t, ctx)   # noqa: E731
    assert ws(3, 1, 1, 1) == 0 and ws(2, 0, 1, 1) == 0 and ws(2, 4, 1, 1) == 0 and ws(1, 1, 0, 1) == 0
    assert ws(2, 1, 1, -1) == 0 and ws(2, 1, 1, 1, nq=12) == 0
    assert B._lib.kv4_attn_workspace_size(None, 32, 2, 1, 1, 1) == 0
    big = desc(rows=64, cfg=synth.replace(CFG, max_seq=200000))
    for d, nq in ((desc(rows=64), 32), (big, 64), (big, 8)):
        for stage in (0, 1, 2):
            last = 0
            for b in (1, 2, 3, 7, 16, 40, 64):
                now = B.kv4_attn_workspace_size(d, nq, stage, b, 1 if stage == 2 else 37 * b, 900)
                assert now >= max(last, 1), (stage, b)
                last = now
            last = 0
            for ctx in (0, 1, 31, 32, 255, 256, 900, 999):
                now = B.kv4_attn_workspace_size(d, nq, stage, 3, 1 if stage == 2 else 70, ctx)
                assert now >= max(last, 1), (stage, ctx)
                last = now


def test_struct_matches_the_header():
    assert ctypes.sizeof(B.kv4_desc) == 4 * 4 + 2 * 8 + 8


def test_set_kv_format_refusals():
    assert B.layer_set_kv_format(None, B.W4_KV_INT4) == B.W4_EINVAL


def test_longest_cache():
    """2^27 slots at most: rows of queries are counted in 31 bits."""
    for n, rc in ((2 ** 27, B.W4_ECAPACITY), (2 ** 27 + 1, B.W4_EUNSUPPORTED)):
        d = desc(max_seq=n, stride_h=(n + 31) // 32 * 32 * 80, stride_b=(n + 31) // 32 * 32 * 80 * 8)
        assert B.kv4_append(d, P, P, P, P, 1, 2, [n - 1], stream=0) == rc
        assert B.kv4_attn_prefill(d, P, 5, n, 32, P, P, 2 * P, P, 1 << 40, stream=0) == rc
        assert (B.kv4_attn_workspace_size(d, 32, 1, 1, 2 ** 31 - 1, 2 ** 31 - 1) > 0) == (rc == B.W4_ECAPACITY)
    cfg = synth.replace(CFG, max_seq=2 ** 27)
    assert B.kv4_layout(cfg, 1)[0] == 0
    assert B.kv4_layout(synth.replace(cfg, max_seq=2 ** 27 + 1), 1)[0] == B.W4_EUNSUPPORTED


def test_keys_and_values_apart():
    """Caches that are written, and outputs, may not be one; sources may."""
    d = desc()
    assert B.kv4_append(d, P, P, P, 2 * P, 1, 2, [0], stream=0) == B.W4_EINVAL and "alias" in B.layer_last_error()
    assert B.kv4_append_step(d, P, P, P, 2 * P, 1, P, stream=0) == B.W4_EINVAL and "alias" in B.layer_last_error()
    assert B.kv4_read(d, P, 2 * P, 1, 2, [0], P, P, stream=0) == B.W4_EINVAL and "alias" in B.layer_last_error()


def test_strides_that_overflow():
    assert B.kv4_append(desc(stride_h=2 ** 62, stride_b=2 ** 62), P, P, P, P, 1, 2, [0], stream=0) == B.W4_EINVAL
    assert "strides" in B.layer_last_error()
