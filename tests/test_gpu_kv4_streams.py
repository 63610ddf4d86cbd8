"""KV4Cache's calls on streams other than torch's current one, eagerly and as branches of a captured graph: results equal
those of the same calls one after the other, bit for bit."""
import numpy as np
import pytest
import torch

from paper_2607_15865_amd import binding, synth
from gpu_helpers import log

pytestmark = pytest.mark.gpu

NQ, NKV, D, N = 8, 2, 128, 3000


def filled(seed, batch=2):
    cfg = synth.replace(synth.CONFIGS["llama8b"], n_heads=NQ, n_kv_heads=NKV, head_dim=D, max_seq=N)
    g = torch.Generator(device="cuda").manual_seed(seed)
    c = binding.KV4Cache(cfg, batch)
    c.append(*(rand(g, (batch, N, NKV, D)) for _ in range(2)), [0] * batch)
    return c, g


def rand(g, shape):
    return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)


def i32(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("order", [(None, "side", None, "side"), ("side", None, "side", None), (None, None, "side", "side")])
def test_branches_of_a_captured_graph(order):
    """Calls of two branches, either first, decode and prefill: every replay equals the eager calls."""
    log(f"branches {order}")
    c, g = filled(1)
    ctx = i32(N - 1, 1700)
    shapes = [(2, NQ, D), (200, NQ, D)]
    qs = [rand(g, shapes[i % 2]) for i in range(4)]
    outs, refs = ([torch.zeros_like(q) for q in qs] for _ in range(2))

    def call(i, out, stream=None):
        if i % 2 == 0:
            c.attn_decode(qs[i], ctx, N - 1, out, stream=stream)
        else:
            c.attn_prefill(qs[i], N - 200, out, row=1, stream=stream)

    for i in range(4):
        call(i, refs[i])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        main = torch.cuda.current_stream()
        side.wait_stream(main)
        for i, where in enumerate(order):
            call(i, outs[i], side if where else None)
        main.wait_stream(side)
    for r in range(5):
        for q in qs:
            q.copy_(rand(g, q.shape))
        graph.replay()
        for i in range(4):
            call(i, refs[i])
        torch.cuda.synchronize()
        for i in range(4):
            assert torch.equal(outs[i], refs[i]), (r, i)


@pytest.mark.parametrize("form", ["stream", "handle"])
def test_first_call_beside_work_on_a_freed_block(form):
    """The current stream still works on a block that the program has let go of; a first call on another stream, which
    nothing orders behind that work, disturbs neither."""
    log(f"freed block, {form}")
    g = torch.Generator(device="cuda").manual_seed(2)
    a = torch.randn((4096, 4096), generator=g, device="cuda")
    for i in range(4):
        c, gc = filled(10 + i)
        q, ctx = rand(gc, (2, NQ, D)), i32(N - 1, 900)
        ref, out = torch.zeros_like(q), torch.zeros_like(q)
        c.attn_decode(q, ctx, N - 1, ref)
        other = binding.KV4Cache(synth.replace(synth.CONFIGS["llama8b"], n_heads=NQ, n_kv_heads=NKV, head_dim=D, max_seq=N), 2)
        other.k.copy_(c.k), other.v.copy_(c.v)
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        x = torch.zeros_like(a)
        for _ in range(20):
            torch.mul(a, 2.0, out=x)
            torch.add(x, 1.0, out=x)
        want = x[::64].clone()
        del x                                                # (its last readers and writers are queued, not done)
        other.attn_decode(q, ctx, N - 1, out, stream=side if form == "stream" else side.cuda_stream)
        torch.cuda.synchronize()
        assert torch.equal(out, ref)
        assert torch.equal(want, (a * 2.0 + 1.0)[::64])


def test_default_stream_named_from_another():
    """stream=0, the default stream, while another one is current."""
    c, g = filled(3)
    q, qp, ctx = rand(g, (2, NQ, D)), rand(g, (200, NQ, D)), i32(N - 1, 40)
    ref, out, refp, outp = (torch.zeros_like(x) for x in (q, q, qp, qp))
    c.attn_decode(q, ctx, N - 1, ref)
    c.attn_prefill(qp, N - 200, refp)
    torch.cuda.synchronize()
    c2, _ = filled(3)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        c2.attn_decode(q, ctx, N - 1, out, stream=0)
        c2.attn_prefill(qp, N - 200, outp, stream=0)
        c2.attn_prefill(qp, N - 200, outp, stream=torch.cuda.default_stream())
    torch.cuda.synchronize()
    assert torch.equal(out, ref) and torch.equal(outp, refp)


def test_one_cache_on_several_streams_at_once():
    """Calls on one cache from three streams, none ordered behind another, with growing workspaces."""
    c, g = filled(4)
    ctx = i32(N - 1, 2000)
    work = [(rand(g, (2, NQ, D)), rand(g, (n, NQ, D))) for n in (40, 300, 900)]
    refs = [(torch.zeros_like(q), torch.zeros_like(p)) for q, p in work]
    for (q, p), (o, op) in zip(work, refs):
        c.attn_decode(q, ctx, N - 1, o)
        c.attn_prefill(p, N - p.shape[0], op)
    streams = [torch.cuda.Stream() for _ in work]
    torch.cuda.synchronize()
    for _ in range(4):
        outs = [(torch.zeros_like(q), torch.zeros_like(p)) for q, p in work]
        torch.cuda.synchronize()
        for (q, p), (o, op), s in zip(work, outs, streams):
            c.attn_decode(q, ctx, N - 1, o, stream=s)
            c.attn_prefill(p, N - p.shape[0], op, stream=s)
        torch.cuda.synchronize()
        for got, ref in zip(outs, refs):
            assert all(torch.equal(a, b) for a, b in zip(got, ref))
    assert np.isfinite(refs[0][0].float().cpu().numpy()).all()


def test_captured_stream_that_is_not_current():
    """A call on the captured stream while another one is current: the graph has a workspace of its own, replayed while
    eager calls on the same stream use theirs."""
    c, g = filled(5)
    ctx, side = i32(N - 1, 1500), torch.cuda.Stream()
    qs = [rand(g, (2, NQ, D)) for _ in range(2)]
    outs, refs = ([torch.zeros_like(q) for q in qs] for _ in range(2))
    torch.cuda.synchronize()
    c.attn_decode(qs[0], ctx, N - 1, refs[0], stream=side)
    torch.cuda.synchronize()
    graph, idle = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        with torch.cuda.stream(idle):
            c.attn_decode(qs[0], ctx, N - 1, outs[0], stream=side)
    for r in range(5):
        for q in qs:
            q.copy_(rand(g, q.shape))
        torch.cuda.synchronize()
        graph.replay()                                       # (on the default stream, beside the eager call on side)
        c.attn_decode(qs[1], ctx, N - 1, outs[1], stream=side)
        torch.cuda.synchronize()
        for q, ref in zip(qs, refs):
            c.attn_decode(q, ctx, N - 1, ref)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, refs)), r


def test_eager_call_beside_a_capture():
    """While one stream is captured, a call on another one that is no part of the capture runs at once."""
    c, g = filled(6)
    q, ctx, idle = rand(g, (2, NQ, D)), i32(N - 1, 333), torch.cuda.Stream()
    out, now, ref = (torch.zeros_like(q) for _ in range(3))
    c.attn_decode(q, ctx, N - 1, ref)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.attn_decode(q, ctx, N - 1, out)
        c.attn_decode(q, ctx, N - 1, now, stream=idle)
    idle.synchronize()
    assert torch.equal(now, ref)
    now.zero_()
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, ref) and not now.any()


def test_cache_made_in_a_capture():
    """A cache made, filled and read in a captured graph: its memory is the graph's, every replay gives the same."""
    _, g = filled(7)
    cfg = synth.replace(synth.CONFIGS["llama8b"], n_heads=NQ, n_kv_heads=NKV, head_dim=D, max_seq=400)
    k, v, q = rand(g, (1, 400, NKV, D)), rand(g, (1, 400, NKV, D)), rand(g, (300, NQ, D))
    out, ref = torch.zeros_like(q), torch.zeros_like(q)
    back = [torch.zeros_like(k) for _ in range(4)]
    e = binding.KV4Cache(cfg, 1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c = binding.KV4Cache(cfg, 1)
        c.append(k, v, [0])
        c.attn_prefill(q, 100, out)
    for _ in range(4):
        for t in (k, v, q):
            t.copy_(rand(g, t.shape))
        graph.replay()
        e.append(k, v, [0])
        e.attn_prefill(q, 100, ref)
        c.read([0], 400, *back[:2])                          # (400 slots end inside a tile, whose rest is anything)
        e.read([0], 400, *back[2:])
        torch.cuda.synchronize()
        assert torch.equal(out, ref) and torch.equal(back[0], back[2]) and torch.equal(back[1], back[3])
