"""Layers, stacks and the model step with an attention window, and layers on drafted tokens.  A windowed call has to
give what the same layer without a window gives where an additive mask hides the same slots, or where the same tokens are
taken one by one (both are compared with the oracle elsewhere); drafted tokens what each path gives on its own."""
import numpy as np
import pytest
import torch

from oracle import kv_attn as O
from paper_2607_15865_amd import binding, synth
from gpu_helpers import assert_parity, bits_to_torch_f32, host_layer, log

pytestmark = pytest.mark.gpu


def layer(name, max_seq=None):
    cfg, w = host_layer(name)
    if max_seq:
        cfg = synth.replace(cfg, max_seq=max_seq)
    return cfg, binding.Layer(cfg, w)


def inputs(cfg, n, seed=0):
    return bits_to_torch_f32(synth.activations(cfg, synth.TID_X_PREFILL + 1000 * seed, n))


def pos(a, b):
    return torch.arange(a, b, dtype=torch.int32, device="cuda")


def filled(cfg, lay, batch, seed=1):
    """A cache with values in every slot."""
    k, v = lay.new_cache(batch)
    g = torch.Generator(device="cuda").manual_seed(seed)
    for t in (k, v):
        t.copy_((torch.randn(t.shape, generator=g, device="cuda")).to(torch.bfloat16).view(torch.int16))
    return k, v


def hidden_mask(cfg, ctx, window, sinks):
    m = torch.full((len(ctx), cfg.max_seq), -float("inf"), device="cuda")
    for b, n in enumerate(ctx):
        m[b, :n + 1][O.seen_from(torch.tensor([n]), torch.arange(n + 1), window, sinks)[0].cuda()] = 0
    return m


def decode(lay, cfg, x, ctx, k, v, mask=None):
    y = torch.empty_like(x)
    c = torch.tensor(ctx, dtype=torch.int32, device="cuda")
    lay.decode(x, c, c, max(ctx), k, v, y, attn_mask=mask)
    torch.cuda.synchronize()
    return y.cpu().numpy()


@pytest.mark.parametrize("name,ctx,window,sinks", [("tiny", [40], 7, 2), ("tiny", [100, 3, 64, 0, 99], 33, 4), ("qwen05b", [700], 256, 4),
                                                   ("qwen05b", [900, 100], 64, 0), ("llama8b", [3000], 1000, 4),
                                                   ("llama8b", [2000, 5, 1500, 700, 2047, 99, 300, 1999], 512, 3)])
def test_windowed_decode_is_a_masked_one(name, ctx, window, sinks):
    log(f"windowed decode {name} {ctx} {window} {sinks}")
    cfg, lay = layer(name)
    x = inputs(cfg, len(ctx))
    k, v = filled(cfg, lay, len(ctx))
    k2, v2 = k.clone(), v.clone()
    lay.set_decode_path(1)
    want = decode(lay, cfg, x, ctx, k, v, hidden_mask(cfg, ctx, window, sinks))
    lay.set_decode_path(0)
    lay.set_window(window, sinks)
    assert_parity(decode(lay, cfg, x, ctx, k2, v2), want, "windowed decode")
    assert torch.equal(k, k2) and torch.equal(v, v2)
    # with a mask besides, and after the window was taken away again
    m = torch.zeros((len(ctx), cfg.max_seq), device="cuda")
    m[:, ::3] = -float("inf")
    lay.set_window(0)
    lay.set_decode_path(1)
    want = decode(lay, cfg, x, ctx, k, v, hidden_mask(cfg, ctx, window, sinks) + m)
    plain = decode(lay, cfg, x, ctx, k, v)
    lay.set_window(window, sinks)
    assert_parity(decode(lay, cfg, x, ctx, k2, v2, m), want, "windowed and masked decode")
    lay.set_window(0)
    assert_parity(decode(lay, cfg, x, ctx, k2, v2), plain, "no window")
    assert lay.error() == 0
    lay.close()


@pytest.mark.parametrize("name,hist,T,window,sinks", [("tiny", 0, 40, 9, 2), ("tiny", 30, 5, 9, 2), ("tiny", 50, 1, 20, 0), ("tiny", 10, 60, 16, 30),
                                                      ("qwen05b", 300, 70, 100, 4), ("qwen05b", 0, 8, 3, 1), ("llama8b", 700, 33, 256, 4)])
def test_windowed_prefill_is_steps_with_a_mask(name, hist, T, window, sinks):
    """Prefills, prefills in chunks and a stack of one layer; the reference takes the tokens one by one."""
    log(f"windowed prefill {name} {hist} {T} {window} {sinks}")
    cfg, lay = layer(name)
    x = inputs(cfg, T)
    k, v = filled(cfg, lay, 1)
    start = [(k.clone(), v.clone()) for _ in range(3)]
    lay.set_decode_path(1)
    want = np.concatenate([decode(lay, cfg, x[t:t + 1].contiguous(), [hist + t], k, v, hidden_mask(cfg, [hist + t], window, sinks)) for t in range(T)])
    lay.set_window(window, sinks)
    for path, (k2, v2) in zip((0, 1), start):
        lay.set_decode_path(path)
        y = torch.empty_like(x)
        lay.prefill_kv(x, pos(hist, hist + T), hist, k2[0], v2[0], y)
        torch.cuda.synchronize()
        assert_parity(y.cpu().numpy(), want, f"windowed prefill, path {path}")
    k2, v2 = start[2]
    y = torch.empty_like(x)
    if hist == 0:
        lay.prefill_chunked(x, pos(0, T), 13, k2[0], v2[0], y)
    else:
        binding.Stack([lay]).prefill(x, pos(hist, hist + T), hist, [k2[0]], [v2[0]], y)
    torch.cuda.synchronize()
    assert_parity(y.cpu().numpy(), want, "chunks, or a stack")
    assert lay.error() == 0
    lay.close()


def test_slots_before_the_window_are_not_read():
    cfg, lay = layer("tiny")
    x = inputs(cfg, 20)
    lay.set_window(12, 3)
    outs = []
    for bad in (False, True):
        k, v = filled(cfg, lay, 1)
        if bad:
            for t in (k, v):
                t[:, :, 3:60 - 11] = 0x7FC0                  # (NaN)
        y, z = torch.empty_like(x), torch.empty_like(x[:1])
        lay.prefill_kv(x, pos(60, 80), 60, k[0], v[0], y)
        c = torch.tensor([80], dtype=torch.int32, device="cuda")
        lay.decode(x[:1].contiguous(), c, c, 80, k, v, z)
        torch.cuda.synchronize()
        outs.append((y, z))
    assert_parity(outs[1][0].cpu().numpy(), outs[0][0].cpu().numpy(), "prefill")
    assert_parity(outs[1][1].cpu().numpy(), outs[0][1].cpu().numpy(), "decode")
    lay.close()


@pytest.mark.parametrize("name,hist,T,window,sinks", [("tiny", 0, 1, 0, 0), ("tiny", 50, 8, 0, 0), ("tiny", 40, 30, 0, 0), ("tiny", 50, 20, 6, 2),
                                                      ("tiny", 30, 7, 4, 0), ("qwen05b", 300, 70, 0, 0), ("llama8b", 500, 20, 200, 4)])
def test_drafted_tokens_are_their_paths(name, hist, T, window, sinks):
    """Every node of a tree: the output, key and value that a prefill of its path alone gives for its last token."""
    log(f"drafted {name} {hist} {T} {window} {sinks}")
    cfg, lay = layer(name)
    x = inputs(cfg, T)
    rng = np.random.default_rng(T + hist)
    parents = [-1] + [int(rng.integers(max(0, i - 4), i)) for i in range(1, T)]
    k, v = filled(cfg, lay, 1)
    k0, v0 = k.clone(), v.clone()
    lay.set_window(window, sinks)
    tree = binding.DraftTree(1, T)
    tree.plan(torch.tensor([parents], dtype=torch.int32, device="cuda"), torch.tensor([hist], dtype=torch.int32, device="cuda"), window, sinks)
    for path in (0, 1):                      # (few tokens as rows of the decode's kernels, and as a prefill)
        lay.set_decode_path(path)
        k.copy_(k0), v.copy_(v0)
        y = torch.empty_like(x)
        lay.verify_tree(x, tree.pos[0], tree.mask[0], hist, k[0], v[0], y)
        torch.cuda.synchronize()
        assert torch.equal(k[0, :, :hist], k0[0, :, :hist]) and torch.equal(k[0, :, hist + T:], k0[0, :, hist + T:])
        picks = range(T) if T <= 30 else sorted({0, 1, T - 1, *rng.integers(0, T, 8).tolist()})
        got, want = [], []
        for i in picks:
            chain = O.ancestors(parents, i)[::-1]
            kk, vv = k0.clone(), v0.clone()
            yy = torch.empty((len(chain), cfg.hidden), dtype=torch.float32, device="cuda")
            lay.prefill_kv(x[chain].contiguous(), pos(hist, hist + len(chain)), hist, kk[0], vv[0], yy)
            torch.cuda.synchronize()
            got.append(y[i].cpu().numpy()), want.append(yy[-1].cpu().numpy())
            bits = lambda t, s: t[0, :, s].contiguous().view(torch.bfloat16).float().cpu().numpy()
            np.testing.assert_allclose(bits(k, hist + i), bits(kk, hist + len(chain) - 1), rtol=2.0 ** -7, atol=2e-2)
            np.testing.assert_allclose(bits(v, hist + i), bits(vv, hist + len(chain) - 1), rtol=2.0 ** -7, atol=2e-2)
        assert_parity(np.stack(got), np.stack(want), f"drafted tokens, path {path}")
    assert lay.error() == 0
    lay.close()


def test_refusals_and_sizes():
    cfg, lay = layer("tiny")
    h = lay.handle
    assert binding.layer_set_window(None, 1, 0) == binding.W4_EINVAL
    assert binding.layer_set_window(h, -1, 0) == binding.W4_EINVAL and binding.layer_set_window(h, 1, -1) == binding.W4_EINVAL
    lay.set_window(16, 2)
    assert binding.layer_set_kv_format(h, binding.W4_KV_INT4) == binding.W4_EUNSUPPORTED
    lay.set_decode_path(2)
    k, v = filled(cfg, lay, 1)
    x, c = inputs(cfg, 1), torch.tensor([3], dtype=torch.int32, device="cuda")
    with pytest.raises(binding.W4Error) as e:
        lay.decode(x, c, c, 3, k, v, torch.empty_like(x))
    assert e.value.code == binding.W4_EUNSUPPORTED
    lay.set_decode_path(0)
    y, ws, n = torch.empty_like(x), torch.empty(1 << 28, dtype=torch.uint8, device="cuda"), 1 << 28
    flat = k.view(-1)
    assert binding.layer_prefill(h, x, c, 1, flat.data_ptr() + 2, v, y, ws, n) == binding.W4_EINVAL         # (alignment)
    tree = binding.DraftTree(1, 1)

    def verify(T=1, hist=0, mask=tree.mask, kk=k, size=n):
        return binding.layer_verify_tree(h, x, c, mask, T, hist, kk, v, y, ws, size)

    assert verify(T=0) == binding.W4_EINVAL and verify(hist=-1) == binding.W4_EINVAL and verify(mask=None) == binding.W4_EINVAL
    assert verify(mask=tree.mask.data_ptr() + 4) == binding.W4_EINVAL and verify(kk=flat.data_ptr() + 2) == binding.W4_EINVAL
    assert verify(hist=128) == binding.W4_ECAPACITY and verify(size=100) == binding.W4_EWORKSPACE
    assert binding.layer_verify_tree(None, x, c, tree.mask, 1, 0, k, v, y, ws, n) == binding.W4_EINVAL
    lay.set_window(0)
    lay.set_kv_format("int4")
    assert verify() == binding.W4_EUNSUPPORTED and binding.layer_set_window(h, 4, 0) == binding.W4_EUNSUPPORTED
    assert binding.layer_workspace_size(h, 3, 1, 4, 10) == 0
    lay.set_kv_format("bf16")
    before = 0
    for T in range(1, 100):
        assert binding.layer_workspace_size(h, 3, 1, T, 20) >= before > -1
        before = binding.layer_workspace_size(h, 3, 1, T, 20)
    assert binding.layer_workspace_size(h, 3, 1, 257, 0) == 0
    lay.set_window(8, 0)                     # (a windowed decode fits the static scratch array)
    for B in (1, 8):
        assert 0 < binding.layer_workspace_size(h, 2, B, 1, 120) <= binding.layer_decode_noalloc_max_bytes()
    lay.close()
    big, lay = layer("llama8b")
    lay.set_window(1024, 4)
    assert 0 < binding.layer_workspace_size(lay.handle, 2, 8, 1, 4000) <= binding.layer_decode_noalloc_max_bytes()
    lay.close()


def test_one_mask_for_a_stack_of_windows():
    """Layers of different windows share a mask only where no window hides a node: those are the layers one by one, the
    others are refused."""
    cfg, w = host_layer("tiny")
    layers = [binding.Layer(cfg, w) for _ in range(3)]
    T, hist = 6, 40
    caches = [filled(cfg, layers[0], 1, seed=i) for i in range(3)]
    x = inputs(cfg, T)
    tree = binding.DraftTree(1, T)
    tree.plan(torch.tensor([[-1, 0, 0, 1, 3, 4]], dtype=torch.int32, device="cuda"), torch.tensor([hist], dtype=torch.int32, device="cuda"))
    stack = binding.Stack(layers)
    y = torch.empty_like(x)

    def run():
        stack.verify_tree(x, tree.pos[0], tree.mask[0], hist, [k[0] for k, _ in caches], [v[0] for _, v in caches], y)

    for lay, window in zip(layers, (0, 6, 17)):
        lay.set_window(window, 2)
    run()
    a, b = x, torch.empty_like(x)
    for lay, (k, v) in zip(layers, caches):
        lay.verify_tree(a, tree.pos[0], tree.mask[0], hist, k[0], v[0], b)
        a, b = b, torch.empty_like(x)
    torch.cuda.synchronize()
    assert_parity(y.cpu().numpy(), a.cpu().numpy(), "stack of windows")
    for windows in (((0, 0), (5, 2), (0, 0)), ((5, 2), (5, 1), (5, 2)), ((5, 2), (5, 2), (4, 2)), ((5, 2), (5, 2), (6, 2))):
        for lay, (window, sinks) in zip(layers, windows):
            lay.set_window(window, sinks)
        with pytest.raises(binding.W4Error) as e:
            run()
        assert e.value.code == binding.W4_EUNSUPPORTED
    for lay in layers:
        lay.set_window(5, 2)
    run()
    torch.cuda.synchronize()
    for lay in layers:
        lay.close()


def test_windowed_decode_without_allocation_and_captured():
    cfg, lay = layer("tiny")
    lay.set_window(20, 2)
    k, v = filled(cfg, lay, 3)
    x, c = inputs(cfg, 3), torch.tensor([90, 10, 50], dtype=torch.int32, device="cuda")
    y, z, w = (torch.empty_like(x) for _ in range(3))
    lay.decode(x, c, c, 90, k, v, y)
    binding.check(binding.layer_decode_noalloc(lay.handle, x, c, c, 90, None, 3, k, v, z))
    torch.cuda.synchronize()
    assert_parity(z.cpu().numpy(), y.cpu().numpy(), "noalloc")
    ws = torch.empty(binding.layer_workspace_size(lay.handle, 2, 3, 1, 90), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        binding.check(binding.layer_decode(lay.handle, x, c, c, 90, None, 3, k, v, w, ws, ws.numel()))
    for step in range(3):
        c.copy_(torch.tensor([90 - step, 10 + step, 50], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        lay.decode(x, c, c, 90, k, v, y)
        torch.cuda.synchronize()
        assert_parity(w.cpu().numpy(), y.cpu().numpy(), "replay")
    lay.close()


@pytest.mark.parametrize("window,sinks", [(0, 0), (24, 3)])
def test_drafted_model_gives_the_tokens_of_the_greedy_loop(window, sinks):
    """A stack of three layers with its embedding and LM head: the greedy loop, and the same by drafted trees (right and wrong
    guesses), each step embed, verify, head, accept and keep."""
    log(f"drafted model window {window}")
    cfg = synth.CONFIGS["tiny"]
    layers = [binding.Layer(cfg, synth.make_layer(cfg, i)) for i in range(3)]
    for lay in layers:
        lay.set_window(window, sinks)
    lw = synth.make_lm(cfg, 1024)
    lm, stack, prompt, steps, N = binding.LM(cfg, lw, max_batch=16), binding.Stack(layers), 20, 40, 12
    ids = (torch.arange(prompt, device="cuda") * 37 % 1024).to(torch.int32)
    x, y = (torch.empty((prompt, cfg.hidden), dtype=torch.float32, device="cuda") for _ in range(2))

    def start():
        caches = [lay.new_cache(1, 0) for lay in layers]
        lm.embed(ids, x)
        stack.prefill(x, pos(0, prompt), 0, [k[0] for k, _ in caches], [v[0] for _, v in caches], y)
        logits, nxt = torch.empty((1, 1024), device="cuda"), torch.empty(1, dtype=torch.int32, device="cuda")
        lm.head(y[-1:].contiguous(), logits, nxt)
        return caches, int(nxt)

    caches, token = start()
    greedy, margin = [token], []
    for i in range(steps + N):
        n = binding.model_decode_workspace_size(stack.handles, lm.handle, 1, cfg.max_seq - 1)
        ws, t = torch.empty(n, dtype=torch.uint8, device="cuda"), torch.tensor([token], dtype=torch.int32, device="cuda")
        c, logits = torch.tensor([prompt + i], dtype=torch.int32, device="cuda"), torch.empty((1, 1024), device="cuda")
        binding.check(binding.model_decode_greedy(stack.handles, lm.handle, t, c, c, cfg.max_seq - 1, 1, [k for k, _ in caches], [v for _, v in caches],
                                                  logits, t, ws, n))
        token = int(t)
        greedy.append(token)
        top = logits[0].topk(2).values
        margin.append(float(top[0] - top[1]))
    log(f"  smallest margin between the two largest logits {min(margin[:steps]):.4f}")

    caches, token = start()
    kv = [binding.KVCache(cfg, 1, k, v) for k, v in caches]
    tree, rng, taken, ctx, used = binding.DraftTree(1, N), np.random.default_rng(3), [token], prompt, 0
    x, y = (torch.empty((N, cfg.hidden), dtype=torch.float32, device="cuda") for _ in range(2))
    logits, picks = torch.empty((N, 1024), device="cuda"), torch.empty(N, dtype=torch.int32, device="cuda")
    while len(taken) < steps:
        parents, tokens, at = [-1], [taken[-1]], 0
        for guess in greedy[len(taken):]:
            if len(tokens) > N - 3:
                break
            for wrong in range(int(rng.integers(0, 3))):
                parents.append(at)
                tokens.append((guess + 1 + wrong) % 1024)
            parents.append(at)
            tokens.append(guess if rng.random() < 0.85 else (guess + 5) % 1024)
            at = len(tokens) - 1
        parents, tokens = parents[:N], tokens[:N]
        parents, tokens = parents + [-1] * (N - len(parents)), tokens + [0] * (N - len(tokens))
        p, t, c = (torch.tensor(z, dtype=torch.int32, device="cuda") for z in ([parents], [tokens], [ctx]))
        tree.plan(p, c, window, sinks)
        lm.embed(t[0], x)
        stack.verify_tree(x, tree.pos[0], tree.mask[0], ctx, [k[0] for k, _ in caches], [v[0] for _, v in caches], y)
        lm.head(y, logits, picks)
        tree.accept(p, t, picks[None])
        tree.keep(kv, c)
        n = int(tree.n_path)
        taken += [tokens[i] for i in tree.path[0, 1:n].tolist()] + [int(tree.next_tokens)]
        ctx, used = ctx + n, used + 1
    assert taken[:steps] == greedy[:steps] and used < 0.7 * steps
    assert all(lay.error() == 0 for lay in layers) and lm.error() == 0
    for lay in layers:
        lay.close()
    lm.close()
