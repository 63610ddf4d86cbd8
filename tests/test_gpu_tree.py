"""The steps of a draft tree on the GPU (plan, accept, append, keep) against oracle/kv_attn.py: whole numbers and bits,
so equal; and a run of the operators as a draft loop uses them, beside greedy decoding token by token."""
import random

import pytest
import torch

from oracle import kv_attn as O
from paper_2607_15865_amd import binding
from gpu_helpers import log
from test_gpu_kv_attn import config, filled, gen, randn, random_tree

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("window,sinks", [(0, 0), (0, 9), (1, 0), (2, 0), (5, 3), (5, 103), (64, 0), (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("N", [1, 2, 31, 63, 64, 65, 128, 129, 200, 256])
def test_plan(N, window, sinks):
    log(f"plan N {N} window {window} sinks {sinks}")
    g = gen(N + window % 97)
    ctx = [100, 0, -1, 7, 100]
    parents = torch.cat([random_tree(g, 1, N, k) for k in ("chain", "random", "random", "star", "forest")])
    tree = binding.DraftTree(5, N)
    tree.mask.fill_(-1)
    tree.plan(parents, ints(ctx), window=window, sinks=sinks)
    torch.cuda.synchronize()
    for b, p in enumerate(parents.tolist()):
        pos, sets = O.plan(p, ctx[b], window, sinks)
        assert tree.pos[b].tolist() == pos and tree.mask[b].tolist() == O.words(sets, N), b


@pytest.mark.parametrize("N", [1, 2, 5, 64, 65, 130, 256])
def test_accept(N):
    """Few different tokens, so that several children fit; whole chains; no child; picks that are no tokens."""
    log(f"accept N {N}")
    g, rng, B = gen(N), random.Random(N), 24
    parents = torch.cat([random_tree(g, 1, N, ("chain", "random", "star", "forest")[b % 4]) for b in range(B)])
    tokens = [[rng.randrange(3) for _ in range(N)] for _ in range(B)]
    picks = [[rng.randrange(3) for _ in range(N)] for _ in range(B)]
    tokens[0], picks[0] = list(range(N)), list(range(1, N + 1))                # (a chain that is taken whole)
    picks[1] = [-1] * N
    tokens[2] = [-1] * N
    tree = binding.DraftTree(B, N)
    tree.accept(parents, ints(tokens), ints(picks))
    torch.cuda.synchronize()
    for b, p in enumerate(parents.tolist()):
        path, pick = O.accept(p, tokens[b], picks[b])
        assert tree.path[b].tolist() == path + [-1] * (N - len(path)) and int(tree.n_path[b]) == len(path) and int(tree.next_tokens[b]) == pick, b
    assert int(tree.n_path[0]) == N


@pytest.mark.parametrize("strides", [False, True])
@pytest.mark.parametrize("nkv,d,T", [(2, 64, 1), (8, 128, 5), (3, 64, 70), (1, 128, 256)])
def test_append_step(nkv, d, T, strides):
    g, ctx, cap = gen(T + d), [0, -1, 40, 299, 300, 2 ** 31 - 1, -2 ** 31, 17], 300
    c = filled(g, nkv, nkv, d, cap, len(ctx), strides)
    want = [c.k.clone(), c.v.clone()]
    new = [randn(g, len(ctx), T, nkv, d) for _ in range(2)]
    c.append_step(*new, ints(ctx))
    torch.cuda.synchronize()
    for t, w, x in zip((c.k, c.v), want, new):
        for b, n in enumerate(ctx):
            for i in range(T):
                if n >= 0 and n + i < cap:
                    w[b, :, n + i] = x[b, i]
        assert torch.equal(t, w)


@pytest.mark.parametrize("strides", [False, True])
@pytest.mark.parametrize("nkv,d,N,layers", [(2, 64, 8, 1), (8, 128, 64, 3), (1, 64, 256, 2), (5, 128, 33, 70)])
def test_keep(nkv, d, N, layers, strides):
    """Rising paths of every length: none, the whole, the last nodes, and one past the cache's end; padded sequences."""
    log(f"keep nkv {nkv} d {d} N {N} layers {layers}")
    g, rng = gen(N), random.Random(N)
    paths = [[0], list(range(N)), [0] + list(range(max(1, N - 3), N)), [0, N - 1]] + [[0] + sorted(rng.sample(range(1, N), rng.randrange(1, N)))
                                                                               for _ in range(3)]
    B, cap = len(paths), 100 + N
    ctx = [3, 40, 100, 70, 0, -1, cap - N // 2]
    caches = [filled(g, nkv, nkv, d, cap, B, strides) for _ in range(layers)]
    want = [(c.k.clone(), c.v.clone()) for c in caches]
    tree = binding.DraftTree(B, N)
    tree.path.fill_(-1)
    for b, p in enumerate(paths):
        tree.path[b, :len(p)] = ints(p)
        tree.n_path[b] = len(p)
    tree.keep(caches, ints(ctx))
    torch.cuda.synchronize()
    for c, w in zip(caches, want):
        for t, x in zip((c.k, c.v), w):
            y = x.clone()
            for b, p in enumerate(paths):
                for i, f in enumerate(p):
                    if ctx[b] >= 0 and ctx[b] + f < cap:
                        y[b, :, ctx[b] + i] = x[b, :, ctx[b] + f]
            assert torch.equal(t, y)


def test_keep_of_counts_and_paths_that_are_none():
    g = gen(3)
    c = filled(g, 2, 2, 64, 50, 4)
    before = c.k.clone()
    tree = binding.DraftTree(4, 6)
    tree.path.copy_(ints([[-1] * 6, [0, 9, 2 ** 31 - 1, -4, 3, 5], [0, 1, 2, 3, 4, 5], [5] * 6]))
    tree.n_path.copy_(ints([0, 5, -3, 2 ** 31 - 1]))
    tree.keep([c], ints([10, 10, 10, 20]))
    torch.cuda.synchronize()
    assert torch.equal(c.k[:3], before[:3])                  # (path[4] = 3 lies before its place)
    for t in range(5):
        assert torch.equal(c.k[3, :, 20 + t], before[3, :, 25])


def test_settled_step_captured_and_replayed():
    g, N = gen(4), 12
    caches = [filled(g, 4, 2, 64, 200, 2) for _ in range(2)]
    tree, ctx = binding.DraftTree(2, N), ints([5, 60])
    parents, tokens, picks = random_tree(g, 2, N, "random"), ints([[0] * N] * 2), ints([[0] * N] * 2)
    new = [randn(g, 2, N, 2, 64) for _ in range(4)]

    def step():
        for i, c in enumerate(caches):
            c.append_step(new[2 * i], new[2 * i + 1], ctx)
        tree.accept(parents, tokens, picks)
        tree.keep(caches, ctx)

    step()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        parents.copy_(random_tree(g, 2, N, "random"))
        tokens.copy_(torch.randint(0, 2, (2, N), generator=g, device="cuda"))
        ctx.copy_(ints([5 + i, 60 - i]))
        for t in new:
            t.copy_(randn(g, *t.shape))
        step()
        torch.cuda.synchronize()
        want = [t.clone() for c in caches for t in (c.k, c.v)] + [tree.path.clone(), tree.n_path.clone(), tree.next_tokens.clone()]
        for c in caches:
            c.k.add_(1)
        tree.path.fill_(3)
        for c, k in zip(caches, want[::2]):
            c.k.copy_(k)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip([t for c in caches for t in (c.k, c.v)] + [tree.path, tree.n_path, tree.next_tokens], want))


@pytest.mark.parametrize("window,sinks", [(0, 0), (24, 2)])
def test_draft_loop_gives_the_tokens_of_greedy_decoding(window, sinks):
    """A model of one attention layer with random tables, whose pick is the largest logit.  Decoded token by token, and by drafts (right, wrong and late
    guesses in random trees): the loop stays on the device, and gives the same tokens and the same cache.  Positions do not enter the
    keys here, so that rows are the same wherever they are written."""
    log(f"draft loop window {window}")
    nq, nkv, d, V, prompt, steps, N = 8, 2, 64, 50, 30, 60, 10
    g, rng = gen(window + 1), random.Random(1)
    wq, wk, wv = (randn(g, V, n, d) for n in (nq, nkv, nkv))
    head = torch.randn((nq * d, V), generator=g, device="cuda") * 4
    cfg = config(nq, nkv, d, 256)

    def start():
        c = binding.KVCache(cfg, 1)
        c.k.zero_(), c.v.zero_()
        t = torch.arange(prompt, device="cuda") * 7 % V
        c.append(wk[t][None].contiguous(), wv[t][None].contiguous(), [0])
        return c, 11

    c, token = start()
    out, greedy = torch.empty((1, nq, d), dtype=torch.bfloat16, device="cuda"), []
    for i in range(steps + N):
        ctx = ints([prompt + i])
        c.append_step(wk[token][None, None].contiguous(), wv[token][None, None].contiguous(), ctx)
        c.attn_decode(wq[token][None].contiguous(), ctx, 255 - N, out, window=window, sinks=sinks)
        token = int((out.float().view(1, -1) @ head).argmax())
        greedy.append(token)

    d_c, token = start()
    tree, taken, ctx, used = binding.DraftTree(1, N), [], ints([prompt]), 0
    outs = torch.empty((1, N, nq, d), dtype=torch.bfloat16, device="cuda")
    while len(taken) < steps:
        # guesses: the right continuation with some wrong siblings before or after it
        parents, tokens, at = [-1], [token], 0
        for guess in greedy[len(taken):]:
            if len(tokens) >= N - 2:
                break
            for wrong in range(rng.randrange(3)):
                if len(tokens) < N - 1:
                    parents.append(at)
                    tokens.append((guess + 1 + wrong) % V)
            parents.append(at)
            tokens.append(guess if rng.random() < 0.8 else (guess + 3) % V)
            at = len(tokens) - 1
        parents, tokens = (x[:N] + [-1] * (N - len(x)) for x in (parents, tokens))
        t = ints([tokens])
        rows = t.long().clamp(min=0)
        d_c.append_step(wk[rows].contiguous(), wv[rows].contiguous(), ctx)
        tree.plan(ints([parents]), ctx, window=window, sinks=sinks)
        d_c.attn_tree(wq[rows].contiguous(), tree, ctx, 255 - N, outs)
        picks = (outs.float().view(1, N, -1) @ head).argmax(-1).to(torch.int32)
        tree.accept(ints([parents]), t, picks)
        tree.keep([d_c], ctx)
        ctx = ctx + tree.n_path
        n = int(tree.n_path)
        taken += [tokens[i] for i in tree.path[0, 1:n].tolist()] + [int(tree.next_tokens)]
        token, used = taken[-1], used + 1
    assert taken[:steps] == greedy[:steps] and used < 0.7 * steps
    n = min(int(ctx), prompt + steps)
    assert torch.equal(d_c.k[:, :, :n], c.k[:, :, :n]) and torch.equal(d_c.v[:, :, :n], c.v[:, :, :n])
