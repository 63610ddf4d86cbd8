"""Attention with a sliding window and sinks, and the verification of drafted
tokens, over a bf16 key/value cache, as cases that can be timed and compared.

A query at position p sees slot j <= p of its sequence if j > p - window (or
window is 0) or j < sinks.  Kinds of case:

  decode   one query per sequence against its cached keys;
  prefill  T queries of one sequence behind a history;
  tree     N drafted tokens per sequence, held in the slots behind its context
           as a tree (parents): a node sees the context and its own ancestors,
           and stands at the context's length plus its depth.  The tree's masks
           and positions are part of the pass: every step drafts another one;
  settle   the end of such a step: the drafts' keys and values are put into
           the caches of some layers, the picks of the model are followed from
           the root for as long as they were drafted, and the slots of that
           path are moved together.

Fields: shape (a configuration of ``synth``), B sequences, ctx the longest
context (the others are at least half as long), T queries, hist cached tokens
before them, N drafted tokens, window, sinks, mask (decode: an additive mask
that hides the first slots), layers (settle).

``own`` selects between the plain form and the calls of the package.
"""
import math

import numpy as np
import torch

own = False

SHAPES = {"qwen05b": (14, 2, 64), "llama8b": (32, 8, 128), "qwen7b": (28, 4, 128)}   # heads, kv heads, head dim


def listed():
    return [
        # Chat on the smallest model, a token behind a short context: latency of a single small call.
        dict(name="decode-05b", kind="decode", shape="qwen05b", B=1, ctx=700, window=512, sinks=4, mask=False),
        # Serving prompts padded on the left, hidden by a mask.
        dict(name="decode-8b-mask", kind="decode", shape="llama8b", B=4, ctx=3001, window=1024, sinks=0, mask=True),
        # Serving long conversations, a full batch of ragged contexts far beyond the window: the largest transfer.
        dict(name="decode-7b-batch32", kind="decode", shape="qwen7b", B=32, ctx=16000, window=8192, sinks=4, mask=False),
        # A short follow-up message to the smallest model.
        dict(name="prefill-05b", kind="prefill", shape="qwen05b", T=61, hist=250, window=128, sinks=4),
        # A chunk of a prompt behind a long history.
        dict(name="prefill-8b", kind="prefill", shape="llama8b", T=512, hist=8192, window=4096, sinks=4),
        # A long document of odd length behind another one, the largest call.
        dict(name="prefill-7b-long", kind="prefill", shape="qwen7b", T=8001, hist=2999, window=4096, sinks=5),
        # A few drafted tokens on the smallest model.
        dict(name="tree-05b", kind="tree", shape="qwen05b", B=1, N=8, ctx=511, window=0, sinks=0),
        # A single conversation, drafted broadly.
        dict(name="tree-8b", kind="tree", shape="llama8b", B=1, N=64, ctx=8190, window=0, sinks=0),
        # Serving a batch of conversations, drafted narrowly.
        dict(name="tree-8b-batch16", kind="tree", shape="llama8b", B=16, N=13, ctx=4000, window=0, sinks=0),
        # A window of a long document, drafted as broadly as pays.
        dict(name="tree-7b-window", kind="tree", shape="qwen7b", B=4, N=129, ctx=16000, window=8192, sinks=4),
        # The end of a step of the smallest model.
        dict(name="settle-05b", kind="settle", shape="qwen05b", B=1, N=8, ctx=211, layers=2),
        # The end of a step of a batch of broad drafts.
        dict(name="settle-8b", kind="settle", shape="llama8b", B=16, N=64, ctx=300, layers=4),
    ]


def draw(rng):
    """One more case: shape, batch, lengths and window over their whole ranges."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))

    shape = rng.choice(["qwen05b", "llama8b", "qwen7b"])
    what = rng.random()
    window = 0 if rng.random() < 0.25 else log_int(1, 8192)
    sinks = 0 if rng.random() < 0.4 else rng.randint(1, 40)
    if what < 0.3:
        B = log_int(1, 32)
        ctx = log_int(1, min(32000, 8 * 16000 // B))
        return dict(kind="decode", shape=shape, B=B, ctx=ctx, window=window, sinks=sinks, mask=rng.random() < 0.3)
    if what < 0.6:
        T = log_int(1, 8000)
        hist = 0 if rng.random() < 0.3 else log_int(1, 14000)
        far = T * min(window + 64 if window else hist + T, hist + T) > 20000000
        return dict(kind="prefill", shape="qwen05b" if far else shape, T=T, hist=hist, window=min(window, 4096) if far and window else window,
                    sinks=sinks)
    B, N = log_int(1, 16), log_int(1, 200)
    if what < 0.9:
        ctx = log_int(1, min(16000, 64000 // B, 4000000 // (B * N)))
        return dict(kind="tree", shape=shape, B=B, N=N, ctx=ctx, window=window, sinks=sinks)
    return dict(kind="settle", shape=shape, B=B, N=min(N, 64), ctx=rng.randint(1, 300), layers=rng.randint(1, 4))


# ---------------------------------------------------------------- inputs

def lengths(case, seed):
    """Per sequence: the cached tokens before this call's."""
    if case["kind"] == "prefill":
        return [case["hist"]]
    top = case["ctx"]
    rng = np.random.default_rng(abs(int(seed)) * 2 + 1)
    return [top] + [int(rng.integers((top + 1) // 2, top + 1)) for _ in range(case["B"] - 1)]


def behind(case):
    """New tokens of a sequence, in the slots behind its context."""
    return {"decode": 1, "prefill": case.get("T")}.get(case["kind"], case.get("N"))


def capacity(case):
    """Slots of the cache."""
    return -(-(case.get("hist", case.get("ctx")) + behind(case)) // 256) * 256


def draft_tree(case, seed):
    """parents [B][N]: node 0 is the root, every other node hangs below one of the nodes before it, mostly a late one."""
    rng = np.random.default_rng(abs(int(seed)) * 7 + 5)
    B, N = case["B"], case["N"]
    back = np.minimum(rng.geometric(0.25, size=(B, N)), np.arange(N))
    parents = np.arange(N) - back
    parents[:, 0] = -1
    return torch.from_numpy(parents.astype(np.int32)).cuda()


def inputs(case, seed):
    """What the caller holds, from the seed alone: bf16 caches filled up to the last new token (keys with a few channels
    far from zero, as rotary keys have them), queries, contexts, mask; the trees and what a model picked."""
    nq, nkv, d = SHAPES[case["shape"]]
    g = torch.Generator(device="cuda").manual_seed((int(seed) * 1009 + 29) % (1 << 62))
    B, cap = case.get("B", 1), capacity(case)
    s = dict(case=case, lens=lengths(case, seed))
    s["ctx"] = torch.tensor(s["lens"], dtype=torch.int32, device="cuda")
    rand = dict(generator=g, device="cuda")
    shift = torch.randn((nkv, 1, d), **rand) * 4 * (torch.rand((nkv, 1, d), **rand) < 0.06)
    layers = case.get("layers", 1)
    s["k"] = [(torch.randn((B, nkv, cap, d), **rand) + shift).to(torch.bfloat16) for _ in range(layers)]
    s["v"] = [torch.randn((B, nkv, cap, d), **rand).to(torch.bfloat16) for _ in range(layers)]
    if case["kind"] in ("tree", "settle"):
        s["parents"] = draft_tree(case, seed)
    if case["kind"] == "settle":
        N = case["N"]
        s["k_new"] = [torch.randn((B, N, nkv, d), **rand).to(torch.bfloat16) for _ in range(layers)]
        s["v_new"] = [torch.randn((B, N, nkv, d), **rand).to(torch.bfloat16) for _ in range(layers)]
        # drafted tokens, and picks: of a node with children mostly the token of one of them
        s["tokens"] = torch.randint(0, 32000, (B, N), **rand).to(torch.int32)
        picks = torch.randint(0, 32000, (B, N), **rand)
        hit = torch.rand((B, N), **rand) < 0.7
        at = torch.where(hit & (s["parents"] >= 0), s["parents"], N).long()
        picks = torch.cat([picks, picks[:, :1]], 1)
        s["picks"] = picks.scatter_(1, at, s["tokens"].long())[:, :N].to(torch.int32).contiguous()
        return s
    rows = (case["T"],) if case["kind"] == "prefill" else (B, case["N"]) if case["kind"] == "tree" else (B,)
    s["q"] = torch.randn(rows + (nq, d), **rand).to(torch.bfloat16)
    s["mask"] = None
    if case.get("mask"):
        s["mask"] = torch.zeros((B, cap), device="cuda")
        for b in range(B):
            s["mask"][b, :(s["lens"][b] * (b + 1)) // (B + 1)] = -math.inf
    return s


def prepare(case, seed):
    """The inputs and the caches that a caller keeps."""
    s = inputs(case, seed)
    if own:
        from paper_2607_15865_amd import binding, synth
        cfg = synth.replace(synth.CONFIGS[case["shape"]], max_seq=capacity(case))
        s["cache"] = [binding.KVCache(cfg, case.get("B", 1), k, v) for k, v in zip(s["k"], s["v"])]
        if "parents" in s:
            s["tree"] = binding.DraftTree(case["B"], case["N"])
        if "q" in s:
            s["out"] = torch.empty_like(s["q"])
    return s


# ---------------------------------------------------------------- plain form

def plain_attend(q, k, v, seen):
    """q [..][m][d], k, v [..][n][d] fp32, seen [..][m][n] what is added to the scores (0 or -inf, or a mask's values)."""
    sc = torch.matmul(q, k.transpose(-1, -2).contiguous()) / math.sqrt(q.shape[-1]) + seen
    top = sc.amax(-1, keepdim=True)
    p = torch.exp(sc - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    return torch.matmul(p, v) / torch.where(total == 0, 1.0, total)


def plain_window(case, pos, slot):
    """0 where a query at pos sees the slot, else -inf."""
    seen = slot <= pos
    if case["window"]:
        seen &= (slot > pos - case["window"]) | (slot < case["sinks"])
    return torch.where(seen, 0.0, -math.inf)


def plain_decode(s):
    """The slots of the sinks and of the window are gathered, then all sequences at once."""
    case, q = s["case"], s["q"].float()
    B, nq, d = q.shape
    k, v = s["k"][0], s["v"][0]
    nkv, top = k.shape[1], case["ctx"] + 1
    pos = s["ctx"].long()[:, None]
    if case["window"] and case["window"] + case["sinks"] < top:
        slot = torch.arange(-case["sinks"], case["window"], device="cuda")[None]
        late = pos - slot
        slot = torch.where(slot < 0, slot + case["sinks"], late)
        seen = torch.where((late >= case["sinks"]) & (late <= pos) | (torch.arange(slot.shape[1], device="cuda")[None] < case["sinks"]) & (slot <= pos),
                           0.0, -math.inf)
        slot = slot.clamp(min=0)
    else:
        slot = torch.arange(top, device="cuda")[None].expand(B, -1)
        seen = plain_window(case, pos, slot)
    if s["mask"] is not None:
        seen = seen + s["mask"].gather(1, slot)
    at = slot[:, None, :, None].expand(-1, nkv, -1, d)
    out = plain_attend(q.view(B, nkv, nq // nkv, d), k.gather(2, at).float(), v.gather(2, at).float(), seen[:, None, None])
    return out.reshape(B, nq, d).to(torch.bfloat16)


def plain_prefill(s):
    """Kv head by kv head."""
    case, q = s["case"], s["q"].float()
    hist, T = case["hist"], case["T"]
    nq, d = q.shape[1:]
    k, v = s["k"][0][0], s["v"][0][0]
    nkv = k.shape[0]
    r = nq // nkv
    seen = plain_window(case, torch.arange(hist, hist + T, device="cuda")[:, None], torch.arange(hist + T, device="cuda")[None])
    out = torch.empty_like(s["q"])
    for h in range(nkv):
        heads = slice(h * r, (h + 1) * r)
        o = plain_attend(q[:, heads].transpose(0, 1).contiguous(), k[h, :hist + T].float()[None], v[h, :hist + T].float()[None], seen)
        out[:, heads] = o.transpose(0, 1).to(torch.bfloat16)
    return out


def plain_plan(s):
    """The ancestors of every node as words of 64 bits, and the nodes' positions."""
    case, parents = s["case"], s["parents"].long()
    B, N = parents.shape
    up = torch.zeros((B, N, N + 1), device="cuda")
    up.scatter_(2, torch.where(parents < 0, N, parents)[:, :, None], 1.0)
    up = up[:, :, :N].contiguous()
    reach = torch.eye(N, device="cuda") + up                # of 0 and 1 steps; then 2, 4, ..
    for _ in range(max(1, math.ceil(math.log2(N + 1)))):
        reach = (torch.matmul(reach, reach) > 0).float()
    depth = reach.sum(-1).long() - 1
    pos = s["ctx"].long()[:, None] + depth
    bits = (reach > 0) & (plain_window(case, pos[:, :, None], pos[:, None, :]) == 0)
    words = -(-N // 64)
    bits = torch.nn.functional.pad(bits, (0, words * 64 - N)).view(B, N, words, 64).long()
    return (bits << torch.arange(64, device="cuda")).sum(-1), pos.to(torch.int32), reach > 0


def plain_tree(s):
    """Sequence by sequence, all heads at once."""
    case, q = s["case"], s["q"].float()
    B, N, nq, d = q.shape
    words, pos, reach = plain_plan(s)
    k, v = s["k"][0], s["v"][0]
    nkv = k.shape[1]
    out = torch.empty_like(s["q"])
    for b in range(B):
        n, depth = s["lens"][b], pos[b].long()
        seen = torch.cat([plain_window(case, depth[:, None], torch.arange(n, device="cuda")[None]),
                          plain_window(case, depth[:, None], depth[None]).masked_fill(~reach[b], -math.inf)], 1)
        qb = q[b].view(N, nkv, nq // nkv, d).permute(1, 2, 0, 3).reshape(nkv, -1, d)
        o = plain_attend(qb, k[b, :, :n + N].float(), v[b, :, :n + N].float(), seen.repeat(nq // nkv, 1)[None])
        out[b] = o.view(nkv, nq // nkv, N, d).permute(2, 0, 1, 3).reshape(N, nq, d).to(torch.bfloat16)
    return [out, words, pos]


def plain_settle(s):
    B, N = s["tokens"].shape
    parents, tokens, picks = s["parents"].long(), s["tokens"].long(), s["picks"].long()
    row, node = torch.arange(B, device="cuda"), torch.arange(N, device="cuda")
    slots = s["ctx"].long()[:, None] + node
    for k, v, k_new, v_new in zip(s["k"], s["v"], s["k_new"], s["v_new"]):
        k[row[:, None], :, slots], v[row[:, None], :, slots] = k_new, v_new
    path = torch.full((B, N), -1, device="cuda")
    cur, alive = torch.zeros(B, dtype=torch.long, device="cuda"), torch.ones(B, dtype=torch.bool, device="cuda")
    last, n_path = cur, torch.zeros(B, dtype=torch.long, device="cuda")
    for t in range(N):
        path[:, t] = torch.where(alive, cur, -1)
        n_path += alive
        last = torch.where(alive, cur, last)
        fits = (parents == cur[:, None]) & (tokens == picks.gather(1, cur[:, None])) & alive[:, None]
        cur = torch.where(fits, node, N).amin(1)
        alive = cur < N
        cur = torch.where(alive, cur, 0)
    source = s["ctx"].long()[:, None] + torch.where(path < 0, node, path)
    for cache in (*s["k"], *s["v"]):
        cache[row[:, None], :, slots] = cache[row[:, None], :, source]
    return [path.to(torch.int32), n_path.to(torch.int32), picks.gather(1, last[:, None])[:, 0].to(torch.int32), *s["k"], *s["v"]]


# ---------------------------------------------------------------- one pass

def run(state):
    s, case = state, state["case"]
    kind = case["kind"]
    if not own:
        return {"decode": plain_decode, "prefill": plain_prefill, "tree": plain_tree, "settle": plain_settle}[kind](s)
    cache = s["cache"][0]
    if kind == "decode":
        cache.attn_decode(s["q"], s["ctx"], case["ctx"], s["out"], window=case["window"], sinks=case["sinks"], attn_mask=s["mask"])
        return s["out"]
    if kind == "prefill":
        cache.attn_prefill(s["q"], case["hist"], s["out"], window=case["window"], sinks=case["sinks"])
        return s["out"]
    tree = s["tree"]
    if kind == "tree":
        tree.plan(s["parents"], s["ctx"], window=case["window"], sinks=case["sinks"])
        cache.attn_tree(s["q"], tree, s["ctx"], case["ctx"], s["out"])
        return [s["out"], tree.mask, tree.pos]
    for c, k_new, v_new in zip(s["cache"], s["k_new"], s["v_new"]):
        c.append_step(k_new, v_new, s["ctx"])
    tree.accept(s["parents"], s["tokens"], s["picks"])
    tree.keep(s["cache"], s["ctx"])
    return [tree.path, tree.n_path, tree.next_tokens, *s["k"], *s["v"]]


def visible(case, pos):
    """Slots that a query at pos sees."""
    return min(pos + 1, case["window"] + min(case["sinks"], max(0, pos + 1 - case["window"]))) if case["window"] else pos + 1


def work(case):
    """Bytes and operations of one pass: the slots that some query sees once, the other inputs once, outputs once (ragged
    contexts: on average three quarters of the longest; drafts and moves as though every path were a quarter of the tree)."""
    nq, nkv, d = SHAPES[case["shape"]]
    slot, B = 2 * nkv * d * 2, case.get("B", 1)
    if case["kind"] == "decode":
        keys = visible(case, case["ctx"]) + (B - 1) * visible(case, case["ctx"] * 3 // 4)
        return {"bytes": keys * (slot + (4 if case["mask"] else 0)) + 2 * B * nq * d * 2, "flops": 4 * nq * d * keys}
    if case["kind"] == "prefill":
        T, hist = case["T"], case["hist"]
        pairs = sum(visible(case, hist + t) for t in range(T))
        keys = min(hist + T, visible(case, hist) + T)
        return {"bytes": keys * slot + 2 * T * nq * d * 2, "flops": 4 * nq * d * pairs}
    N = case["N"]
    if case["kind"] == "tree":
        keys = visible(case, case["ctx"]) + (B - 1) * visible(case, case["ctx"] * 3 // 4) + B * N
        return {"bytes": keys * slot + B * N * (2 * nq * d * 2 + 8 + 8 * -(-N // 64)), "flops": 4 * nq * d * N * keys}
    moved = case["layers"] * B * slot * (2 * N + 2 * (N // 4))
    return {"bytes": moved + B * N * 16, "flops": B * N * N}


# ---------------------------------------------------------------- 64 bits

def exact(case, seed):
    s = inputs(case, seed)
    nq, nkv, d = SHAPES[case["shape"]]
    r = nq // nkv

    def attend(qs, kk, vv, hidden, add=None):
        """Rows of qs [m][d] over keys [n][d]: weights by logsumexp, 0 for a row that sees nothing."""
        z = (qs.double() @ kk.double().T.contiguous()) * (float(d) ** -0.5)
        if add is not None:
            z = z + add.double()
        z[hidden.expand_as(z)] = -math.inf
        lse = torch.logsumexp(z, dim=-1, keepdim=True)
        return torch.exp(z - torch.where(lse == -math.inf, 0.0, lse)) @ vv.double()

    def out_of_reach(pos, slot):
        """True where a query at pos does not see the slot."""
        away = pos - slot
        late = away < 0
        return late | ((away >= case["window"]) & (slot >= case["sinks"])) if case["window"] > 0 else late

    def chain(parents, i):
        found = []
        while i >= 0:
            found.append(i)
            i = parents[i]
        return found

    if case["kind"] == "decode":
        out = torch.zeros((case["B"], nq, d), dtype=torch.float64, device="cuda")
        for b, n in enumerate(s["lens"]):
            hidden = out_of_reach(n, torch.arange(n + 1, device="cuda"))[None]
            for h in range(nkv):
                out[b, h * r:(h + 1) * r] = attend(s["q"][b, h * r:(h + 1) * r], s["k"][0][b, h, :n + 1], s["v"][0][b, h, :n + 1], hidden,
                                                   None if s["mask"] is None else s["mask"][b, :n + 1])
        return out
    if case["kind"] == "prefill":
        T, hist = case["T"], case["hist"]
        out = torch.zeros((T, nq, d), dtype=torch.float64, device="cuda")
        for t0 in range(0, T, 1024):                         # (1024 queries at a time)
            t1 = min(T, t0 + 1024)
            hidden = out_of_reach(torch.arange(hist + t0, hist + t1, device="cuda")[:, None], torch.arange(hist + t1, device="cuda")[None])
            for i in range(nq):
                out[t0:t1, i] = attend(s["q"][t0:t1, i], s["k"][0][0, i // r, :hist + t1], s["v"][0][0, i // r, :hist + t1], hidden)
        return out
    B, N = case["B"], case["N"]
    trees = s["parents"].tolist()
    if case["kind"] == "tree":
        out = torch.zeros((B, N, nq, d), dtype=torch.float64, device="cuda")
        words, places = np.zeros((B, N, -(-N // 64)), dtype=np.uint64), np.zeros((B, N), dtype=np.int64)
        for b, n in enumerate(s["lens"]):
            chains = [chain(trees[b], i) for i in range(N)]
            pos = np.array([n + len(c) - 1 for c in chains])
            hidden = np.ones((N, n + N), dtype=bool)
            hidden[:, :n] = out_of_reach(torch.from_numpy(pos)[:, None], torch.arange(n)[None]).numpy()
            for i, c in enumerate(chains):
                for a in c:
                    if not bool(out_of_reach(torch.tensor(int(pos[i])), torch.tensor(int(pos[a])))):
                        hidden[i, n + a] = False
                        words[b, i, a // 64] |= np.uint64(1) << np.uint64(a % 64)
            places[b] = pos
            hidden = torch.from_numpy(hidden).cuda()
            for i in range(nq):
                out[b, :, i] = attend(s["q"][b, :, i], s["k"][0][b, i // r, :n + N], s["v"][0][b, i // r, :n + N], hidden)
        return [out, torch.from_numpy(words.view(np.int64)).cuda(), torch.from_numpy(places).cuda()]
    tokens, picks = s["tokens"].tolist(), s["picks"].tolist()
    paths, lens, nexts = [], [], []
    for b, n in enumerate(s["lens"]):
        path = [0]
        while True:
            fits = [c for c in range(N) if trees[b][c] == path[-1] and tokens[b][c] == picks[b][path[-1]]]
            if not fits:
                break
            path.append(fits[0])
        for side in ("k", "v"):
            for cache, new in zip(s[side], s[side + "_new"]):
                rows = new[b].transpose(0, 1)
                cache[b, :, n:n + N] = rows
                cache[b, :, n:n + len(path)] = rows[:, path]
        paths.append(path + [-1] * (N - len(path)))
        lens.append(len(path))
        nexts.append(picks[b][path[-1]])
    whole = [torch.tensor(x, device="cuda") for x in (paths, lens, nexts)]
    return whole + [c.double() for c in (*s["k"], *s["v"])]
