"""Operators over a key/value cache held in 4 bits, as cases that can be timed and compared.

The cache holds, per token and kv head, 4-bit codes of the head's dims in
groups of 32.  Of a group's values x (bf16, taken as fp16):

    lo = min x,  s = fp16((max x - lo) / 15),  c = min(15, floor((x - lo) / s + 1/2))

(c = 0 where s = 0); the value that is held is lo + s c.  Kinds of case:

  store    new keys and values are written into the cache (ragged slots, one
           run of T per sequence) and read back as bf16 values;
  decode   one query per sequence against its cached keys;
  prefill  T queries of one sequence, causal, over a history and themselves.

Fields: shape (a configuration of ``synth``), B sequences, T tokens, hist
cached tokens before them, ctx the longest context of a decode (the others are
at least half as long), step (store: slots on the device, one token per
sequence), mask (decode: an additive mask that hides the first slots).

``own`` selects between the plain form and the calls of the package.
"""
import math

import numpy as np
import torch

own = False

GROUP = 32
SHAPES = {"qwen05b": (14, 2, 64), "llama8b": (32, 8, 128), "qwen7b": (28, 4, 128)}   # heads, kv heads, head dim


def listed():
    return [
        # One decode step of the smallest model: its key and value go into the cache; latency of the smallest calls.
        dict(name="store-05b-step", kind="store", shape="qwen05b", B=1, T=1, hist=511, step=True),
        # Speculative decoding in a batch: a few accepted tokens of eight sequences at ragged slots.
        dict(name="store-8b-draft", kind="store", shape="llama8b", B=8, T=5, hist=2043, step=False),
        # A prompt of odd length moved into the cache.
        dict(name="store-7b-prompt", kind="store", shape="qwen7b", B=1, T=2011, hist=0, step=False),
        # A whole long conversation taken into the cache and handed out again, the largest transfer.
        dict(name="store-8b-long", kind="store", shape="llama8b", B=2, T=16384, hist=3, step=False),
        # Chat on the smallest model: one token, short context; latency of a single small call.
        dict(name="decode-05b", kind="decode", shape="qwen05b", B=1, ctx=512, mask=False),
        # The headline decode step of the 8B-shaped layer.
        dict(name="decode-8b", kind="decode", shape="llama8b", B=1, ctx=2048, mask=False),
        # Serving prompts padded on the left, hidden by a mask.
        dict(name="decode-8b-mask", kind="decode", shape="llama8b", B=4, ctx=1500, mask=True),
        # Serving: a full batch of long, ragged contexts, seven query heads per kv head.
        dict(name="decode-7b-batch8", kind="decode", shape="qwen7b", B=8, ctx=8192, mask=False),
        # Serving long documents, for which the cache is held in 4 bits in the first place.
        dict(name="decode-8b-long", kind="decode", shape="llama8b", B=16, ctx=32767, mask=False),
        # A short follow-up message to the smallest model.
        dict(name="prefill-05b", kind="prefill", shape="qwen05b", T=61, hist=250),
        # A chunk of a prompt after a history.
        dict(name="prefill-8b", kind="prefill", shape="llama8b", T=512, hist=4096),
        # The last chunk of a long document, odd lengths, the largest call.
        dict(name="prefill-7b-long", kind="prefill", shape="qwen7b", T=2011, hist=14001),
    ]


def draw(rng):
    """One more case: shape, batch and lengths over their whole ranges."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    shape = rng.choice(["qwen05b", "llama8b", "qwen7b"])
    what = rng.random()
    if what < 0.3:
        B = log_int(1, 16)
        step = rng.random() < 0.25
        T = 1 if step else log_int(1, 32768 // B)
        return dict(kind="store", shape=shape, B=B, T=T, hist=rng.randint(0, 2000), step=step)
    if what < 0.7:
        B = log_int(1, 32)
        ctx = log_int(1, min(32000, 16 * 32000 // B))
        return dict(kind="decode", shape=shape, B=B, ctx=ctx, mask=rng.random() < 0.3)
    T = log_int(1, 2000)
    hist = 0 if rng.random() < 0.3 else log_int(1, 14000)
    return dict(kind="prefill", shape="qwen7b" if T * (hist + T) > 8000000 else shape, T=T, hist=hist)


# ---------------------------------------------------------------- inputs

def lengths(case, seed):
    """Per sequence: the cached tokens before this call's (store: its first slot)."""
    if case["kind"] == "prefill":
        return [case["hist"]]
    top = case["hist"] if case["kind"] == "store" else case["ctx"]
    rng = np.random.default_rng(abs(int(seed)) * 2 + 1)
    return [top] + [int(rng.integers((top + 1) // 2, top + 1)) for _ in range(case["B"] - 1)]


def capacity(case):
    """Slots of the cache."""
    n = case["ctx"] + 1 if case["kind"] == "decode" else case["hist"] + case["T"]
    return -(-n // 256) * 256


def keys_values(g, B, n, nkv, d):
    """bf16 [B][n][nkv][d]: keys with a few channels far from zero, as rotary keys have them, and plain values."""
    rand = dict(generator=g, device="cuda", dtype=torch.float32)
    shift = torch.randn((nkv, d), **rand) * 4 * (torch.rand((nkv, d), **rand) < 0.06)
    k = torch.empty((B, n, nkv, d), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    for b in range(B):
        k[b] = torch.randn((n, nkv, d), **rand) + shift
        v[b] = torch.randn((n, nkv, d), **rand)
    return k, v


def inputs(case, seed):
    """What the caller holds, from the seed alone: bf16 keys, values and queries, contexts, mask."""
    nq, nkv, d = SHAPES[case["shape"]]
    g = torch.Generator(device="cuda").manual_seed((int(seed) * 1009 + 17) % (1 << 62))
    s = dict(case=case, lens=lengths(case, seed))
    if case["kind"] == "store":
        s["k"], s["v"] = keys_values(g, case["B"], case["T"], nkv, d)
        return s
    B = case.get("B", 1)
    n = case["ctx"] + 1 if case["kind"] == "decode" else case["hist"] + case["T"]
    s["k"], s["v"] = keys_values(g, B, n, nkv, d)
    rows = B if case["kind"] == "decode" else case["T"]
    s["q"] = torch.randn((rows, nq, d), generator=g, device="cuda").to(torch.bfloat16)
    s["mask"] = None
    if case.get("mask"):
        cap = capacity(case)
        s["mask"] = torch.zeros((B, cap), device="cuda")
        for b in range(B):
            s["mask"][b, :(s["lens"][b] * (b + 1)) // (B + 1)] = -math.inf
    return s


def prepare(case, seed):
    """The inputs and the cache that a caller keeps: for attention, already filled."""
    s = inputs(case, seed)
    nq, nkv, d = SHAPES[case["shape"]]
    B, cap = case.get("B", 1), capacity(case)
    if case["kind"] != "store":
        s["lens_dev"] = torch.tensor(s["lens"], dtype=torch.int32, device="cuda")
    if own:
        from paper_2607_15865_amd import binding, synth
        s["cache"] = binding.KV4Cache(synth.replace(synth.CONFIGS[case["shape"]], max_seq=cap), B)
        if case["kind"] == "store":
            s["k_out"], s["v_out"] = torch.empty_like(s["k"]), torch.empty_like(s["v"])
            s["lens_dev"] = torch.tensor(s["lens"], dtype=torch.int32, device="cuda")
        else:
            s["cache"].append(s["k"], s["v"], [0] * B)
            s["out"] = torch.empty_like(s["q"])
    elif case["kind"] == "store":
        s["cache"] = [plain_empty(B, nkv, cap, d) for _ in range(2)]
    else:
        s["cache"] = [plain_quantise(s[x].transpose(1, 2)) for x in ("k", "v")]
    if case["kind"] != "store":
        del s["k"], s["v"]
    return s


# ---------------------------------------------------------------- plain form

def plain_empty(B, nkv, n, d):
    return (torch.zeros((B, nkv, n, d), dtype=torch.uint8, device="cuda"),
            torch.zeros((B, nkv, n, d // GROUP), dtype=torch.float16, device="cuda"),
            torch.zeros((B, nkv, n, d // GROUP), dtype=torch.float16, device="cuda"))


def plain_quantise(x):
    """Codes [..][d], scales and offsets [..][d / GROUP] of values [B][..][d] (in 64 bits: codes lie next to borders)."""
    codes = torch.empty(x.shape, dtype=torch.uint8, device=x.device)
    scale = torch.empty(x.shape[:-1] + (x.shape[-1] // GROUP,), dtype=torch.float16, device=x.device)
    low = torch.empty_like(scale)
    for b in range(x.shape[0]):                      # (a sequence at a time: 64-bit copies are large)
        g = x[b].half().double().unflatten(-1, (-1, GROUP))
        lo, hi = g.amin(-1), g.amax(-1)
        s = ((hi - lo) / 15).half()
        sd = s.double().unsqueeze(-1)
        q = torch.floor((g - lo.unsqueeze(-1)) / torch.where(sd > 0, sd, torch.inf) + 0.5)
        codes[b] = q.clamp(max=15).flatten(-2).to(torch.uint8)
        scale[b], low[b] = s, lo.half()
    return codes, scale, low


def plain_values(cache):
    """fp32 values that the codes stand for."""
    codes, scale, low = cache
    g = codes.float().unflatten(-1, (-1, GROUP))
    return (low.float().unsqueeze(-1) + scale.float().unsqueeze(-1) * g).flatten(-2)


def plain_store(s):
    T = s["case"]["T"]
    out = []
    for name, cache in zip(("k", "v"), s["cache"]):
        new = plain_quantise(s[name].transpose(1, 2))
        back = []
        for b, at in enumerate(s["lens"]):
            for part, val in zip(cache, new):
                part[b, :, at:at + T] = val[b]
            back.append(plain_values([part[b, :, at:at + T] for part in cache]).transpose(0, 1))
        out.append(torch.stack(back).to(torch.bfloat16))
    return out


def plain_softmax_out(scores, v):
    p = torch.exp(scores - scores.amax(-1, keepdim=True))
    return torch.matmul(p, v) / p.sum(-1, keepdim=True)


def plain_decode(s):
    """Sequence by sequence: scores, softmax and output over the visible keys."""
    q = s["q"].float()
    B, nq, d = q.shape
    nkv = s["cache"][0][0].shape[1]
    out = torch.empty_like(s["q"])
    for b in range(B):
        n = s["lens"][b] + 1
        k, v = (plain_values([part[b, :, :n] for part in cache]) for cache in s["cache"])
        sc = torch.matmul(q[b].view(nkv, nq // nkv, d), k.transpose(1, 2).contiguous()) / math.sqrt(d)
        if s["mask"] is not None:
            sc = sc + s["mask"][b, :n]
        out[b] = plain_softmax_out(sc, v).reshape(nq, d).to(torch.bfloat16)
    return out


def plain_prefill(s):
    """Kv head by kv head, with the causal mask after the history."""
    hist, T = s["case"]["hist"], s["case"]["T"]
    q = s["q"].float()
    _, nq, d = q.shape
    k, v = (plain_values([part[0] for part in cache]) for cache in s["cache"])
    nkv, n = k.shape[0], k.shape[1]
    r = nq // nkv
    late = torch.arange(n, device="cuda")[None, :] > torch.arange(T, device="cuda")[:, None] + hist
    out = torch.empty_like(s["q"])
    for h in range(nkv):
        qh = q[:, h * r:(h + 1) * r].transpose(0, 1).contiguous()
        sc = torch.matmul(qh, k[h].t().contiguous()) / math.sqrt(d)
        sc.masked_fill_(late, -math.inf)
        out[:, h * r:(h + 1) * r] = plain_softmax_out(sc, v[h]).transpose(0, 1).to(torch.bfloat16)
    return out


# ---------------------------------------------------------------- one pass

def run(state):
    s, kind = state, state["case"]["kind"]
    if not own:
        return {"store": plain_store, "decode": plain_decode, "prefill": plain_prefill}[kind](s)
    cache, case = s["cache"], s["case"]
    if kind == "store":
        if case["step"]:
            cache.append_step(s["k"], s["v"], s["lens_dev"])
        else:
            cache.append(s["k"], s["v"], s["lens"])
        cache.read(s["lens"], case["T"], s["k_out"], s["v_out"])
        return [s["k_out"], s["v_out"]]
    if kind == "decode":
        cache.attn_decode(s["q"], s["lens_dev"], case["ctx"], s["out"], attn_mask=s["mask"])
    else:
        cache.attn_prefill(s["q"], case["hist"], s["out"])
    return s["out"]


def work(case):
    """Bytes and operations of one pass: inputs and the cache's slots once, outputs once (ragged contexts: on average
    three quarters of the longest)."""
    nq, nkv, d = SHAPES[case["shape"]]
    slot = 2 * nkv * (d // 2 + d // GROUP * 4)               # of the cache, K and V
    if case["kind"] == "store":
        n = case["B"] * case["T"]
        return {"bytes": 2 * n * slot + 2 * n * 2 * nkv * d * 2, "flops": 10 * n * 2 * nkv * d}
    if case["kind"] == "decode":
        keys = case["ctx"] + 1 + (case["B"] - 1) * (case["ctx"] * 3 // 4 + 1)
        return {"bytes": keys * (slot + (4 if case["mask"] else 0)) + 2 * case["B"] * nq * d * 2, "flops": 4 * nq * d * keys}
    pairs = case["T"] * case["hist"] + case["T"] * (case["T"] + 1) // 2
    return {"bytes": (case["hist"] + case["T"]) * slot + 2 * case["T"] * nq * d * 2, "flops": 4 * nq * d * pairs}


# ---------------------------------------------------------------- 64 bits

def exact_values(x):
    """float64 values that the cache holds of bf16 values [..][d]: the code counts the borders (k + 1/2) s at or
    below x - lo."""
    near = x.to(torch.float16).to(torch.float64)             # (one rounding: bf16 values are wider only in range)
    out = torch.empty_like(near)
    for i in range(0, x.shape[-1], GROUP):
        g = near[..., i:i + GROUP]
        lo = torch.min(g, dim=-1, keepdim=True).values
        span = (torch.max(g, dim=-1, keepdim=True).values - lo) / 15.0
        s = torch.from_numpy(span.cpu().numpy().astype(np.float16).astype(np.float64)).to(x.device)
        code = torch.zeros_like(g)
        for k in range(15):
            code += ((g - lo) >= (k + 0.5) * s) & (s > 0)
        out[..., i:i + GROUP] = lo + s * code
    return out


def exact(case, seed):
    nq, nkv, d = SHAPES[case["shape"]]
    s = inputs(case, seed)
    if case["kind"] == "store":
        return [exact_values(s["k"]), exact_values(s["v"])]
    rows, r = s["q"].shape[0], nq // nkv
    out = torch.zeros((rows, nq, d), dtype=torch.float64, device="cuda")
    q = s["q"].to(torch.float64)

    def attend(qs, kk, vv, add):
        z = (qs @ kk.T.contiguous()) * (float(d) ** -0.5)
        if add is not None:
            z = z + add
        return torch.exp(z - torch.logsumexp(z, dim=-1, keepdim=True)) @ vv

    for h in range(nkv):
        heads = slice(h * r, (h + 1) * r)
        if case["kind"] == "decode":
            for b in range(rows):
                n = s["lens"][b] + 1
                kk, vv = exact_values(s["k"][b, :n, h]), exact_values(s["v"][b, :n, h])
                out[b, heads] = attend(q[b, heads].contiguous(), kk, vv, None if s["mask"] is None else s["mask"][b, :n].double())
            continue
        kk, vv = exact_values(s["k"][0, :, h]), exact_values(s["v"][0, :, h])
        for t0 in range(0, rows, 256):                       # (256 queries at a time)
            t1 = min(rows, t0 + 256)
            n = case["hist"] + t1
            seen = torch.arange(n, device="cuda")[None] <= torch.arange(t0, t1, device="cuda")[:, None] + case["hist"]
            add = torch.where(seen, 0.0, -math.inf).double()
            for i in range(h * r, (h + 1) * r):
                out[t0:t1, i] = attend(q[t0:t1, i].contiguous(), kk[:n], vv[:n], add)
    return out
