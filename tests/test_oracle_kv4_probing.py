"""The bound and the probing queries with which the prefill kernel is tested (oracle.kv4.attend_heads, probing_queries):
the bound holds for a computation in the kernel's precision, and mistakes of the kinds that a kernel makes pass it."""
import numpy as np
import pytest
import torch

from oracle import kv4
from oracle.layer import round_bf16

SHAPES = [(7, 1, 128, 160, 1501), (4, 4, 64, 300, 0), (6, 2, 64, 181, 970), (16, 2, 128, 70, 63)]


def setup(nq, nkv, d, T, first, seed=1):
    rng = np.random.default_rng(seed)
    n = first + T
    k, v = (round_bf16(rng.standard_normal((nkv, n, d)) + (rng.random(d) < 0.06) * rng.standard_normal(d) * 5) for _ in range(2))
    q = kv4.probing_queries(rng, k, nq, T, first)
    k16, v16 = (torch.from_numpy(kv4.fp16_operands(kv4.held(x))) for x in (k, v))
    return torch.from_numpy(q), k16, v16


def limit(out, tol):
    return tol * 1.01 + out.abs() * 2.0 ** -8


@pytest.mark.parametrize("shape", SHAPES)
def test_bound_holds_in_the_kernel_s_precision(shape):
    """fp32 scores and sums, weights rounded to fp16, the result to bf16: within the bound everywhere; and the bound is
    small beside the outputs."""
    nq, nkv, d, T, first = shape
    q, k, v = setup(*shape)
    n, r = k.shape[1], nq // nkv
    seen = torch.arange(n)[None] <= torch.arange(T)[:, None] + first
    for h, out, tol in kv4.attend_heads(q, k, v, first):
        z = torch.where(seen, (q[:, h].float() @ k[h // r].float().t()) * d ** -0.5, -torch.inf)
        p = torch.exp(z - z.amax(-1, keepdim=True))
        got = ((p.half().float() @ v[h // r].float()) / p.sum(-1, keepdim=True)).bfloat16().double()
        assert ((got - out).abs() <= limit(out, tol)).all()
        assert tol.median() < 0.02 * out.abs().median()


@pytest.mark.parametrize("shape", SHAPES)
def test_attend_heads_against_attend(shape):
    nq, nkv, d, T, first = shape
    q, k, v = setup(*shape)
    n = k.shape[1]
    got = {h: out for h, out, _ in kv4.attend_heads(q, k, v, first)}
    for t in (0, T // 2, T - 1):
        ref, _ = kv4.attend(q[t].numpy(), k.numpy(), v.numpy(), np.arange(n) <= first + t)
        for h in range(nq):
            assert np.allclose(got[h][t].numpy(), ref[h], rtol=1e-10, atol=1e-12)


def caught(good, bad):
    """Rows [T] of each head where the wrong result passes the bound: [nq][T]."""
    return torch.stack([((b[1] - g[1]).abs() > limit(g[1], g[2]) + g[1].abs() * 2.0 ** -7).any(-1) for g, b in zip(good, bad)])


@pytest.mark.parametrize("shape", SHAPES)
def test_mistakes_are_seen(shape):
    """A stage of 64 keys left out, for each stage and each block of 256 rows; the mask one key too short or too long; a
    plain average; zeros; scores 3% too small; another kv head's keys or values."""
    nq, nkv, d, T, first = shape
    q, k, v = setup(*shape)
    n, r = k.shape[1], nq // nkv
    good = list(kv4.attend_heads(q, k, v, first))

    def wrong(q=q, k=k, v=v, first=first, drop=None):
        return caught(good, list(kv4.attend_heads(q, k, v, first, drop=drop)))

    row = (torch.arange(T)[:, None] * r + torch.arange(nq)[None] % r).t()           # [nq][T]: of its kv head
    last, j = torch.arange(T)[:, None] + first, torch.arange(n)[None]
    stages = (n + 63) // 64
    blocks = 0
    for st in range(stages):
        bad = wrong(drop=(j // 64 == st) & (last >= 64))     # (rows that see nothing else keep it)
        for g in range(nkv):
            heads = slice(g * r, (g + 1) * r)
            for b0 in range(0, T * r, 256):
                block = (row[heads] >= b0) & (row[heads] < b0 + 256)
                whole = block & (last[:, 0] >= max(64, 64 * st + 63))               # rows that see all of the stage
                if int(whole.sum()) >= 2 * stages:           # (every other row looks at a stage)
                    assert bad[heads][block].any(), (st, g, b0)
                    blocks += 1
    assert blocks > 0
    short, long = wrong(drop=(j == last) & (last > 0)), wrong(first=first + 1)
    for h in range(nq):                                      # rows near the last key, and near the one behind it
        assert short[h][(row[h] % 8 == 1) & (last[:, 0] > 0)].all()
        assert long[h][(row[h] % 8 == 3)[:-1].nonzero()].all()
    assert caught(good, [(h, v[h // r].mean(0).expand(T, d)) for h in range(nq)]).any(-1).all()
    assert wrong(v=v * 0).any(-1).all()
    assert wrong(q=q * 0.97).any()
    if nkv > 1:
        assert wrong(k=k.flip(0).contiguous()).any(-1).all() and wrong(v=v.flip(0).contiguous()).any(-1).all()
