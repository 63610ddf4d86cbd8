"""How the prefill over the 4-bit cache deals out its work, on the host: every stage of every row tile has one block, a
state one slot inside the workspace, and the merge finds the states."""
import os
import random

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2607_15865_amd", "libw4layer.so")

if not os.path.exists(LIB):
    from paper_2607_15865_amd import build as _b
    _b.build()

import ctypes  # noqa: E402

from paper_2607_15865_amd import binding as B  # noqa: E402
from paper_2607_15865_amd import synth  # noqa: E402
import test_gpu_kv4_prefill as G  # noqa: E402


def plan(T, hist, nkv, r, d):
    x = [ctypes.c_int() for _ in range(4)]
    B._lib.w4_kv4_prefill_plan(T, hist, nkv, r, d, *map(ctypes.byref, x))
    return tuple(v.value for v in x)


def workspace(T, hist, nkv, r, d):
    rc, de = B.kv4_layout(synth.replace(synth.CONFIGS["llama8b"], n_kv_heads=nkv, head_dim=d, max_seq=hist + T), 1)
    assert rc == 0
    return B.kv4_attn_workspace_size(de, nkv * r, 1, 1, T, hist)


def test_gpu_cases_take_the_forms_they_name():
    for form, nq, nkv, d, T, hist in G.CASES + G.BIG:
        assert G.form_of(nq, nkv, d, T, hist) == form, (nq, nkv, d, T, hist)
    taken = {(form, d) for form, _, _, d, _, _ in G.CASES}
    assert taken == {(form, d) for form in ("runs", "parts", "whole", "rows") for d in (64, 128)}


def blocks_of(T, hist, nkv, r, chunk, nblocks):
    """Per block its runs (kv head, row tile, first stage, end, slot or None), by the kernel's rules; and the stages of the
    row tiles."""
    R = T * r
    nqt = (R + 255) // 256
    st = [(hist + (min((i + 1) * 256, R) - 1) // r) // 64 + 1 for i in range(nqt)]
    out = []
    if chunk:
        units = [(q, p, -(-st[q] // chunk)) for q in reversed(range(nqt)) for p in range(-(-st[q] // chunk))]
        assert nblocks == len(units) * nkv
        for b in range(nblocks):
            q, p, n = units[b // nkv]
            s0, s1 = st[q] * p // n, st[q] * (p + 1) // n
            out.append([(b % nkv, q, s0, s1, b if n > 1 else None)])
        return out, st
    total = sum(st) * nkv
    for b in range(nblocks):
        u, u1, runs = total * b // nblocks, total * (b + 1) // nblocks, []
        while u < u1:
            hk, left = divmod(u, sum(st))
            q = 0
            while left >= st[q]:
                left -= st[q]
                q += 1
            end = min(st[q], left + u1 - u)
            runs.append((hk, q, left, end, None if (left, end) == (0, st[q]) else 2 * b + (left == 0)))
            u += end - left
        out.append(runs)
    return out, st


SEEDS = range(8)


@pytest.mark.parametrize("seed", SEEDS)
def test_every_stage_once_and_every_state_a_slot(seed):
    rng = random.Random(seed)
    forms = set()
    shapes = [(T, hist, nkv, nq // nkv, d) for _, nq, nkv, d, T, hist in G.CASES + G.BIG] if seed == 0 else []
    for _ in range(120):
        shapes.append((int(2 ** rng.uniform(0, 12)), rng.choice([0, 1, int(2 ** rng.uniform(0, 14))]), rng.randint(1, 16),
                       rng.randint(1, 8), rng.choice([64, 128])))
    for T, hist, nkv, r, d in shapes:
        single, chunk, nblocks, merge = plan(T, hist, nkv, r, d)
        if single:
            continue
        what = (T, hist, nkv, r, d, chunk, nblocks)
        blocks, st = blocks_of(T, hist, nkv, r, chunk, nblocks)
        seen, slots = {}, {}
        for b, runs in enumerate(blocks):
            for hk, q, s0, s1, slot in runs:
                assert 0 <= s0 < s1 <= st[q], what
                seen.setdefault((hk, q), []).append((s0, s1, b, slot))
                if slot is not None:
                    assert slot not in slots, what
                    slots[slot] = (hk, q)
        state = 8 * (2 + 16 * (d // 32)) * 64 * 4
        if slots:
            assert merge and (max(slots) + 1) * state <= workspace(T, hist, nkv, r, d), what
        total = sum(st) * nkv
        for hk in range(nkv):
            for q in range(len(st)):
                parts = sorted(seen[hk, q])
                assert parts[0][0] == 0 and parts[-1][1] == st[q], what
                assert all(a[1] == b[0] for a, b in zip(parts, parts[1:])), what
                # the merge's slots: in a line the blocks of the tile's first and last stage, and those between
                if chunk:
                    before = sum(-(-st[i] // chunk) for i in range(q + 1, len(st)))
                    want = [(before + p) * nkv + hk for p in range(len(parts))]
                else:
                    first = hk * sum(st) + sum(st[:q])
                    b0, b1 = (((x + 1) * nblocks - 1) // total for x in (first, first + st[q] - 1))
                    want = [2 * b + (b == b0) for b in range(b0, b1 + 1)]
                # (a tile of one part has no state, and the merge leaves it alone)
                assert [p[3] for p in parts] == (want if len(want) > 1 else [None]), what
        forms.add("runs" if not chunk else "parts" if merge else "whole")
    if seed == 0:
        assert forms == {"runs", "parts", "whole"}


@pytest.mark.parametrize("nkv,r,d", [(8, 4, 128), (4, 7, 128), (2, 7, 64), (1, 8, 128), (16, 1, 64)])
def test_up_to_four_queries_run_as_rows_of_the_decode_kernel(nkv, r, d):
    """Whatever the context: the prefill kernel would work on 256 rows.  The workspace holds that form's states too."""
    for hist in (0, 5000, 65000, 131000, 1000000, 2 ** 26):
        last = 0
        for T in range(1, 9):
            assert plan(T, hist, nkv, r, d)[0] or T > 4, (T, hist)
            n = workspace(T, hist, nkv, r, d)
            tiles = (hist + T + 31) // 32
            assert n >= max(last, min(512, T * nkv * tiles) * r * (d + 2) * 4)
            last = n
