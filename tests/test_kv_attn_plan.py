"""How calls of attention over the bf16 cache are cut up, on the host: every plan stays inside what the launches and the
workspace allow, and the sizes that a caller asks for cover the plan of every smaller call."""
import ctypes
import os
import random

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2607_15865_amd", "libw4layer.so")

if not os.path.exists(LIB):
    from paper_2607_15865_amd import build as _b
    _b.build()

from paper_2607_15865_amd import binding  # noqa: E402


def plan(B, N, nkv, r, d, max_ctx, window, sinks, tree):
    out = [ctypes.c_int() for _ in range(3)] + [ctypes.c_size_t() for _ in range(2)]
    binding._lib.w4_kv_attn_plan(B, N, nkv, r, d, max_ctx, window, sinks, tree, *[ctypes.byref(x) for x in out])
    p = dict(zip(("kind", "nsplit", "whole", "part", "bound"), [x.value for x in out]))
    p["few"], p["rows"] = p["kind"] == 1, {0: 256, 1: 16, 2: 128}[p.pop("kind")]
    return p


def shapes(seed, count):
    rng = random.Random(seed)
    log = lambda a, b: int(a * (b / a) ** rng.random())
    for _ in range(count):
        kind = rng.choice(["decode", "prefill", "tree"])
        B, N = {"decode": (log(1, 65535), 1), "prefill": (1, log(1, 200000)), "tree": (log(1, 2000), log(1, 257))}[kind]
        yield (B, min(N, 256) if kind == "tree" else N, log(1, 65), log(1, 65), rng.choice([64, 128]), log(1, 1 << rng.randint(1, 26)),
               rng.choice([0, log(1, 1 << 27)]), rng.choice([0, log(1, 1 << 27)]), kind == "tree")


@pytest.mark.parametrize("seed", range(4))
def test_plans_fit_launches_and_workspaces(seed):
    for s in shapes(seed, 400):
        B, N, nkv, r, d, max_ctx, window, sinks, tree = s
        p = plan(*s)
        R = N * r
        assert p["nsplit"] >= 1 and p["part"] <= p["bound"], s
        if p["few"]:
            assert p["whole"] == 0
            tiles = -(-R // 16)
            assert p["nsplit"] <= 65535 and nkv * tiles < 2 ** 31
            assert p["nsplit"] == 1 or B * nkv * tiles * p["nsplit"] <= 512, s
            assert p["part"] == (B * nkv * R * p["nsplit"] * (d + 2) * 4 if p["nsplit"] > 1 else 0)
            if p["nsplit"] > 1:              # (the merge's grid)
                assert R <= 65535
        else:
            blocks = B * nkv * -(-R // p["rows"])
            rest = blocks - p["whole"]
            assert 0 <= p["whole"] <= blocks and (p["nsplit"] > 1) == (rest > 0) and rest * p["nsplit"] <= 512, s
            assert p["part"] == rest * p["nsplit"] * p["rows"] * (d + 4) * 4


@pytest.mark.parametrize("seed", range(4))
def test_sizes_cover_smaller_calls(seed):
    rng = random.Random(seed + 100)
    for s in shapes(seed + 50, 200):
        B, N, nkv, r, d, max_ctx, window, sinks, tree = s
        bound = plan(*s)["bound"]
        for _ in range(5):
            b, n, c = (rng.randint(1, x) for x in (B, N, max_ctx))
            w, k = rng.choice([0, rng.randint(1, max_ctx + 1)]), rng.randint(0, 100)
            assert plan(b, n, nkv, r, d, c, w, k, tree)["part"] <= bound, (s, b, n, c, w, k)


def test_single_queries_and_long_prefills():
    """A single query's rows are few, a long prompt's many, those of many sequences' drafts between; a window bounds the work however long the context is."""
    assert plan(1, 1, 8, 4, 128, 100000, 0, 0, False)["few"] and plan(1, 4000, 8, 4, 128, 0, 0, 0, False)["rows"] == 256
    assert plan(16, 13, 8, 4, 128, 4000, 0, 0, True)["rows"] == 128
    assert plan(1, 1, 8, 4, 128, 1 << 26, 256, 4, False) == plan(1, 1, 8, 4, 128, 1 << 20, 256, 4, False) | dict(
        bound=plan(1, 1, 8, 4, 128, 1 << 26, 256, 4, False)["bound"])
