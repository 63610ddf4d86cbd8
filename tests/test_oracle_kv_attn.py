"""Pins of oracle/kv_attn.py: closed forms, counted visibilities, trees worked out by hand."""
import math

import pytest
import torch

from oracle import kv_attn as O


def test_equal_scores_average_the_visible_values():
    v = torch.arange(12, dtype=torch.float64).reshape(6, 2)
    seen = torch.tensor([[1, 0, 0, 1, 1, 0], [0, 0, 0, 0, 0, 0]], dtype=torch.bool)
    out, tol, spread = O.attend(torch.zeros((2, 2), dtype=torch.float64), torch.ones((6, 2), dtype=torch.float64), v, seen)
    assert torch.allclose(out[0], (v[0] + v[3] + v[4]) / 3) and torch.all(out[1] == 0)
    assert torch.all(tol > 0) and torch.allclose(spread[0], 2.0 ** -16 / math.sqrt(3) / 3 * ((v[[0, 3, 4]] ** 2).sum(0) + 3 * out[0] ** 2).sqrt())


def test_two_keys_by_hand_and_a_mask():
    q, k = torch.tensor([[2.0, 0.0]], dtype=torch.float64), torch.tensor([[1.0, 5.0], [0.0, 7.0]], dtype=torch.float64)
    v, seen = torch.tensor([[1.0], [0.0]], dtype=torch.float64), torch.ones((1, 2), dtype=torch.bool)
    z = 2 / math.sqrt(2)
    assert math.isclose(O.attend(q, k, v, seen)[0].item(), 1 / (1 + math.exp(-z)))
    add = torch.tensor([-1.0, 0.5], dtype=torch.float64)
    assert math.isclose(O.attend(q, k, v, seen, add)[0].item(), 1 / (1 + math.exp(-z + 1.5)))
    add[0] = -math.inf
    assert O.attend(q, k, v, seen, add)[0].item() == 0
    assert O.attend(q, k * math.nan, v, seen & False)[0].item() == 0


@pytest.mark.parametrize("window,sinks,count", [(0, 0, 11), (0, 5, 11), (1, 0, 1), (4, 0, 4), (4, 3, 7), (4, 9, 11), (50, 2, 11), (10, 1, 11), (9, 1, 10)])
def test_visible_slots_are_counted(window, sinks, count):
    seen = O.seen_from(torch.tensor([10]), torch.arange(30), window, sinks)
    assert int(seen.sum()) == count and bool(seen[0, 10]) and not bool(seen[0, 11:].any())


def test_plan_by_hand():
    #       0 -> 1 -> 3 -> 5;  0 -> 2 -> 4;  6 is a root of its own (so is 7: its parent comes later)
    parents = [-1, 0, 0, 1, 2, 3, -7, 9]
    pos, sets = O.plan(parents, 10, 0, 0)
    assert pos == [10, 11, 11, 12, 12, 13, 10, 10]
    assert sets == [{0}, {0, 1}, {0, 2}, {0, 1, 3}, {0, 2, 4}, {0, 1, 3, 5}, {6}, {7}]
    assert O.plan(parents, 10, 2, 0)[1] == [{0}, {0, 1}, {0, 2}, {1, 3}, {2, 4}, {3, 5}, {6}, {7}]
    assert O.plan(parents, 10, 2, 11)[1] == [{0}, {0, 1}, {0, 2}, {0, 1, 3}, {0, 2, 4}, {0, 3, 5}, {6}, {7}]
    assert O.plan(parents, -1, 0, 0)[0] == [0, 1, 1, 2, 2, 3, 0, 0]
    assert O.words([{0, 63}, {64}, {1, 65}], 66) == [[1 - (1 << 63), 0], [0, 1], [2, 2]]


def test_accept_by_hand():
    parents, tokens = [-1, 0, 0, 1, 2, 3, 2], [5, 7, 8, 9, 4, 6, 4]
    assert O.accept(parents, tokens, [8, 0, 4, 0, 1, 2, 3]) == ([0, 2, 4], 1)      # (4 before 6: the lower index)
    assert O.accept(parents, tokens, [7, 9, 0, 6, 1, 2, 3]) == ([0, 1, 3, 5], 2)
    assert O.accept(parents, tokens, [6, 9, 4, 6, 1, 2, 3]) == ([0], 6)            # (6 hangs below node 3 only)
