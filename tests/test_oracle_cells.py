"""Pins of oracle/cells.py: closed forms, hand-made states, and what must hold whatever the calls."""
import math

import numpy as np
import pytest

from oracle import cells as O
from oracle import serving as V
from tests.cells import random_state


def test_rotation_closed_forms():
    x = np.zeros((3, 1, 4))
    x[:, 0] = [1.0, 2.0, 3.0, 4.0]
    r = O.rotate_heads(x, [0, 1, -1], [math.pi / 2, 0.0], eps=None, weight=None, interleaved=False)["y"][:, 0]
    assert np.allclose(r[0], [1, 2, 3, 4]) and np.allclose(r[1], [-3, 2, 1, 4]) and np.allclose(r[2], [3, 2, -1, 4])
    r = O.rotate_heads(x, [0, 1, -1], [math.pi / 2], eps=None, weight=None, interleaved=True)["y"][:, 0]
    assert np.allclose(r[1], [-2, 1, 3, 4])                      # the last two columns do not turn
    r = O.rotate_heads(x, None, None, eps=0.0, weight=[1, 1, 1, 2], interleaved=False)["y"][:, 0]
    assert np.allclose(r[0], np.array([1, 2, 3, 8]) / math.sqrt(7.5))
    # products of turned rows depend on the distance alone
    rng = np.random.default_rng(0)
    a, b = rng.standard_normal(8), rng.standard_normal(8)
    f = rng.random(4)
    turn = lambda v, p: O.rotate_heads(v[None, None], [p], f, eps=None, weight=None, interleaved=False)["y"][0, 0]
    assert np.allclose(turn(a, 7) @ turn(b, 3), turn(a, 104) @ turn(b, 100))


def test_scores_are_the_attention_weights():
    """Over every token the scores of the rows that see something sum to their share of the rows."""
    rng = np.random.default_rng(1)
    s = random_state(rng, [37, 1, 16, 2], 16, 32, 20)
    q = rng.standard_normal((2, 3, 4, 20))
    att = V.cache_attention(q, s, s["table"], s["lens"], None)
    r = O.cache_scores(q, s, s["table"], s["lens"], att["lse"], None, 60)["scores"]
    for c, n in enumerate([37, 1, 16, 2]):
        rows = sum(1 for t in range(3) if n - (2 - t) > 0)
        assert np.isclose(np.nansum(r[c]), rows / 3) and np.isnan(r[c, n:]).all() and not np.isnan(r[c, :n]).any()


def test_selection_by_hand():
    x = np.array([[1.0, 5.0, 5.0, math.nan, 0.0, 5.0, 9.0]])
    sel = lambda k, r, n=7: O.cache_select(x, [n], [k], r)[0]
    assert sel(0, 2) == [] and sel(1, 2) == [6] and sel(2, 2) == [5, 6] and sel(3, 2) == [3, 5, 6]
    assert sel(4, 2) == [1, 3, 5, 6] and sel(3, 0) == [1, 3, 6] and sel(9, 1) == list(range(7)) and sel(2, 1, 3) == [1, 2]


def test_fork_release_by_hand():
    rng = np.random.default_rng(2)
    s = random_state(rng, [40, 0, 0, 0], 16, 32, 8, W=3, n_blocks=8)
    row = s["table"][0].tolist()
    free = s["free_list"][:s["n_free"]].tolist()
    up = O.fork(s, [0, 0, 0], [1, 2, 1])                       # the third pair names cell 1 again
    assert up["refused"] == 1 and up["lens"].tolist() == [40, 40, 40, 0]
    assert up["table"][1].tolist() == row[:2] + [free[-1]] and up["table"][2].tolist() == row[:2] + [free[-2]]
    assert up["shared"][row[0]] == 2 and up["shared"][row[2]] == 0
    assert np.array_equal(up["k"][free[-1]], s["k"][row[2]])
    O.invariants(up)
    # cut into a block that others hold: a copy of it; a cell that ends leaves the others theirs
    down = O.release(up, [20, 0, 99, 0])
    O.invariants(down)
    assert down["lens"].tolist() == [20, 0, 40, 0] and down["table"][0, 0] == row[0] and down["table"][0, 1] == free[-3]
    assert down["shared"][row[0]] == 1 and down["shared"][row[1]] == 0 and down["table"][2, 1] == row[1]
    end = O.release(down, [0, 0, 0, 0])
    O.invariants(end)
    assert end["n_free"] == 8 and not end["shared"].any()


def test_compaction_by_hand():
    rng = np.random.default_rng(3)
    s = random_state(rng, [40, 30], 16, 32, 8, W=3, n_blocks=8)
    before, _, _ = V.cache_rows(s, s["table"][0], 40)
    pos = list(range(16)) + [18, 33, 39]
    r = O.compact(s, [0, 19, 19], pos)
    O.invariants(r)
    assert r["refused"] == 0 and r["lens"].tolist() == [19, 0] and r["table"][0, 0] == s["table"][0, 0]
    after, _, _ = V.cache_rows(r, r["table"][0], 19)
    assert np.array_equal(after[:16], before[:16])
    tiny = 2.0 ** (int(r["k_exp"][r["table"][0, 1]]) - 127 - 10)  # half of the least value
    assert np.all(np.abs(after[16:] - before[[18, 33, 39]]) <= np.maximum(np.abs(after[16:]) * 2.0 ** -4, tiny))
    for bad in ([5, 5], [3, 2], [39, 40], [-1, 3]):
        x = O.compact(s, [0, 2], bad)
        assert x["refused"] == 1 and np.array_equal(x["table"], s["table"]) and x["lens"].tolist() == [40, 30]
    assert O.compact(s, [0, 2, 1], [1, 2])["refused"] == 2


@pytest.mark.parametrize("seed", range(6))
def test_any_calls_keep_every_block_once(seed):
    rng = np.random.default_rng(100 + seed)
    C, W, bs = 9, 5, 16
    s = random_state(rng, [int(rng.integers(0, 80)) if c < 4 else 0 for c in range(C)], bs, 32, 4, W=W, n_blocks=24)
    for _ in range(12):
        what = rng.integers(0, 3)
        if what == 0:
            P = int(rng.integers(1, 5))
            s = O.fork(s, rng.integers(-1, C + 1, P), rng.integers(-1, C + 1, P), rng.integers(-1, 90, P))
        elif what == 1:
            s = O.release(s, np.where(rng.random(C) < 0.5, rng.integers(0, 80, C), 99))
        else:
            pos, off = [], [0]
            for c in range(C):
                n = int(s["lens"][c])
                pos += sorted(rng.permutation(n)[:int(rng.integers(0, n + 1))].tolist())
                off.append(len(pos))
            s = O.compact(s, off, pos)
        O.invariants(s)
