"""CPU oracle of the operators around the cache: rotation of heads, scores of
cached tokens, selection, and cells that share blocks (fork, release,
compaction).

TEST INFRASTRUCTURE ONLY, like oracle/serving.py: plain float64 and integer
transcriptions of the definitions in include/fw.h, one row, token or cell after
the other, sharing no code with the HIP library.
"""
from __future__ import annotations

import math
from typing import Dict, Optional, Sequence

import numpy as np

from oracle.serving import E4M3, cache_rows, e4m3_code, scale_byte


def rotate_heads(x, pos, freq, *, eps: Optional[float], weight, interleaved: bool) -> Dict[str, np.ndarray]:
    """Rows x [T][H][d].  `mag` is |u| + |v| of each turned pair (|x| of a column that does not turn), after the norm."""
    x = np.asarray(x, np.float64)
    d = x.shape[2]
    if eps is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
        if weight is not None:
            x = x * np.asarray(weight, np.float64)
    y, mag = x.copy(), np.abs(x)
    half = 0 if freq is None else len(freq)
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        for t in range(x.shape[0]):
            angle = float(pos[t]) * float(freq[i])
            c, s = math.cos(angle), math.sin(angle)
            y[t, :, a] = x[t, :, a] * c - x[t, :, b] * s
            y[t, :, b] = x[t, :, b] * c + x[t, :, a] * s
        mag[:, :, a] = mag[:, :, b] = np.abs(x[:, :, a]) + np.abs(x[:, :, b])
    return dict(y=y, mag=mag)


def cache_scores(q, cache, table, lens, lse, scale, n: int) -> Dict[str, np.ndarray]:
    """q [S][T][Hq][d]: the mean weight [S*Hkv][n] of every token (NaN behind a cell's end), and `err`, the mean over the
    rows of each weight times what one unit of rounding does to it: (d + 4) sum |q_c k_c| |scale| + |lse| + 2."""
    q = np.asarray(q, np.float64)
    S, T, Hq, d = q.shape
    table = np.asarray(table)
    Hkv, bs = table.shape[0] // S, cache["k"].shape[1]
    G = Hq // Hkv
    w, err = np.full((S * Hkv, n), np.nan), np.zeros((S * Hkv, n))
    for c in range(S * Hkv):
        s, h = divmod(c, Hkv)
        length = max(0, min(int(lens[c]), table.shape[1] * bs))
        K, _, ok = cache_rows(cache, table[c], length)
        f = 1 / math.sqrt(d) if scale is None else float(scale[h])
        total, bound = np.zeros(length), np.zeros(length)
        for t in range(T):
            seen = max(0, length - (T - 1 - t))
            for g in range(G):
                row, l = q[s, t, h * G + g], float(lse[s, t, h * G + g])
                with np.errstate(invalid="ignore", over="ignore"):
                    e = np.where(ok[:seen], np.exp(f * (K[:seen] @ row) - l), 0.0)
                    total[:seen] += e
                    bound[:seen] += e * ((d + 4) * abs(f) * (np.abs(K[:seen]) @ np.abs(row)) + abs(l) + 2)
        m = min(length, n)
        w[c, :m], err[c, :m] = total[:m] / (T * G), bound[:m] / (T * G)
    return dict(scores=w, err=err)


def cache_select(scores, lens, keep, recent: int):
    """Kept positions of every cell, ascending."""
    out = []
    for row, n, k in zip(scores, lens, keep):
        n = max(0, min(int(n), len(row)))
        k = max(0, min(int(k), n))
        r = min(recent, k)
        rank = sorted(range(n - r), key=lambda j: (-math.inf if math.isnan(row[j]) else -float(row[j]), not math.isnan(row[j]), j))
        out.append(sorted(rank[:k - r]) + list(range(n - r, n)))
    return out


# ----------------------------------------------------------------------------
# cells that share blocks.  A state holds table [C][W], lens [C], free_list,
# n_free, shared [n_blocks], and the cache's k, v, k_exp, v_exp and d.
# ----------------------------------------------------------------------------

ARRAYS = ("table", "lens", "free_list", "shared", "k", "v", "k_exp", "v_exp")


def copy_state(s):
    return dict(s, **{key: np.array(s[key]) for key in ARRAYS})


def _blocks(n: int, bs: int) -> int:
    return -(-n // bs)


def _copy(s, a: int, b: int):
    for key in ("k", "v", "k_exp", "v_exp"):
        s[key][b] = s[key][a]


class _Stack:
    """Takes from the top of the stack as it was, and gives back in ascending order at the end."""

    def __init__(self, s):
        self.s, self.top, self.asked, self.taken, self.owners = s, s["n_free"], 0, 0, {}

    def ask(self, n: int) -> Optional[list]:
        first, self.asked = self.asked, self.asked + n
        if n and self.asked > self.top:
            return None
        got = [int(self.s["free_list"][self.top - 1 - i]) for i in range(first, first + n)]
        if n:
            self.taken = self.asked
        return got

    def leave(self, b: int):
        self.owners[b] = self.owners.get(b, int(self.s["shared"][b]) + 1) - 1

    def done(self):
        s, left = self.s, self.top - self.taken
        for b in sorted(self.owners):
            if self.owners[b] == 0:
                s["free_list"][left] = b
                left += 1
            s["shared"][b] = max(0, self.owners[b] - 1)
        s["n_free"] = left


def fork(s, src, dst, length=None) -> Dict[str, object]:
    was, s = s, copy_state(s)
    bs, C = s["k"].shape[1], s["table"].shape[0]
    stack, refused, named = _Stack(s), 0, set()
    for p, (a, b) in enumerate(zip(src, dst)):
        a, b = int(a), int(b)
        first = b not in named
        named.add(b)
        if not (0 <= a < C and 0 <= b < C and first and was["lens"][b] == 0):
            refused += 1
            continue
        n = int(was["lens"][a]) if length is None else max(0, min(int(length[p]), int(was["lens"][a])))
        got = stack.ask(1 if n % bs else 0)
        if got is None:
            refused += 1
            continue
        for j in range(n // bs):
            s["table"][b, j] = was["table"][a, j]
            s["shared"][was["table"][a, j]] += 1
        if n % bs:
            s["table"][b, n // bs] = got[0]
            _copy(s, was["table"][a, n // bs], got[0])
        s["lens"][b] = n
    s["n_free"] = stack.top - stack.taken
    return dict(s, refused=refused)


def release(s, new_len) -> Dict[str, object]:
    was, s = s, copy_state(s)
    bs = s["k"].shape[1]
    stack, refused = _Stack(s), 0
    for c in range(s["table"].shape[0]):
        old = int(was["lens"][c])
        n = min(max(int(new_len[c]), 0), old)
        last = int(was["table"][c, n // bs]) if n % bs else -1
        got = stack.ask(1 if n % bs and was["shared"][last] > 0 else 0)
        if got is None:
            refused += 1
            continue
        for j in range(_blocks(n, bs), _blocks(old, bs)):
            stack.leave(int(was["table"][c, j]))
            s["table"][c, j] = -1
        if got:
            stack.leave(last)
            s["table"][c, n // bs] = got[0]
            _copy(s, last, got[0])
        s["lens"][c] = n
    stack.done()
    return dict(s, refused=refused)


def compact(s, offsets, kept_pos, which=None) -> Dict[str, object]:
    was, s = s, copy_state(s)
    bs, C = s["k"].shape[1], s["table"].shape[0]
    P, N = len(offsets) - 1, len(kept_pos)
    down = any(offsets[i] > offsets[i + 1] for i in range(P))
    stack, refused, named = _Stack(s), 0, set()
    for p in range(P):
        c = p if which is None else int(which[p])
        first = c not in named
        named.add(c)
        a, e = int(offsets[p]), int(offsets[p + 1])
        ok = not down and first and 0 <= c < C and 0 <= a and e <= N
        pos = [int(x) for x in kept_pos[a:e]] if ok else []
        old = int(was["lens"][c]) if ok else 0
        ok = ok and all(x > y for x, y in zip(pos, [-1] + pos)) and (not pos or pos[-1] < old)
        if not ok:
            refused += 1
            continue
        n = len(pos)
        change = []
        for j in range(_blocks(n, bs)):
            part = pos[j * bs:(j + 1) * bs]
            stays = part == list(range(j * bs, j * bs + len(part)))
            if not stays or (len(part) < bs and was["shared"][was["table"][c, j]] > 0):
                change.append(j)
        take = [j for j in change if was["shared"][was["table"][c, j]] > 0]
        got = stack.ask(len(take))
        if got is None:
            refused += 1
            continue
        to = dict(zip(take, got))
        for j in change:
            b = int(was["table"][c, j])
            if j in to:
                stack.leave(b)
                s["table"][c, j] = b = to[j]
            part = pos[j * bs:(j + 1) * bs]
            for key, exp in (("k", "k_exp"), ("v", "v_exp")):
                rows = []
                for x in part:
                    at = int(was["table"][c, x // bs])
                    codes = was[key][at, x % bs] if key == "k" else was[key][at, :, x % bs]
                    rows.append(E4M3[codes] * 2.0 ** (int(was[exp][at]) - 127))
                top = scale_byte(rows)
                s[exp][b] = top
                for t, row in enumerate(rows):
                    new = [e4m3_code(math.ldexp(float(x), 127 - top)) for x in row]
                    if key == "k":
                        s[key][b, t] = new
                    else:
                        s[key][b, :, t] = new
        for j in range(_blocks(n, bs), _blocks(old, bs)):
            stack.leave(int(was["table"][c, j]))
            s["table"][c, j] = -1
        s["lens"][c] = n
    stack.done()
    return dict(s, refused=refused)


def invariants(s, holders: Sequence[int] = ()) -> None:
    """Every block is free once or held by 1 + shared cells; no block twice in a cell."""
    bs, n = s["k"].shape[1], len(s["shared"])
    held = np.zeros(n, int)
    for c in range(s["table"].shape[0]):
        row = [int(b) for b in s["table"][c, :_blocks(int(s["lens"][c]), bs)]]
        assert len(set(row)) == len(row) and all(0 <= b < n for b in row), (c, row)
        assert np.all(s["table"][c, len(row):] == -1), c
        held[row] += 1
    free = [int(b) for b in s["free_list"][:s["n_free"]]]
    assert len(set(free)) == len(free)
    assert np.array_equal(np.sort(np.concatenate([free, np.flatnonzero(held)]).astype(int)), np.arange(n))
    assert np.array_equal(np.maximum(held - 1, 0), s["shared"])
