"""CPU oracle of the serving operators: prompt attention, block tables, the
8-bit cache's store and the attention over it.

TEST INFRASTRUCTURE ONLY, like oracle/fw_oracle.py: plain float64 and integer
transcriptions of the definitions in include/fw.h, sharing no code with the
HIP library.  Beside each attention result it gives what rounding can do to
it: sum_j p_j |v_j| per output, and sum_c |q_c k_jc| (its largest per row),
from which the tests derive their tolerances.
"""
from __future__ import annotations

import math
from typing import Dict, Optional, Sequence

import numpy as np


def attend(q: np.ndarray, k: np.ndarray, v: np.ndarray, scale: float, seen: Sequence[int]) -> Dict[str, np.ndarray]:
    """Rows q [R][d] over keys k [n][d], of which row r sees the first seen[r].
    Definition 2.1's dense output per row, and log sum exp of the logits."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    R, d = q.shape
    o, abs_o = np.zeros((R, v.shape[1])), np.zeros((R, v.shape[1]))
    lse, dots = np.full(R, -np.inf), np.zeros(R)
    for r in range(R):
        n = max(0, min(int(seen[r]), k.shape[0]))
        if n == 0:
            continue
        with np.errstate(invalid="ignore", over="ignore"):
            z = scale * (k[:n] @ q[r])
            m = np.max(z)
            e = np.exp(z - m)
            p = e / e.sum()
            o[r] = p @ v[:n]
            abs_o[r] = p @ np.abs(v[:n])
            lse[r] = m + math.log(e.sum()) if np.isfinite(m) else m
            dots[r] = abs(scale) * np.max(np.abs(k[:n]) @ np.abs(q[r]))
    return dict(o=o, lse=lse, abs_o=abs_o, dots=dots)


def prompt_attention(q, k, v, cu_q, cu_k, scale: Optional[np.ndarray], causal: bool) -> Dict[str, np.ndarray]:
    """q [Tq][Hq][d], k and v [Tk][Hkv][d]; NaN where no sequence has a row."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    Tq, Hq, d = q.shape
    Hkv = k.shape[1]
    out = dict(o=np.full((Tq, Hq, d), np.nan), lse=np.full((Tq, Hq), np.nan), abs_o=np.zeros((Tq, Hq, d)),
               dots=np.zeros((Tq, Hq)))
    for b in range(len(cu_q) - 1):
        a0, a1, k0, k1 = (int(x) for x in (cu_q[b], cu_q[b + 1], cu_k[b], cu_k[b + 1]))
        Lq, Lk = a1 - a0, k1 - k0
        seen = [i + Lk - Lq + 1 if causal else Lk for i in range(Lq)]
        for h in range(Hq):
            g = h // (Hq // Hkv)
            r = attend(q[a0:a1, h], k[k0:k1, g], v[k0:k1, g], 1 / math.sqrt(d) if scale is None else float(scale[g]), seen)
            for key in out:
                out[key][a0:a1, h] = r[key]
    return out


# ----------------------------------------------------------------------------
# block tables: the cells one after the other
# ----------------------------------------------------------------------------


def block_tables(old, new, table, free_list, n_free: int, block_size: int, n_slots: int) -> Dict[str, object]:
    """Copies of table, free_list and n_free after the call, with the slots (None: not written), offsets, lengths and
    the number of refused cells."""
    table, stack = np.array(table), np.array(free_list)
    C, W = table.shape
    nb = lambda n: -(-n // block_size)
    old, new = [max(0, int(x)) for x in old], [max(0, int(x)) for x in new]
    # what comes back, the first block given back on top of the stack
    back = []
    for c in range(C):
        if nb(new[c]) <= W:
            for j in range(nb(new[c]), nb(old[c])):
                back.append(int(table[c, j]))
                table[c, j] = -1
    for i, b in enumerate(reversed(back)):
        stack[n_free + i] = b
    top = n_free + len(back)
    asked = taken = refused = 0
    slots, offsets, lens = [], [0], []
    for c in range(C):
        fits = nb(new[c]) <= W
        need = max(0, nb(new[c]) - nb(old[c])) if fits else 0
        asked += need
        ok = fits and (need == 0 or asked <= top)
        if ok:
            for j in range(need):
                table[c, nb(old[c]) + j] = stack[top - taken - 1]
                taken += 1
        refused += not ok
        lens.append(new[c] if ok else old[c])
        for pos in range(old[c], new[c]):
            slots.append(int(table[c, pos // block_size]) * block_size + pos % block_size if ok else -1)
        offsets.append(len(slots))
    return dict(table=table, free_list=stack, n_free=top - taken, slots=(slots + [None] * n_slots)[:n_slots],
                offsets=np.array(offsets), lens=np.array(lens), refused=refused)


# ----------------------------------------------------------------------------
# the 8-bit cache
# ----------------------------------------------------------------------------


def _e4m3_table() -> np.ndarray:
    """The value of each code: sign, 4 exponent bits of bias 7, 3 mantissa bits; 0x7f and 0xff are NaN."""
    v = np.zeros(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = math.nan if (e, m) == (15, 7) else (1 + m / 8) * 2.0 ** (e - 7) if e else m / 8 * 2.0 ** -6
        v[c] = -x if c & 128 else x
    return v


E4M3 = _e4m3_table()


def e4m3_code(x: float) -> int:
    """The code nearest to x, |x| <= 448, ties to the even code; 0x7f for what is not finite."""
    if not math.isfinite(x):
        return 0x7F
    a = abs(x)
    lo = int(np.searchsorted(E4M3[:127], a, side="right")) - 1
    if lo < 126 and E4M3[lo] != a:
        mid = (E4M3[lo] + E4M3[lo + 1]) / 2
        if a > mid or (a == mid and lo % 2 == 1):
            lo += 1
    return lo | (128 if math.copysign(1.0, x) < 0 else 0)


def scale_byte(values) -> int:
    """Least e in 1 .. 253 with |x| <= 448 * 2^(e - 127) for every finite x."""
    a = [abs(float(x)) for x in np.ravel(values) if math.isfinite(x)]
    top, e = max(a, default=0.0), 1
    while e < 253 and top > math.ldexp(448.0, e - 127):
        e += 1
    return e


def cache_store(cache: Dict[str, np.ndarray], k, v, slots) -> Dict[str, np.ndarray]:
    """cache: k [n][bs][dp], v [n][dp][bs], k_exp, v_exp [n] (uint8), d.  Copies of the buffers after the call."""
    c = {key: np.array(x) for key, x in cache.items() if key != "d"}
    n, bs, _ = c["k"].shape
    d = cache["d"]
    i, N = 0, len(slots)
    while i < N:
        s = int(slots[i])
        if not 0 <= s < n * bs:
            i += 1
            continue
        j = i + 1
        while j < N and int(slots[j]) == s + j - i and (s + j - i) % bs != 0:
            j += 1
        b, off = divmod(s, bs)
        for name, x in (("k", k), ("v", v)):
            x = np.asarray(x, np.float64)[i:j]
            codes = c[name][b] if name == "k" else c[name][b].T     # [token][dp]
            e = scale_byte(x)
            if off:
                was = min(int(c[name + "_exp"][b]), 253)
                e = max(e, was)
                if e > was:
                    for t in range(off):
                        for col in range(d):
                            codes[t, col] = e4m3_code(math.ldexp(E4M3[codes[t, col]], was - e))
            c[name + "_exp"][b] = e
            for t in range(j - i):
                for col in range(d):
                    codes[off + t, col] = e4m3_code(math.ldexp(x[t, col], 127 - e))
        i = j
    return c


def cache_rows(cache: Dict[str, np.ndarray], blocks: Sequence[int], length: int):
    """Keys and values [length][d] of a cell, and which of its tokens lie in a valid block."""
    n, bs, _ = cache["k"].shape
    d = cache["d"]
    K, V, ok = np.zeros((length, d)), np.zeros((length, d)), np.zeros(length, bool)
    for t in range(length):
        b = int(blocks[t // bs])
        if 0 <= b < n:
            ok[t] = True
            K[t] = E4M3[cache["k"][b, t % bs, :d]] * 2.0 ** (int(cache["k_exp"][b]) - 127)
            V[t] = E4M3[cache["v"][b, :d, t % bs]] * 2.0 ** (int(cache["v_exp"][b]) - 127)
    return K, V, ok


def cache_attention(q, cache: Dict[str, np.ndarray], table, lens, scale: Optional[np.ndarray]) -> Dict[str, np.ndarray]:
    """q [S][T][Hq][d], table [S*Hkv][W], lens [S*Hkv]."""
    q = np.asarray(q, np.float64)
    S, T, Hq, d = q.shape
    table = np.asarray(table)
    Hkv, bs = table.shape[0] // S, cache["k"].shape[1]
    G = Hq // Hkv
    out = dict(o=np.zeros((S, T, Hq, d)), lse=np.zeros((S, T, Hq)), abs_o=np.zeros((S, T, Hq, d)),
               dots=np.zeros((S, T, Hq)))
    for c in range(S * Hkv):
        s, h = divmod(c, Hkv)
        n = max(0, min(int(lens[c]), table.shape[1] * bs))
        K, V, ok = cache_rows(cache, table[c], n)
        for t in range(T):
            upto = max(0, n - (T - 1 - t))
            use = ok[:upto]
            r = attend(q[s, t, h * G:(h + 1) * G], K[:upto][use], V[:upto][use],
                       1 / math.sqrt(d) if scale is None else float(scale[h]), [int(use.sum())] * G)
            for key in out:
                out[key][s, t, h * G:(h + 1) * G] = r[key]
    return out
