"""Pins of the serving oracle against closed forms, torch and brute force."""
import math

import numpy as np
import pytest
import torch

from oracle import serving as O


def test_codes_match_the_format():
    """Every code's value and every rounding, against torch's float8_e4m3fn."""
    t = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(np.isnan(t), np.isnan(O.E4M3))
    assert np.array_equal(t[~np.isnan(t)], O.E4M3[~np.isnan(t)])
    rng = np.random.default_rng(0)
    mids = (O.E4M3[:126] + O.E4M3[1:127]) / 2
    x = np.concatenate([mids, -mids, O.E4M3[:127], rng.standard_normal(500) * 50, rng.standard_normal(200) * 2 ** -9])
    x = np.clip(x, -448, 448)
    got = np.array([O.e4m3_code(float(y)) for y in x], np.uint8)
    want = torch.tensor(x).to(torch.float32).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(got, want)


@pytest.mark.parametrize("top,e", [(448.0, 127), (448.0000305, 128), (896.0, 128), (1.0, 119), (1.75, 119), (1.7500001, 120),
                                   (0.0, 1), (2.0 ** -130, 1), (3.3e38, 247)])
def test_scale_byte(top, e):
    assert O.scale_byte([top, -top / 2, math.inf, math.nan]) == e


def test_attend_closed_forms():
    # equal logits: the mean and log n; one key: its value; none: zero and -inf
    v = np.arange(12.0).reshape(4, 3)
    r = O.attend(np.zeros((3, 2)), np.ones((4, 2)), v, 1.0, [4, 1, 0])
    assert np.allclose(r["o"][0], v.mean(0)) and np.allclose(r["lse"][0], math.log(4))
    assert np.array_equal(r["o"][1], v[0]) and r["lse"][1] == 0
    assert np.array_equal(r["o"][2], np.zeros(3)) and r["lse"][2] == -math.inf
    # weights 1 : 3 by a logit difference of log 3
    r = O.attend(np.ones((1, 1)), np.array([[0.0], [math.log(3)]]), np.array([[0.0], [1.0]]), 1.0, [2])
    assert np.allclose(r["o"], 0.75) and np.allclose(r["lse"], math.log(4))


@pytest.mark.parametrize("causal", [True, False])
def test_prompt_matches_a_masked_softmax(causal):
    rng = np.random.default_rng(1)
    lq, lk = [3, 0, 5, 4], [3, 2, 9, 2]
    cu_q, cu_k = np.cumsum([0] + lq), np.cumsum([0] + lk)
    q, k, v = (rng.standard_normal(s) for s in ((12, 4, 6), (16, 2, 6), (16, 2, 6)))
    r = O.prompt_attention(q, k, v, cu_q, cu_k, None, causal)
    for b in range(4):
        for h in range(4):
            Q, K, V = q[cu_q[b]:cu_q[b + 1], h], k[cu_k[b]:cu_k[b + 1], h // 2], v[cu_k[b]:cu_k[b + 1], h // 2]
            z = torch.tensor(Q @ K.T / math.sqrt(6))
            if causal:
                i, j = np.arange(lq[b])[:, None], np.arange(lk[b])
                z = z.masked_fill(torch.tensor(j > i + lk[b] - lq[b]), -math.inf)
            o = torch.nan_to_num(torch.softmax(z, 1), nan=0.0).numpy() @ V
            assert np.allclose(r["o"][cu_q[b]:cu_q[b + 1], h], o, atol=1e-12)
            assert np.allclose(r["lse"][cu_q[b]:cu_q[b + 1], h], torch.logsumexp(z, 1).numpy(), atol=1e-12)


def test_block_tables_by_hand():
    t = np.full((3, 3), -1)
    t[0, 0], t[1, :2] = 7, [4, 5]
    f = np.array([0, 1, 2, 3, 9, 9, 9, 9])
    # cell 0 grows into its block and one more, cell 1 gives one back, cell 2 does not fit its row
    r = O.block_tables([10, 20, 0], [30, 16, 99], t, f, 4, 16, 200)
    assert r["table"].tolist() == [[7, 5, -1], [4, -1, -1], [-1, -1, -1]]   # the block that came back goes out first
    assert r["n_free"] == 4 and r["free_list"][:5].tolist() == [0, 1, 2, 3, 5]
    assert r["lens"].tolist() == [30, 16, 0] and r["refused"] == 1
    assert r["offsets"].tolist() == [0, 20, 20, 119]
    assert r["slots"][:20] == [7 * 16 + i for i in range(10, 16)] + [5 * 16 + i for i in range(14)]
    assert r["slots"][20:119] == [-1] * 99 and r["slots"][119:] == [None] * 81


def test_block_tables_refuse_only_cells_that_need_blocks():
    """After the stack has run out, a cell that shrinks, stays, or grows within its last block is served."""
    t = np.full((5, 4), -1)
    t[0, 0], t[1, :3], t[2, 0], t[3, :2], t[4, 0] = 0, [1, 2, 3], 4, [5, 6], 7
    f = np.array([8, 9] + [-7] * 8)
    # 2 free and 2 given back; cell 0 wants 3 more, cell 2 another 3 (refused), cell 4 the block that is left (refused)
    r = O.block_tables([16, 40, 10, 20, 16], [64, 5, 64, 25, 17], t, f, 2, 16, 200)
    assert r["lens"].tolist() == [64, 5, 10, 25, 16] and r["refused"] == 2
    assert r["table"].tolist() == [[0, 2, 3, 9], [1, -1, -1, -1], [4, -1, -1, -1], [5, 6, -1, -1], [7, -1, -1, -1]]
    assert r["n_free"] == 1 and r["free_list"][0] == 8
    assert r["offsets"].tolist() == [0, 48, 48, 102, 107, 108]
    assert r["slots"][48:102] == [-1] * 54 and r["slots"][102:107] == [6 * 16 + i for i in range(4, 9)]
    assert r["slots"][107] == -1
    # shrinking behind the refused cell: what it gives back leaves its table and its length together
    t[3, 2:] = [10, 11]
    r = O.block_tables([16, 5, 10, 60], [16, 5, 99, 20], t[:4], np.array([8] + [-7] * 11), 1, 16, 0)
    assert r["refused"] == 1 and r["lens"].tolist() == [16, 5, 10, 20] and r["table"][3].tolist() == [5, 6, -1, -1]
    assert r["n_free"] == 3 and r["free_list"][:3].tolist() == [8, 11, 10]
    t[3, 2:] = [10, 11]
    r = O.block_tables([16, 5, 10, 60], [64, 5, 64, 20], t[:4], np.array([8] + [-7] * 11), 1, 16, 0)
    assert r["refused"] == 1 and r["lens"].tolist() == [64, 5, 10, 20] and r["n_free"] == 0
    assert r["table"].tolist() == [[0, 10, 11, 8], [1, 2, 3, -1], [4, -1, -1, -1], [5, 6, -1, -1]]


def test_block_tables_return_restores_the_stack():
    rng = np.random.default_rng(2)
    old, new = rng.integers(0, 50, 9), rng.integers(50, 150, 9)
    W, bs = 10, 16
    ids = rng.permutation(120)
    t = np.full((9, W), -1)
    at = 0
    for c in range(9):
        for j in range(-(-int(old[c]) // bs)):
            t[c, j], at = ids[at], at + 1
    f = np.concatenate([ids[at:], np.full(at, -1)])
    up = O.block_tables(old, new, t, f, 120 - at, bs, 0)
    assert up["refused"] == 0
    down = O.block_tables(new, old, up["table"], up["free_list"], up["n_free"], bs, 0)
    assert np.array_equal(down["table"], t) and down["n_free"] == 120 - at
    assert np.array_equal(down["free_list"][:120 - at], f[:120 - at])


def test_store_error_and_growth():
    """Codes are within half a step of the block's rows; a larger row shifts what was there."""
    rng = np.random.default_rng(3)
    bs, d = 16, 5
    c = dict(k=np.zeros((3, bs, 32), np.uint8), v=np.zeros((3, 32, bs), np.uint8), k_exp=np.zeros(3, np.uint8),
             v_exp=np.zeros(3, np.uint8), d=d)
    x, y = rng.standard_normal((20, d)), rng.standard_normal((20, d)) * 1e-3
    slots = [16 + i for i in range(16)] + [i for i in range(4)]
    r = dict(O.cache_store(c, x, y, slots), d=d)
    K, V, ok = O.cache_rows(r, [1, 0], 20)
    assert ok.all()
    # normal codes are off by at most 2^-4 of their value, subnormal ones by half of 2^-9 at the block's scale
    assert np.all(np.abs(K - x) <= 2.0 ** -4 * np.abs(x) + 2.0 ** -10 * 2.0 ** (r["k_exp"][[1] * 16 + [0] * 4] - 127.0)[:, None])
    assert np.all(np.abs(V - y) <= 2.0 ** -4 * np.abs(y) + 2.0 ** -10 * 2.0 ** (r["v_exp"][[1] * 16 + [0] * 4] - 127.0)[:, None])
    assert np.all(r["k"][:, :, d:] == 0) and np.all(r["k"][2] == 0)
    big = dict(O.cache_store(r, [[800.0] * d], [[0.0] * d], [4]), d=d)
    assert big["k_exp"][0] == 128 and big["v_exp"][0] == r["v_exp"][0]
    K2, _, _ = O.cache_rows(big, [1, 0], 21)
    assert np.all(np.abs(K2[20] - 800) <= 800 * 2.0 ** -4)
    assert np.all(np.abs(K2[16:20] - K[16:]) <= 2.0 ** -4 * np.abs(K[16:]) + 2.0 ** -9)
    assert np.array_equal(K2[:16], K[:16])


def test_cache_attention_is_attention_over_its_rows():
    rng = np.random.default_rng(4)
    bs, d, S, T, Hkv, G = 16, 8, 2, 3, 2, 2
    c = dict(k=np.zeros((9, bs, 32), np.uint8), v=np.zeros((9, 32, bs), np.uint8), k_exp=np.zeros(9, np.uint8),
             v_exp=np.zeros(9, np.uint8), d=d)
    table = np.array([[5, 2], [1, -1], [7, 99], [0, 3]])
    lens = [20, 2, 30, 0]
    for cell, n in enumerate(lens):
        s = [int(table[cell, p // bs]) * bs + p % bs for p in range(n)]
        c = dict(O.cache_store(c, rng.standard_normal((n, d)), rng.standard_normal((n, d)), s), d=d)
    q = rng.standard_normal((S, T, Hkv * G, d))
    r = O.cache_attention(q, c, table, lens, None)
    K, V, ok = O.cache_rows(c, table[0], 20)
    want = O.prompt_attention(q[0, :, :2], K[:, None], V[:, None], [0, 3], [0, 20], None, True)
    assert np.allclose(r["o"][0, :, :2], want["o"]) and np.allclose(r["lse"][0, :, :2], want["lse"])
    assert np.array_equal(r["o"][0, 0, 2:], np.zeros((2, d))) and np.all(r["lse"][0, 0, 2:] == -np.inf)  # 2 - 2 tokens
    K, V, ok = O.cache_rows(c, table[2], 30)
    assert ok.sum() == 16                       # the second block is out of range
    assert np.all(r["o"][1, :, 2:] == 0)        # an empty cell
