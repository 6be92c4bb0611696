"""Cells of nearly 2^31 tokens, the most that a table may list: every token is scored, and those of the cells behind."""
import math

import numpy as np
import pytest

from oracle.serving import E4M3

pytestmark = pytest.mark.gpu
BS, D, BLOCKS = 16, 32, 8
W = (1 << 27) - 1                       # blocks of a table row: 2^31 - 16 tokens
LENS = (W * BS - 3, 100)                # the first needs one tile of 64 tokens more than (2^31 - 64) / 64
TAIL = BLOCKS - 1                       # block that the first cell ends with, and no other entry names


@pytest.fixture(scope="module")
def tf():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2608_25230_amd import fw
    fw.lib()
    yield torch, fw
    torch.cuda.empty_cache()


def _state(tf, seed):
    """Keys of about unit size.  The last block's first column is large, so that with a query of 1 there its tokens weigh
    as much as all others; behind the end of the first cell it holds NaN."""
    torch, fw = tf
    rng = np.random.default_rng(seed)
    k, v = (rng.integers(0, 256, (BLOCKS, *x)).astype(np.uint8) for x in ((BS, D), (D, BS)))
    for x in (k, v):
        x[(x & 0x7F) == 0x7F] = 0
    k[:, :, 0] = 0
    k[TAIL, :, 0] = 0x7E                # 448
    k[TAIL, LENS[0] % BS:] = 0x7F
    v[TAIL, :, LENS[0] % BS:] = 0xFF
    e = np.full(BLOCKS, 120, np.uint8)  # 2^-7: values up to 3.5
    e_v = rng.integers(119, 122, BLOCKS).astype(np.uint8)
    cache = fw.KvCache(*(torch.tensor(x, device="cuda") for x in (k, v, e, e_v)), D)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    table = torch.randint(0, TAIL, (len(LENS), W), generator=gen, device="cuda", dtype=torch.int32)
    table[0, -1] = TAIL
    lens = torch.tensor(LENS, dtype=torch.int32, device="cuda")
    K = E4M3[k] * 2.0 ** (e[:, None, None].astype(int) - 127)
    V = E4M3[v].transpose(0, 2, 1) * 2.0 ** (e_v[:, None, None].astype(int) - 127)
    return cache, table, lens, K, V


def _queries(tf, dtype, T, G, seed):
    torch, _ = tf
    q = 0.1 * np.random.default_rng(seed).standard_normal((1, T, len(LENS) * G, D))
    q[..., 0] = 1
    return torch.tensor(q, dtype=torch.bfloat16 if dtype == "bf16" else torch.float32)


@pytest.mark.parametrize("dtype,T,G", [("bf16", 2, 4), ("f32", 3, 2), ("bf16", 5, 8), ("f32", 9, 3)])
def test_scores(tf, dtype, T, G):
    """By few_rows and many_rows.  The bounds are those of test_gpu_scores._check."""
    torch, fw = tf
    print(f"scores of {LENS[0]} tokens {dtype} T={T} G={G}", flush=True)
    cache, table, lens, K, _ = _state(tf, T)
    q = _queries(tf, dtype, T, G, T)
    f, R, u = 7.0, T * G, 2.0 ** -24
    scale = torch.full((len(LENS),), f, device="cuda")
    lse = torch.tensor(20 + np.random.default_rng(T).random((1, T, len(LENS) * G)), dtype=torch.float32)
    got = fw.cache_scores(q.cuda(), cache, table, lens, lse.cuda(), scale=scale)["scores"]
    torch.cuda.synchronize()
    assert got.shape == (len(LENS), W * BS)
    for c, n in enumerate(LENS):
        rows, l = (x[0, :, c * G:(c + 1) * G].double().numpy() for x in (q, lse))
        with np.errstate(invalid="ignore"):
            e = np.exp(f * np.einsum("bxd,tgd->tgbx", K, rows) - l[..., None, None])
            err = e * ((D + 4) * f * np.einsum("bxd,tgd->tgbx", np.abs(K), np.abs(rows)) + np.abs(l)[..., None, None] + 2)
        tol = lambda x, y: 2 * u * y + (R + 8) * u * x + 2.0 ** -126
        want, bound = e.sum((0, 1)) / R, err.sum((0, 1)) / R
        both = torch.tensor(np.stack([want, tol(want, bound)]), device="cuda")
        full = (n - (T - 1)) // BS      # blocks whose tokens every row sees
        for b0 in range(0, full, 1 << 21):
            b1 = min(b0 + (1 << 21), full)
            x, t = both[:, table[c, b0:b1].long()]
            worst = ((got[c, b0 * BS:b1 * BS].view(-1, BS).double() - x).abs() / t).max()
            assert float(worst) <= 1, (c, b0, float(worst))
        for j in range(full * BS, n):
            at = (slice(max(0, j - (n - T)), None), slice(None), int(table[c, j // BS]), j % BS)  # position t sees n - (T - 1 - t)
            x, y = e[at].sum() / R, err[at].sum() / R
            assert abs(float(got[c, j]) - x) <= tol(x, y), (c, j)
        assert not got[c, n:].any(), c


@pytest.mark.parametrize("dtype,T,G", [("bf16", 2, 4), ("f32", 3, 2), ("bf16", 2, 9)])
def test_attention(tf, dtype, T, G):
    """Two cells' weights and values, summed over each kind of token with its count.

    256 workgroups of four waves share 2^25 + 2 tiles and four more for each cell, so a wave sums at most N = 2^15 + 1 of
    them: a row's weights of a tile one by one in a lane group (16) and then to the sum, its products with the values in
    2 MFMA for each of two (bf16) or three (float32) parts of the weights.  Each step is off by 2^-23 at most, also where
    a product's sum is cut, not rounded.  64 more steps hold the sums inside an MFMA, over lane groups, waves and
    workgroups, and the scalings.  A weight's argument is off as in test_gpu_scores._check; parts leave 2^-15 at most of
    a weight in bf16."""
    torch, fw = tf
    print(f"attention over {LENS[0]} tokens {dtype} T={T} G={G}", flush=True)
    cache, table, lens, K, V = _state(tf, T + G)
    q = _queries(tf, dtype, T, G, T + G)
    f, u = 6.0, 2.0 ** -24
    got = fw.cache_attention(q.cuda(), cache, table, lens, scale=torch.full((len(LENS),), f, device="cuda"))
    o, lse = (got[x].double().cpu().numpy()[0] for x in ("o", "lse"))
    count = [torch.bincount(table[c, :n // BS], minlength=BLOCKS).cpu().numpy() for c, n in enumerate(LENS)]
    N, parts = 2 ** 15 + 1, 2 if dtype == "bf16" else 3
    half_step = 2.0 ** -8 if dtype == "bf16" else u
    for c, n in enumerate(LENS):
        for t in range(T):
            seen = n - (T - 1 - t)
            w = np.zeros((BLOCKS, BS)) + count[c][:, None]
            for j in range(min(seen, n // BS * BS), max(seen, n // BS * BS)):   # the last block's, and full blocks' hidden ones
                w[int(table[c, j // BS]), j % BS] += 1 if seen > n // BS * BS else -1
            here = w > 0
            k, v, w = K[here], V[here], w[here]
            for g in range(G):
                row = q[0, t, c * G + g].double().numpy()
                z = f * (k @ row)
                p = w * np.exp(z)
                want = math.log(p.sum())
                off = 2 * u * ((D + 4) * f * (np.abs(k) @ np.abs(row)).max() + abs(want) + 2)
                assert abs(lse[t, c * G + g] - want) <= (N + 64) * 2.0 ** -23 + off, (c, t, g)
                x, a = p @ v / p.sum(), p @ np.abs(v) / p.sum()
                tol = a * (((2 * parts + 1) * N + 64) * 2.0 ** -23 + 2 * off + 2.0 ** -15)
                assert np.all(np.abs(o[t, c * G + g] - x) <= tol + half_step * (np.abs(x) + tol)), (c, t, g)
