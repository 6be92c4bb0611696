"""fw_cache_scores and fw_cache_select against the oracle."""
import numpy as np
import pytest

from oracle import cells as O
from oracle import serving as V
from tests.cells import random_state

pytestmark = pytest.mark.gpu
DP = {20: 32, 64: 64, 80: 96, 128: 128, 160: 192, 256: 256}


@pytest.fixture(scope="module")
def tf():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2608_25230_amd import fw
    fw.lib()
    return torch, fw


def _cuda(torch, x, dtype=None):
    return torch.tensor(np.asarray(x), dtype=dtype, device="cuda")


def _cache(tf, s):
    torch, fw = tf
    return fw.KvCache(*(_cuda(torch, s[key]) for key in ("k", "v", "k_exp", "v_exp")), s["d"])


def _state(rng, lens, bs, d):
    """Keys of about unit size, so that logits are of the size that attention meets."""
    s = random_state(rng, lens, bs, DP[d], d, spread=2)
    s["k_exp"] -= np.uint8(7)  # codes up to 448 stand for values up to 3.5 2^2
    return s


def _inputs(tf, rng, s, dtype, S, T, G):
    torch, fw = tf
    Hkv = len(s["lens"]) // S
    q = torch.tensor(rng.standard_normal((S, T, Hkv * G, s["d"])), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32)
    scale = (0.5 + rng.random(Hkv)).astype(np.float32) / np.float32(np.sqrt(s["d"]))
    att = V.cache_attention(q.double().numpy(), s, s["table"], s["lens"], scale)
    return q, scale, att["lse"].astype(np.float32)


def _check(got, ref, R):
    """A weight's argument is off by `err` units of rounding (the logit's d products and sums and two scalings, the
    log-sum-exp's change to base 2, the difference), its exponential by 2 more, which `err` holds; twice that bounds the
    weight.  R weights and their sum over lanes and turns, the mean and the earlier score round once each.  A weight
    below the least normal number may be lost."""
    u = 2.0 ** -24
    inside = ~np.isnan(ref["scores"])
    x = np.where(inside, ref["scores"], 0)
    tol = 2 * u * ref["err"] + (R + 8) * u * np.abs(x) + 2.0 ** -126
    e = np.where(inside, np.abs(np.where(inside, got, 0) - x) / tol, 0)
    assert np.max(e, initial=0) <= 1, float(np.max(e))
    return inside


def _run(tf, dtype, d, bs, lens, S, T, G, n=None, seed=0):
    torch, fw = tf
    print(f"scores {dtype} d={d} bs={bs} lens={lens if len(lens) < 12 else len(lens)} S={S} T={T} G={G} n={n}", flush=True)
    rng = np.random.default_rng(seed + d + len(lens))
    s = _state(rng, lens, bs, d)
    q, scale, lse = _inputs(tf, rng, s, dtype, S, T, G)
    W = s["table"].shape[1]
    ref = O.cache_scores(q.double().numpy(), s, s["table"], s["lens"], lse, scale, n or W * bs)
    args = (q.cuda(), _cache(tf, s), _cuda(torch, s["table"]), _cuda(torch, s["lens"]), _cuda(torch, lse))
    out = None if n is None else torch.full((len(lens), n), 7.0, device="cuda")
    got = fw.cache_scores(*args, scale=_cuda(torch, scale), scores=out)["scores"].cpu().numpy()
    inside = _check(got, ref, T * G)
    assert np.all(got[~inside] == (0.0 if n is None else 7.0))
    return s, args, scale, ref, got


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,bs", [(20, 16), (64, 32), (80, 16), (128, 64), (160, 128), (256, 256), (128, 16)])
def test_widths_and_blocks(tf, dtype, d, bs):
    _run(tf, dtype, d, bs, [1, 70, 129, 300], 2, 3, 4)
    _run(tf, dtype, d, bs, [64, 63], 1, 1, 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,G", [(1, 8), (5, 3), (16, 1), (17, 1), (64, 4), (33, 8), (300, 2)])
def test_rows(tf, dtype, T, G):
    """Rows of one tile and of several, more than LDS holds at a time, more positions than tokens."""
    _run(tf, dtype, 128, 64, [5, 400], 1, T, G)


@pytest.mark.parametrize("dtype,d,T,G", [("bf16", 20, 1100, 2), ("bf16", 20, 520, 2), ("f32", 20, 350, 2), ("f32", 80, 60, 3),
                                         ("bf16", 160, 100, 2), ("bf16", 256, 65, 2), ("bf16", 256, 300, 1), ("f32", 256, 23, 2),
                                         ("f32", 256, 100, 1)])
def test_rows_past_what_is_held(tf, dtype, d, T, G):
    """Rows that a workgroup of twice the waves holds, in one turn and in several, at every kind of width."""
    _run(tf, dtype, d, 16, [90, 0, 700, 3], 1, T, G)


@pytest.mark.parametrize("C,top", [(1, 5000), (64, 700), (300, 60), (1500, 20)])
def test_many_and_long_cells(tf, C, top):
    rng = np.random.default_rng(C)
    lens = rng.integers(0, top + 1, C).tolist()
    lens[0] = top
    _run(tf, "bf16", 64, 16, lens, 1, 1, 2)


def test_fewer_columns_than_tokens(tf):
    _run(tf, "bf16", 64, 16, [200, 90, 0, 33], 2, 4, 2, n=90)
    _run(tf, "f32", 64, 16, [200, 90], 1, 700, 1, n=77)


def test_earlier_scores(tf):
    """Added, from the same tensor and from another, with one turn of the rows and with several."""
    torch, fw = tf
    for T in (2, 400):
        s, args, scale, ref, got = _run(tf, "f32", 128, 32, [130, 7, 0, 64], 2, T, 2)
        old = torch.rand(got.shape, device="cuda")
        ref = dict(ref, scores=ref["scores"] + old.double().cpu().numpy())
        a = fw.cache_scores(*args, scale=_cuda(torch, scale), earlier=old)["scores"]
        inside = _check(a.cpu().numpy(), ref, 2 * T)
        assert not a.cpu().numpy()[~inside].any()
        b = old.clone()
        fw.cache_scores(*args, scale=_cuda(torch, scale), earlier=b, scores=b)
        t = torch.tensor(inside, device="cuda")
        assert torch.equal(b[t], a[t]) and torch.equal(b[~t], old[~t])


def test_hidden_and_missing_tokens(tf):
    """Codes of NaN behind the end and among hidden tokens, blocks out of range, rows that see nothing."""
    torch, fw = tf
    rng = np.random.default_rng(5)
    s = _state(rng, [40, 3, 100, 20], 16, 64)
    s["table"][2, 1], s["table"][2, 3] = -1, 10 ** 6
    s["k"][s["table"][0, 2], 8:] = 0x7F          # behind 40 tokens
    s["k"][s["table"][3, 1], 3] = 0xFF           # token 19 of 20: the last position alone sees it
    q, scale, lse = _inputs(tf, rng, s, "bf16", 2, 5, 2)
    ref = O.cache_scores(q.double().numpy(), s, s["table"], s["lens"], lse, scale, 112)
    c, l = _cache(tf, s), _cuda(torch, lse)
    l[0, 0] = float("-inf")                      # cell 1's first positions see nothing: whatever they hold is not looked at
    seen = lse.copy()
    got = fw.cache_scores(q.cuda(), c, _cuda(torch, s["table"]), _cuda(torch, s["lens"]), _cuda(torch, seen),
                          scale=_cuda(torch, scale))["scores"].cpu().numpy()
    assert np.isnan(got[3, 19]) and np.isnan(ref["scores"][3, 19])
    ref["scores"][3, 19] = np.nan
    assert np.array_equal(got[2, 16:32], np.zeros(16)) and np.array_equal(got[2, 48:64], np.zeros(16))
    keep = got.copy()
    keep[3, 19] = 0
    _check(keep, ref, 10)


@pytest.mark.parametrize("dtype,T,G", [("bf16", 5, 2), ("f32", 5, 3), ("bf16", 5, 8), ("f32", 17, 2)])
def test_nan_keys_reach_only_rows_that_see_them(tf, dtype, T, G):
    """Keys of NaN among the last tokens, which some rows see and others do not: they alone score NaN.  The log-sum-exps
    are those of the cache before, and NaN for rows that see nothing, which are not looked at."""
    torch, fw = tf
    rng = np.random.default_rng(T + G)
    lens = [40, 3, 100, 20, 200, 64]
    s = _state(rng, lens, 16, 64)
    q, scale, lse = _inputs(tf, rng, s, dtype, 2, T, G)
    lse[np.isneginf(lse)] = np.nan
    assert np.isnan(lse).any()
    bad = [(0, 37), (2, 97), (3, 19), (4, 199), (4, 196), (5, 63)]
    for c, j in bad:
        s["k"][s["table"][c, j // 16], j % 16, 5] = 0x7F
    ref = O.cache_scores(q.double().numpy(), s, s["table"], s["lens"], lse, scale, 208)
    want = np.full((6, 208), False)
    for c, j in bad:
        want[c, j] = True
    for c, n in enumerate(lens):
        assert np.array_equal(np.isnan(ref["scores"][c, :n]), want[c, :n])
    got = fw.cache_scores(q.cuda(), _cache(tf, s), _cuda(torch, s["table"]), _cuda(torch, s["lens"]), _cuda(torch, lse),
                          scale=_cuda(torch, scale))["scores"].cpu().numpy()
    assert np.array_equal(np.isnan(got), want)
    ref["err"][want] = 0
    inside = _check(got, ref, T * G)
    assert inside.sum() == sum(lens) - len(bad)


def test_they_are_the_weights_of_cache_attention(tf):
    """Scores with cache_attention's lse sum to the share of rows that see something, at the sizes of a window."""
    torch, fw = tf
    rng = np.random.default_rng(6)
    lens = [3000, 801, 64, 5000, 40, 1]
    s = _state(rng, lens, 64, 128)
    q = torch.tensor(rng.standard_normal((3, 64, 8, 128)), dtype=torch.bfloat16, device="cuda")
    c, t, n = _cache(tf, s), _cuda(torch, s["table"]), _cuda(torch, s["lens"])
    lse = fw.cache_attention(q, c, t, n)["lse"]
    got = fw.cache_scores(q, c, t, n, lse)["scores"].double().sum(1).cpu().numpy()
    share = np.array([sum(1 for p in range(64) if m - (63 - p) > 0) / 64 for m in lens])
    # a weight is off by a factor of 1 +- 2 (d + 4) 2^-24 times the logit's products, below 2^9 here, in both calls
    assert np.all(np.abs(got - share) <= 4 * 132 * 2.0 ** -24 * 2 ** 9 * share)


def test_scores_captured_and_repeated(tf):
    torch, fw = tf
    s, args, scale, ref, _ = _run(tf, "bf16", 128, 64, [500, 90, 1000, 1], 2, 8, 2)
    scale = _cuda(torch, scale)
    out = torch.zeros(4, s["table"].shape[1] * 64, device="cuda")
    fw.cache_scores(*args, scale=scale, scores=out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        fw.cache_scores(*args, scale=scale, scores=out)
    for i in range(4):
        args[0].copy_(torch.randn(args[0].shape, device="cuda"))
        args[3][0] = 500 - 100 * i
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, fw.cache_scores(*args, scale=scale)["scores"])


def test_strided_queries(tf):
    torch, fw = tf
    s, args, scale, _, got = _run(tf, "bf16", 64, 16, [50, 90, 200, 1], 2, 3, 2)
    wide = torch.zeros(3, 2, 4, 67, dtype=torch.bfloat16, device="cuda")
    q = wide.transpose(0, 1)[..., 1:65]
    q.copy_(args[0])
    again = fw.cache_scores(q, *args[1:], scale=_cuda(torch, scale))["scores"].cpu().numpy()
    assert np.array_equal(again, got)


# ---------------------------------------------------------------------------
# selection
# ---------------------------------------------------------------------------

def _select(tf, x, lens, keep, recent, extra=0):
    torch, fw = tf
    ref = O.cache_select(x, lens, keep, recent)
    n = max(0, sum(len(r) for r in ref) + extra)
    got = fw.cache_select(_cuda(torch, x, torch.float32), _cuda(torch, lens, torch.int32), _cuda(torch, keep, torch.int32),
                          recent=recent, n_kept=n)
    off = np.cumsum([0] + [len(r) for r in ref])
    assert np.array_equal(got["offsets"].cpu().numpy(), off)
    flat = np.array([p for r in ref for p in r], np.int64)
    want = np.full(n, -1)
    want[:min(n, len(flat))] = flat[:n]
    assert np.array_equal(got["kept_pos"].cpu().numpy(), want)


@pytest.mark.parametrize("C,n", [(1, 1), (3, 7), (5, 1000), (4, 1024), (3, 1025), (2, 5000), (40, 300), (1300, 20), (2, 40000)])
@pytest.mark.parametrize("what", ["normal", "ties", "equal", "odd"])
def test_select(tf, C, n, what):
    print(f"select C={C} n={n} {what}", flush=True)
    rng = np.random.default_rng(C + n)
    x = np.exp(2 * rng.standard_normal((C, n))).astype(np.float32)
    if what == "ties":
        x = np.floor(4 * x) / 4
    if what == "equal":
        x[:] = 0.25
    if what == "odd":
        x = rng.choice(np.array([0.0, -0.0, 1.0, -1.0, np.inf, -np.inf, np.nan, 1e-42], np.float32), (C, n))
        x[rng.random((C, n)) < 0.3] = rng.standard_normal()
    lens = rng.integers(0, n + 1, C)
    lens[0] = n
    keep = rng.integers(-1, n + 2, C)
    for recent in (0, 3, n):
        _select(tf, x, lens, keep, recent)
    _select(tf, x, lens, np.full(C, n // 2), 2)
    _select(tf, x, lens + 5, keep, 1, extra=9)          # lengths past the row, room behind the last kept token
    _select(tf, x, lens, keep, 1, extra=-2)             # fewer places than kept tokens
    _select(tf, x, np.zeros(C, int) - 1, keep, 1, extra=4)


@pytest.mark.parametrize("C,n", [(5000, 70), (3, 4096), (3, 4097), (2, 8192), (2, 8193), (2, 16385), (2, 32768), (2, 32769), (3, 70001), (60, 34000)])
@pytest.mark.parametrize("what", ["normal", "ties"])
def test_select_widths(tf, C, n, what):
    """Every width of a row, rows in slices, and more cells than every workgroup sums for itself."""
    print(f"select C={C} n={n} {what}", flush=True)
    rng = np.random.default_rng(n)
    x = rng.standard_normal((C, n)).astype(np.float32)
    if what == "ties":
        x = np.floor(x).astype(np.float32)
    lens = rng.integers(0, n + 1, C)
    lens[0], lens[-1] = n, n
    keep = rng.integers(0, n + 1, C)
    _select(tf, x, lens, keep, 40)
    keep[0], keep[1], keep[-1] = n, 0, n - 1
    _select(tf, x, lens, keep, 0, extra=5)


def test_select_captured(tf):
    torch, fw = tf
    x = torch.rand(6, 3000, device="cuda")
    lens, keep = torch.full((6,), 3000, dtype=torch.int32, device="cuda"), torch.full((6,), 700, dtype=torch.int32, device="cuda")
    fw.cache_select(x, lens, keep, recent=9, n_kept=4200)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = fw.cache_select(x, lens, keep, recent=9, n_kept=4200)
    for i in range(4):
        x.copy_(torch.rand(6, 3000, device="cuda"))
        lens[2], keep[1] = 2000 - i, 10 * i
        g.replay()
        torch.cuda.synchronize()
        e = fw.cache_select(x, lens, keep, recent=9, n_kept=4200)
        assert torch.equal(out["offsets"], e["offsets"]) and torch.equal(out["kept_pos"], e["kept_pos"])


def test_refusals(tf):
    torch, fw = tf
    s, args, scale, _, _ = _run(tf, "bf16", 64, 16, [50, 90], 1, 1, 2)
    q, c, t, n, l = args
    i32 = torch.zeros(2, dtype=torch.int32, device="cuda")
    x = torch.zeros(2, 9, device="cuda")
    for f in (lambda: fw.cache_scores(q, c, t, n, l[..., :1]), lambda: fw.cache_scores(q, c, t, n, l.double()),
              lambda: fw.cache_scores(q.half(), c, t, n, l), lambda: fw.cache_scores(q[..., :63], c, t, n, l),
              lambda: fw.cache_scores(q, c, t, n[:1], l), lambda: fw.cache_scores(q, c, t, n, l, scale=l.view(-1)[:3]),
              lambda: fw.cache_scores(q, c, t, n, l, scores=torch.zeros(3, 9, device="cuda")),
              lambda: fw.cache_scores(q, c, t, n, l, scores=x, earlier=torch.zeros(2, 8, device="cuda")),
              lambda: fw.cache_scores(q, c, t, n, l, scores=x.t()),
              lambda: fw.cache_select(x, i32[:1], i32, n_kept=2), lambda: fw.cache_select(x, i32, i32.long(), n_kept=2),
              lambda: fw.cache_select(x, i32, i32, n_kept=-1), lambda: fw.cache_select(x, i32, i32, n_kept=2, recent=-1),
              lambda: fw.cache_select(x[:, :5], i32, i32, n_kept=2), lambda: fw.cache_select(x.double(), i32, i32, n_kept=2)):
        with pytest.raises(fw.FwError):
            f()
