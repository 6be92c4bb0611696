"""Serving calls in forms that a program meets beside the plain ones."""
import numpy as np
import pytest

from oracle import serving as O
from tests.serving import HALF, tolerances
from tests.test_gpu_cache import _attend, _check_tables, _empty, _host, _i32, _setup, _tables, tf  # noqa: F401
from tests.test_gpu_prompt import _inputs, _run

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------
# block tables
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("C,bs,W,grow,n_slots", [(4, 16, 8, 3, 50), (4, 16, 8, 0, 5), (2048, 64, 65, 1, 4096),
                                                 (256, 16, 120, 90, 40000), (3000, 16, 12, 5, 30000)])
def test_no_slot_behind_the_last_token(tf, C, bs, W, grow, n_slots):
    """n_slots is an upper bound: entries without a token are -1, whatever the memory held before."""
    torch, fw = tf
    print(f"slots C={C} grow={grow} n_slots={n_slots}", flush=True)
    old = np.full(C, 7)
    new = old + np.where(np.arange(C) % 3 == 0, grow, 0)
    rng = np.random.default_rng(C)
    table, free, n_free = _tables(rng, old, W, bs, int(np.sum(-(-new // bs))) + 2)
    old_memory = torch.full((n_slots,), 3, dtype=torch.int64, device="cuda")     # a slot that exists
    del old_memory
    out = fw.block_tables(_i32(torch, old), _i32(torch, new), _i32(torch, table), _i32(torch, free), _i32(torch, [n_free]),
                          bs, n_slots=n_slots)
    torch.cuda.synchronize()
    ref = O.block_tables(old, new, table, free, n_free, bs, n_slots)
    got, n = out["slots"].cpu().numpy(), int((new - old).sum())
    assert n < n_slots and got[:n].tolist() == ref["slots"][:n]
    assert np.all(got[n:] == -1)


def test_captured_steps_in_which_fewer_cells_grow(tf):
    """One captured step, with n_slots for every cell, replayed while cells stop one after the other: a replay stores
    the tokens that come and touches no others."""
    torch, fw = tf
    rng = np.random.default_rng(3)
    C, bs, W, d = 6, 16, 4, 32
    old = np.array([15, 3, 20, 31, 1, 40])
    table, free, n_free = _tables(rng, old, W, bs, 30)
    cache = _empty(fw, 30, bs, d, seed=1)
    t, f, nf = _i32(torch, table), _i32(torch, free), _i32(torch, [n_free])
    lens, grows = _i32(torch, old), _i32(torch, np.zeros(C, int))
    k, v = (torch.zeros(C, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    fw.cache_store(cache, k, v, torch.full((C,), -1, dtype=torch.int64, device="cuda"))    # loads the kernels
    fw.block_tables(lens, lens, t, f, nf, bs, n_slots=C)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = fw.block_tables(lens, lens + grows, t, f, nf, bs, n_slots=C, lens=lens)
        fw.cache_store(cache, k, v, out["slots"])
    ref, rt, rf, rn, rl = dict(_host(cache), d=d), table, free, n_free, old
    for step, grow in enumerate(([1] * 6, [1, 0, 1, 0, 1, 1], [0, 0, 1, 0, 0, 1], [0] * 6, [0, 1, 0, 0, 0, 0])):
        n = sum(grow)
        x = torch.tensor(rng.standard_normal((2, C, d)).astype(np.float32)).bfloat16()
        k.copy_(x[0])
        v.copy_(x[1])
        grows.copy_(_i32(torch, grow))
        g.replay()
        torch.cuda.synchronize()
        r = O.block_tables(rl, rl + np.array(grow), rt, rf, rn, bs, C)
        rt, rf, rn, rl = r["table"], r["free_list"], r["n_free"], r["lens"]
        ref = dict(O.cache_store(ref, x[0, :n].double().numpy(), x[1, :n].double().numpy(), r["slots"][:n]), d=d)
        got = _host(cache)
        assert np.array_equal(lens.cpu().numpy(), rl) and np.array_equal(t.cpu().numpy(), rt), step
        for name in ("k", "v", "k_exp", "v_exp"):
            assert np.array_equal(got[name], ref[name]), (step, name)


@pytest.mark.parametrize("C,W,bs", [(256, 120, 16), (2048, 9, 16), (2049, 10, 16), (40, 500, 32)])
def test_tables_over_the_whole_card(tf, C, W, bs):
    """Growth, release and exchange of so many blocks and slots that several launches do it, for at most 2048 cells
    (whose offsets are staged) and more; a pure release of more blocks than the scan's workgroup moves itself."""
    torch, fw = tf
    print(f"whole card C={C} W={W}", flush=True)
    rng = np.random.default_rng(C)
    old, new = np.zeros(C, int), rng.integers(W * bs // 3, W * bs + 1, C)
    blocks = int(np.sum(-(-new // bs)))
    table, free, n_free = _tables(rng, old, W, bs, blocks + 5)
    n = int(new.sum())
    assert n > 8192 and C * W > 16384 and blocks > 4096
    t, f, nf, out = _check_tables(tf, old, new, table, free, n_free, bs, n)
    grown = (t.cpu().numpy(), f.cpu().numpy(), int(nf))
    _check_tables(tf, new, old, *grown, bs, 0)                                   # everything comes back
    some = np.where(np.arange(C) % 2 == 0, 0, new)
    half = O.block_tables(new, some, *grown, bs, 0)
    m = (half["table"], half["free_list"], half["n_free"])
    swap = np.where(np.arange(C) % 2 == 0, new, 0)                               # one half ends, the other begins
    k = int(np.maximum(swap - some, 0).sum())
    assert k > 8192
    _check_tables(tf, some, swap, *m, bs, k)
    step = np.where(np.arange(C) % 2 == 0, np.minimum(1 + np.arange(C) % 3, W * bs), 0)   # few slots, many blocks back
    _check_tables(tf, some, step, *m, bs, int(step.sum()))


@pytest.mark.parametrize("C,W,bs,grow", [(3000, 3, 64, 100), (50, 20, 128, 1200), (16384, 1, 16, 9), (500, 30, 16, 17)])
def test_short_tables_that_list_many_slots(tf, C, W, bs, grow):
    torch, fw = tf
    print(f"short tables C={C} grow={grow}", flush=True)
    rng = np.random.default_rng(C)
    old = rng.integers(0, W * bs - grow + 1, C)
    new = old + grow
    table, free, n_free = _tables(rng, old, W, bs, int(np.sum(-(-new // bs))) + 1)
    assert C * grow > 8192 and C * W <= 16384
    t, f, nf, out = _check_tables(tf, old, new, table, free, n_free, bs, C * grow)
    _check_tables(tf, new, old, t.cpu().numpy(), f.cpu().numpy(), int(nf), bs, 0)


# ---------------------------------------------------------------------------
# prompt attention
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,d", [("f32", 81), ("f32", 96), ("f32", 97), ("f32", 129), ("f32", 161), ("f32", 192),
                                     ("f32", 193), ("bf16", 91), ("bf16", 163), ("bf16", 190)])
@pytest.mark.parametrize("causal", [True, False])
def test_prompt_widths_of_the_general_kernel(tf, dtype, d, causal):
    print(f"general width {dtype} {d} causal={causal}", flush=True)
    _run(tf, 90, [70, 1, 33], [70, 5, 20], 4, 2, d, dtype, causal)
    _run(tf, 91, [3], [2500], 2, 1, d, dtype, causal)          # ranges of keys, joined


# ---------------------------------------------------------------------------
# weights in two bf16 parts
# ---------------------------------------------------------------------------

def _two_parts(ref, d, n):
    """tolerances() of float32 rows, but for the output's rounding, which is bf16's; and each weight is the sum of two
    bf16 roundings (the second is off by 2^-8 of what the first leaves, which is 2^-8 of the weight), either of which
    may underflow."""
    tol, _ = tolerances(ref, "f32", d, n)
    tol += 2.0 ** -16 * ref["abs_o"] * (1 + 2.0 ** -7) + n * 2.0 ** -117
    return tol + HALF["bf16"] * (np.abs(ref["o"]) + tol)


@pytest.mark.parametrize("d,lq,lk,causal", [(128, [300, 65], None, True), (64, [1, 129, 40], None, True),
                                            (80, [200, 33], None, False), (256, [150], None, True),
                                            (128, [3, 40], [4097, 2500], True), (64, [7], [3000], False),
                                            (192, [70, 5, 3], [10, 0, 300], True)])
def test_prompt_weights_keep_their_bits(tf, d, lq, lk, causal):
    """fine_weights: an output is off by its own rounding and what float32 loses, however much its terms cancel."""
    torch, fw = tf
    print(f"fine weights d={d} {lq} {lk}", flush=True)
    lk = lk or lq
    dev, f64, cu, cun = _inputs(torch, 60 + d, lq, lk, 4, 2, d, "bf16")
    out = fw.prompt_attention(*dev, *cu, causal=causal, fine_weights=True)
    plain = fw.prompt_attention(*dev, *cu, causal=causal)
    torch.cuda.synchronize()
    assert torch.equal(out["lse"], plain["lse"])
    ref = O.prompt_attention(*f64, *cun, None, causal)
    worst = np.max(np.abs(out["o"].double().cpu().numpy() - ref["o"]) / _two_parts(ref, d, max(lk)))
    assert worst <= 1, worst


def test_prompt_fine_weights_of_hidden_values_and_scales(tf):
    """Values that are not finite reach the rows that see them and no others; zero and negative scales."""
    torch, fw = tf
    for d in (64, 128, 256):
        dev, f64, cu, cun = _inputs(torch, 70, [70, 100], [70, 100], 2, 1, d, "bf16")
        clean = fw.prompt_attention(*dev, *cu, fine_weights=True)
        v = dev[2].clone()
        v[40, 0, 3], v[169, 0, 5] = float("inf"), float("nan")
        got = fw.prompt_attention(dev[0], dev[1], v, *cu, fine_weights=True)
        torch.cuda.synchronize()
        hit = torch.zeros(got["o"].shape, dtype=torch.bool)
        hit[40:70, :, 3] = True
        hit[169, :, 5] = True
        o, c = got["o"].float().cpu(), clean["o"].float().cpu()
        assert torch.equal(~torch.isfinite(o), hit) and torch.equal(o[~hit], c[~hit])
        for s in (0.0, -0.3):
            out = fw.prompt_attention(*dev, *cu, scale=torch.tensor([s], device="cuda"), fine_weights=True)
            ref = O.prompt_attention(*f64, *cun, np.float32([s]).astype(np.float64), True)
            assert np.all(np.abs(out["o"].double().cpu().numpy() - ref["o"]) <= _two_parts(ref, d, 100))


def test_fine_weights_leave_float32_rows_alone(tf):
    torch, fw = tf
    dev, f64, cu, cun = _inputs(torch, 71, [90], [90], 4, 2, 40, "f32")
    a, b = (fw.prompt_attention(*dev, *cu, fine_weights=x) for x in (False, True))
    torch.cuda.synchronize()
    assert torch.equal(a["o"], b["o"]) and torch.equal(a["lse"], b["lse"])


# ---------------------------------------------------------------------------
# attention over the cache
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("d,T,G,lens", [(128, 1, 4, [700, 90]), (64, 1, 4, [64, 333]), (128, 4, 8, [300, 41]),
                                        (64, 8, 8, [500, 100]), (256, 1, 2, [200, 65]), (128, 1, 4, [9000, 17]),
                                        (64, 5, 4, [5000, 2500])])
def test_decode_weights_keep_their_bits(tf, d, T, G, lens):
    """bf16 queries: the product with the values takes the softmax weights to 2^-16 of each, so that an output is off
    by its own rounding and what float32 loses, however much its terms cancel."""
    torch, fw = tf
    print(f"weights d={d} T={T} G={G} {lens}", flush=True)
    cache, table, q = _setup(tf, 40 + d + T, 1, T, 2, G, d, 64, lens, "bf16", garbage=False)
    out = fw.cache_attention(q.cuda(), cache, _i32(torch, table), _i32(torch, lens))
    torch.cuda.synchronize()
    ref = O.cache_attention(q.double().numpy(), _host(cache), table, lens, None)
    n = max(lens)
    worst = np.max(np.abs(out["o"].double().cpu().numpy() - ref["o"]) / _two_parts(ref, d, n))
    assert worst <= 1, worst


@pytest.mark.parametrize("dtype,d,T,G,lens", [("bf16", 64, 1, 8, [300, 200]), ("f32", 64, 1, 8, [300, 200]),
                                              ("bf16", 128, 3, 4, [5000, 70]), ("f32", 96, 3, 4, [3000, 70]),
                                              ("bf16", 64, 8, 8, [700, 90]), ("bf16", 256, 2, 4, [100, 2500])])
def test_decode_rows_do_not_depend_on_their_neighbours(tf, dtype, d, T, G, lens):
    """With the same lengths, a row's bits come from its query and what it sees: not from the other rows of its cell
    or from other cells."""
    torch, fw = tf
    print(f"neighbours {dtype} d={d} T={T} G={G}", flush=True)
    cache, table, q = _setup(tf, 50 + d, 1, T, 2, G, d, 16, lens, dtype)
    # every row's maximum rises along its keys, and by more than its neighbours' or by less
    for c, n in enumerate(lens):
        for j in range(-(-n // 16)):
            cache.k_exp[int(table[c, j])] = 112 + min(j, 10)
    q, t, n = q.cuda(), _i32(torch, table), _i32(torch, lens)
    a = fw.cache_attention(q, cache, t, n)
    q2 = q.clone()
    q2[:, 0, 1::2] *= 16.0
    b = fw.cache_attention(q2, cache, t, n)
    torch.cuda.synchronize()
    keep = torch.ones(q.shape[:3], dtype=torch.bool)
    keep[:, 0, 1::2] = False
    assert torch.equal(a["o"].cpu()[keep], b["o"].cpu()[keep]) and torch.equal(a["lse"].cpu()[keep], b["lse"].cpu()[keep])
    for blk in table[1]:
        if blk >= 0:
            cache.k_exp[int(blk)] += 3
            cache.v[int(blk)] = 0x7F
    c = fw.cache_attention(q, cache, t, n)
    torch.cuda.synchronize()
    assert torch.equal(a["o"][:, :, :G], c["o"][:, :, :G]) and torch.equal(a["lse"][:, :, :G], c["lse"][:, :, :G])


@pytest.mark.parametrize("dtype,d,T,G", [("bf16", 192, 1, 4), ("bf16", 256, 1, 2), ("bf16", 256, 4, 8), ("bf16", 96, 1, 3),
                                         ("bf16", 32, 1, 1), ("bf16", 33, 2, 3), ("bf16", 128, 4, 8), ("bf16", 128, 8, 8),
                                         ("f32", 80, 1, 3), ("f32", 80, 4, 3), ("f32", 128, 1, 2), ("f32", 192, 1, 2),
                                         ("f32", 256, 1, 2), ("f32", 200, 3, 7), ("f32", 96, 5, 4), ("f32", 64, 8, 8)])
def test_decode_widths_and_rows_over_shared_cells(tf, dtype, d, T, G):
    """Every width and several row tiles where cells are cut over workgroups and joined; some hold no token, one, or
    fewer than the new positions."""
    lens = [2600, 3, 0, 700, 2049, 512, 1111, 1]
    print(f"shared {dtype} d={d} T={T} G={G}", flush=True)
    cache, table, q = _setup(tf, 80 + d + T, 2, T, 4, G, d, 64, lens, dtype, extra=1)
    assert table.shape[1] > 32                # tiles of 64 tokens: more than one workgroup takes whole
    out = _attend(tf, cache, table, q, lens, dtype, what=f"shared {dtype} d={d} T={T} G={G}")
    assert out["_ws"] is not None


WIDE = [(128, 4, 8), (128, 8, 8), (128, 1, 17), (96, 5, 7), (64, 4, 8), (64, 8, 8), (64, 1, 33), (64, 20, 4), (32, 8, 8),
        (32, 3, 9)]


def _wide(table, d, bs):
    """The table with columns of -1 up to what holds more than 256 MB of codes for its cells."""
    dp = next(x for x in (32, 64, 96, 128) if x >= d)
    W = (1 << 28) // (table.shape[0] * bs * 2 * dp) + 1
    assert W > table.shape[1]
    return np.concatenate([table, np.full((table.shape[0], W - table.shape[1]), -1)], 1)


@pytest.mark.parametrize("d,T,G", WIDE)
def test_decode_row_tiles_of_tables_past_the_last_level_cache(tf, d, T, G):
    """bf16 queries of more than 16 rows a cell over tables that could hold more than 256 MB: several row tiles in a
    wave; NaN codes that some rows see and others do not."""
    torch, fw = tf
    print(f"row tiles d={d} T={T} G={G}", flush=True)
    lens = [2600, 3, 0, 700, 2049, 512, 1111, 70]
    cache, table, q = _setup(tf, 95 + d + T, 2, T, 4, G, d, 256, lens, "bf16")
    table = _wide(table, d, 256)
    clean = _attend(tf, cache, table, q, lens, "bf16", what=f"row tiles d={d} T={T} G={G}")
    if T > 1:
        b, at = int(table[3, 699 // 256]), 699 % 256
        cache.v[b, 5, at] = 0x7F            # the last token of cell 3, which its last position alone sees
        got = fw.cache_attention(q.cuda(), cache, _i32(torch, table), _i32(torch, lens))
        torch.cuda.synchronize()
        hit = torch.zeros(got["o"].shape, dtype=torch.bool)
        hit[0, T - 1, 3 * G:4 * G, 5] = True
        o, c = got["o"].cpu(), clean["o"].cpu()
        assert torch.equal(torch.isnan(o), hit) and torch.equal(o[~hit], c[~hit])
        assert torch.equal(got["lse"], clean["lse"])


@pytest.mark.parametrize("d,T,G", [(128, 4, 8), (96, 6, 8), (64, 8, 8), (64, 4, 5)])
def test_decode_row_tiles_of_many_short_tables(tf, d, T, G):
    """Tables that one workgroup takes whole, together past 256 MB."""
    print(f"row tiles, short tables d={d} T={T} G={G}", flush=True)
    rng = np.random.default_rng(d + T)
    Hkv, bs = 2, 256
    S = {64: 520, 96: 345, 128: 260}[d]
    lens = rng.integers(0, 9, S * Hkv)
    lens[5], lens[S] = 300, 100
    cache, table, q = _setup(tf, 96 + d, S, T, Hkv, G, d, bs, lens, "bf16")
    table = np.concatenate([table, np.full((S * Hkv, 8 - table.shape[1]), -1)], 1)       # 2048 tokens: 32 tiles
    assert S * Hkv * 2048 * 2 * d > 1 << 28
    out = _attend(tf, cache, table, q, lens, "bf16", what=f"many short tables d={d} T={T} G={G}")
    assert out["_ws"] is None
