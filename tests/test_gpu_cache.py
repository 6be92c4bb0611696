"""fw_block_tables, fw_cache_store and fw_cache_attention against the oracle,
and the serving path end to end."""
import numpy as np
import pytest

from oracle import serving as O
from tests.parity import record
from tests.serving import check, rows

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tf():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2608_25230_amd import fw
    fw.lib()
    return torch, fw


def _i32(torch, x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


# ---------------------------------------------------------------------------
# block tables
# ---------------------------------------------------------------------------

def _tables(rng, old, W, bs, n_blocks):
    ids = rng.permutation(n_blocks)
    table, at = np.full((len(old), W), -1), 0
    for c, n in enumerate(old):
        for j in range(-(-int(n) // bs)):
            table[c, j], at = ids[at], at + 1
    return table, np.concatenate([ids[at:], np.full(at, -7)]), n_blocks - at


def _check_tables(tf, old, new, table, free, n_free, bs, n_slots, alias=False):
    torch, fw = tf
    t, f, nf = _i32(torch, table), _i32(torch, free), _i32(torch, [n_free])
    o = _i32(torch, old)
    out = fw.block_tables(o, _i32(torch, new), t, f, nf, bs, n_slots=n_slots, lens=o if alias else None)
    torch.cuda.synchronize()
    ref = O.block_tables(old, new, table, free, n_free, bs, n_slots)
    assert np.array_equal(t.cpu().numpy(), ref["table"])
    assert np.array_equal(f.cpu().numpy(), ref["free_list"])
    assert int(nf) == ref["n_free"] and int(out["refused"]) == ref["refused"]
    assert np.array_equal(out["offsets"].cpu().numpy(), ref["offsets"])
    assert np.array_equal(out["lens"].cpu().numpy(), ref["lens"])
    got = out["slots"].cpu().numpy()
    assert got.shape == (n_slots,)
    for i, s in enumerate(ref["slots"]):
        assert s is None or got[i] == s, i
    return t, f, nf, out


@pytest.mark.parametrize("C,bs,top", [(1, 16, 1), (1, 64, 500), (3, 16, 40), (70, 32, 200), (1030, 64, 90), (2500, 16, 33),
                                      (9, 256, 700), (5, 128, 0)])
@pytest.mark.parametrize("what", ["fill", "step", "mix", "empty"])
def test_tables_match_the_cells_in_order(tf, C, bs, top, what):
    print(f"tables C={C} bs={bs} top={top} {what}", flush=True)
    rng = np.random.default_rng(C + bs)
    old = rng.integers(0, top + 1, C)
    new = rng.integers(0, top + 1, C)
    if what == "fill":
        old = np.zeros(C, int)
    if what == "step":
        new = old + 1
    if what == "empty":
        new = np.zeros(C, int)
    W = -(-(top + 1) // bs)
    nb = int(np.sum(-(-np.maximum(old, new) // bs))) + 3
    table, free, n_free = _tables(rng, old, W, bs, nb)
    n = int(np.maximum(new - old, 0).sum())
    _check_tables(tf, old, new, table, free, n_free, bs, n, alias=what == "mix")


@pytest.mark.parametrize("C,bs", [(6, 16), (300, 32), (40, 64)])
def test_tables_many_blocks_and_slots(tf, C, bs):
    """More blocks and slots than one workgroup takes; then everything goes back, and the stack is as before."""
    torch, fw = tf
    rng = np.random.default_rng(C)
    old, new = np.zeros(C, int), rng.integers(0, 24000 // C * 3, C)
    W = int(new.max()) // bs + 2
    table, free, n_free = _tables(rng, old, W, bs, int(np.sum(-(-new // bs))) + 5)
    n = int(new.sum())
    assert n > 8192 and C * W > 256
    t, f, nf, out = _check_tables(tf, old, new, table, free, n_free, bs, n)
    stack = f.cpu().numpy()
    back = fw.block_tables(out["lens"], _i32(torch, old), t, f, nf, bs, n_slots=0)
    assert np.array_equal(t.cpu().numpy(), table) and int(nf) == n_free and int(back["refused"]) == 0
    assert np.array_equal(f.cpu().numpy()[:n_free], free[:n_free]) and np.array_equal(f.cpu().numpy(), stack)


@pytest.mark.parametrize("C", [4, 50, 1500])
@pytest.mark.parametrize("spare", [0, 1, 3, 17])
def test_tables_refuse_whole_cells(tf, C, spare):
    """Too few free blocks, lengths beyond the row, negative lengths: cells are refused whole, in order."""
    rng = np.random.default_rng(C + spare)
    bs, W = 16, 6
    old = rng.integers(0, W * bs + 1, C)
    new = rng.integers(-5, W * bs + 40, C)
    table, free, n_free = _tables(rng, old, W, bs, int(np.sum(-(-old // bs))) + spare)
    n = int(np.maximum(new - old, 0).sum())
    _check_tables(tf, old, new, table, free, n_free, bs, n)


@pytest.mark.parametrize("C,W,few", [(6, 6, True), (1500, 6, True), (6, 40, False), (300, 40, False), (4000, 6, True),
                                     (4000, 6, False), (2500, 30, False)])
def test_tables_serve_cells_without_need_after_the_stack_ran_out(tf, C, W, few):
    """Every third cell grows until there are no blocks; the others shrink or stay within their last block."""
    rng = np.random.default_rng(C + W)
    bs = 16
    old = rng.integers(bs + 1, W * bs + 1, C)
    most = 3 * bs if few else W * bs
    new = np.where(np.arange(C) % 3 == 0, np.minimum(old + rng.integers(bs, most + 1, C), W * bs), old)
    new = np.where(np.arange(C) % 3 == 1, np.maximum(old - rng.integers(0, 2 * bs, C), 0), new)
    new = np.where(np.arange(C) % 3 == 2, -(-old // bs) * bs, new)
    table, free, n_free = _tables(rng, old, W, bs, int(np.sum(-(-old // bs))))
    n = int(np.maximum(new - old, 0).sum())
    _, _, nf, out = _check_tables(tf, old, new, table, free, n_free, bs, n)
    lens = out["lens"].cpu().numpy()
    assert np.array_equal(lens[1::3], new[1::3]) and np.array_equal(lens[2::3], new[2::3]) and int(nf) >= 0
    _check_tables(tf, old, new, table, free, n_free, bs, 0, alias=True)


def test_tables_write_no_slot_past_the_last_token(tf):
    torch, fw = tf
    L = fw.lib()
    for n_slots, many in ((40, False), (20000, True), (7, False)):
        table = torch.full((2, 1200), -1, dtype=torch.int32, device="cuda")
        free, nf = torch.arange(3000, dtype=torch.int32, device="cuda"), _i32(torch, [3000])
        new = [9, 14] if not many else [5000, 9000]
        slots = torch.full((n_slots + 50,), -9, dtype=torch.int64, device="cuda")
        offsets, lens, refused = torch.zeros(3, dtype=torch.int64, device="cuda"), _i32(torch, [0, 0]), _i32(torch, [0])
        need = L.fw_block_tables_workspace_size(2)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        assert L.fw_block_tables(2, lens.data_ptr(), _i32(torch, new).data_ptr(), 16, 1200, table.data_ptr(), 3000,
                                 free.data_ptr(), nf.data_ptr(), n_slots, slots.data_ptr(), offsets.data_ptr(),
                                 lens.data_ptr(), refused.data_ptr(), ws.data_ptr(), need,
                                 torch.cuda.current_stream().cuda_stream) == 0
        torch.cuda.synchronize()
        n = min(sum(new), n_slots)
        assert torch.all(slots[n:] == -9) and torch.all(slots[:n] >= 0) and slots[:n].unique().numel() == n


# ---------------------------------------------------------------------------
# the store
# ---------------------------------------------------------------------------

def _empty(fw, n_blocks, bs, d, seed=None):
    c = fw.kv_cache(n_blocks, bs, d)
    if seed is not None:      # filled before: any codes, middling exponents
        rng = np.random.default_rng(seed)
        import torch
        for t in (c.k, c.v):
            x = rng.integers(0, 127, t.shape) + 128 * rng.integers(0, 2, t.shape)
            t.copy_(torch.tensor(np.where(x % 128 == 127, 0, x).astype(np.uint8)))
        c.k[:, :, d:] = 0
        c.v[:, d:, :] = 0
        for t in (c.k_exp, c.v_exp):
            t.copy_(torch.tensor(rng.integers(110, 130, t.shape).astype(np.uint8)))
    return c


def _host(c):
    return dict(k=c.k.cpu().numpy(), v=c.v.cpu().numpy(), k_exp=c.k_exp.cpu().numpy(), v_exp=c.v_exp.cpu().numpy(), d=c.d)


def _same_cache(c, ref):
    for name in ("k_exp", "v_exp", "k", "v"):
        a, b = getattr(c, name).cpu().numpy(), ref[name]
        if name in "kv":     # NaN has two codes
            a, b = np.where(a % 128 == 127, 127, a), np.where(b % 128 == 127, 127, b)
        assert np.array_equal(a, b), (name, int((a != b).sum()), np.argwhere(a != b)[:3])


def _slots(rng, runs, n_blocks, bs):
    """Slots of (offset in the first block, tokens) runs, each in blocks of its own."""
    ids, at, out = rng.permutation(n_blocks), 0, []
    for off, n in runs:
        for p in range(off, off + n):
            out.append(int(ids[at + p // bs]) * bs + p % bs)
        at += -(-(off + n) // bs)
    return np.array(out, np.int64)


RUNS = [[(0, 1)], [(5, 1), (0, 3), (15, 2), (0, 0)], [(0, 16), (0, 17), (3, 70)], [(i % 16, 1) for i in range(40)]]


@pytest.mark.parametrize("runs", RUNS)
@pytest.mark.parametrize("dtype,d,bs", [("bf16", 128, 64), ("bf16", 128, 16), ("f32", 80, 32), ("bf16", 64, 256),
                                        ("f32", 7, 16), ("bf16", 33, 128), ("bf16", 256, 64), ("bf16", 1, 16)])
def test_store(tf, runs, dtype, d, bs):
    torch, fw = tf
    print(f"store {runs[:3]} {dtype} d={d} bs={bs}", flush=True)
    rng = np.random.default_rng(d + bs)
    n_blocks = 3 + sum(-(-(a + b) // bs) for a, b in runs)
    cache = _empty(fw, n_blocks, bs, d, seed=5)
    slots = _slots(rng, runs, n_blocks, bs)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    N = len(slots)
    # rows of every size: blocks grow, keep their exponent, hold zeros only
    size = 2.0 ** rng.integers(-12, 12, (N, 1))
    k, v = (torch.tensor((rows(rng, (N, d)) * size).astype(np.float32)).to(dt) for _ in range(2))
    if N > 2:
        v[1] = 0
    ref = O.cache_store(_host(cache), k.double().numpy(), v.double().numpy(), slots)
    fw.cache_store(cache, k.cuda(), v.cuda(), torch.tensor(slots).cuda())
    torch.cuda.synchronize()
    _same_cache(cache, ref)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_store_rows_of_a_fused_projection_and_odd_starts(tf, dtype):
    torch, fw = tf
    rng = np.random.default_rng(1)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    for d, pad in ((128, 0), (80, 8), (40, 3)):
        kv = torch.tensor(rng.standard_normal((50, 2 * d + pad)).astype(np.float32)).to(dt)
        k, v = kv[:, pad:pad + d], kv[:, pad + d:]
        cache = _empty(fw, 4, 32, d)
        slots = np.arange(7, 57)
        ref = O.cache_store(_host(cache), k.double().numpy(), v.double().numpy(), slots)
        dev = kv.cuda()
        fw.cache_store(cache, dev[:, pad:pad + d], dev[:, pad + d:], torch.tensor(slots).cuda())
        torch.cuda.synchronize()
        _same_cache(cache, ref)


def test_store_skips_slots_out_of_range(tf):
    torch, fw = tf
    rng = np.random.default_rng(2)
    cache = _empty(fw, 4, 16, 32, seed=3)
    slots = np.array([-1, 5, 6, -1, -1, 64, 1 << 40, 20, 63, 64, -(1 << 40), 32, 33, 34, 47], np.int64)
    x = torch.tensor(rng.standard_normal((len(slots), 32)).astype(np.float32))
    keep = slots != 47      # 34 and 47 would be two runs of one block
    ref = O.cache_store(_host(cache), x.double().numpy()[keep], x.double().numpy()[keep], slots[keep])
    fw.cache_store(cache, x[keep].cuda(), x[keep].cuda(), torch.tensor(slots[keep]).cuda())
    torch.cuda.synchronize()
    _same_cache(cache, ref)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_store_non_finite_subnormal_and_huge(tf, dtype):
    torch, fw = tf
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    d = 8
    x = torch.zeros(6, d)
    x[0] = torch.tensor([float("nan"), float("inf"), -float("inf"), 1.0, -2.0, 0.0, -0.0, 3.5])
    x[1] = float("inf")
    x[2] = 1e-40
    x[3] = torch.tensor([3.3e38, -3.3e38, 1.0, 1e30, 2e36, 7e35, 1e34, 0.0])
    x[4] = torch.tensor([2.0 ** -126, 2.0 ** -120, 2.0 ** -133, 0.0, 2.0 ** -118, 2.0 ** -128, 0.0, 2.0 ** -119])
    x[5] = torch.tensor([448.0, 449.0, -464.0, 480.0, 16.5, 17.5, 0.001, 2.0 ** -10])
    x = x.to(dt)
    cache = _empty(fw, 6, 16, d)
    slots = np.arange(6) * 16          # a block for each row
    ref = O.cache_store(_host(cache), x.double().numpy(), x.flip(1).double().numpy(), slots)
    fw.cache_store(cache, x.cuda(), x.flip(1).cuda(), torch.tensor(slots).cuda())
    torch.cuda.synchronize()
    _same_cache(cache, ref)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_store_token_by_token_and_at_once(tf, dtype):
    """A prompt's rows at once, over many blocks and workgroup chunks; then tokens one call at a time."""
    torch, fw = tf
    rng = np.random.default_rng(4)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    d, bs, cells = 64, 16, 3
    cache = _empty(fw, 60, bs, d)
    N = [200, 33, 90]
    slots = _slots(rng, [(0, n + 20) for n in N], 60, bs)
    ends = np.cumsum([n + 20 for n in N])
    first = np.concatenate([np.arange(e - n - 20, e - 20) for e, n in zip(ends, N)])
    k, v = (torch.tensor(rng.standard_normal((len(slots), d)).astype(np.float32)).to(dt) for _ in range(2))
    ref = O.cache_store(_host(cache), k.double().numpy()[first], v.double().numpy()[first], slots[first])
    fw.cache_store(cache, k[first].cuda(), v[first].cuda(), torch.tensor(slots[first]).cuda())
    torch.cuda.synchronize()
    _same_cache(cache, ref)
    for s in range(20):
        at = ends - 20 + s
        ref = O.cache_store(dict(ref, d=d), k.double().numpy()[at] * 2.0 ** (s % 5), v.double().numpy()[at], slots[at])
        fw.cache_store(cache, (k[at] * 2.0 ** (s % 5)).cuda(), v[at].cuda(), torch.tensor(slots[at]).cuda())
    torch.cuda.synchronize()
    _same_cache(cache, ref)


def test_store_many_rows(tf):
    """Enough rows that a workgroup takes a chunk of them; sampled blocks against the oracle."""
    torch, fw = tf
    rng = np.random.default_rng(6)
    d, bs = 128, 64
    lens = rng.integers(1, 2000, 150)
    n_blocks = int(np.sum(-(-lens // bs)))
    slots = _slots(rng, [(0, int(n)) for n in lens], n_blocks, bs)
    N = len(slots)
    assert N > 2 * 2048 * 16
    g = torch.Generator(device="cuda").manual_seed(0)
    k, v = (torch.randn(N, d, generator=g, device="cuda").bfloat16() for _ in range(2))
    cache = fw.kv_cache(n_blocks, bs, d)
    fw.cache_store(cache, k, v, torch.tensor(slots).cuda())
    torch.cuda.synchronize()
    h = _host(cache)
    # every block, the fast way: its largest magnitude's exponent and torch's rounding
    b, off = slots // bs, slots % bs
    for name, x in (("k", k), ("v", v)):
        x = x.double().cpu().numpy()
        top = np.zeros(n_blocks)
        np.maximum.at(top, b, np.abs(x).max(1))
        e = np.ceil(np.log2(top / 448)).astype(int) + 127
        assert np.array_equal(h[name + "_exp"], e)
        want = torch.tensor(x * 2.0 ** (127 - e[b])[:, None]).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
        got = h["k"][b, off] if name == "k" else h["v"][b, :, off]
        assert np.array_equal(got, want), name


# ---------------------------------------------------------------------------
# attention over the cache
# ---------------------------------------------------------------------------

def _setup(tf, seed, S, T, Hkv, G, d, bs, lens, dtype, extra=0, garbage=True):
    torch, fw = tf
    rng = np.random.default_rng(seed)
    C = S * Hkv
    W = max(1, max(-(-int(n) // bs) for n in lens)) + extra
    n_blocks = sum(-(-int(n) // bs) for n in lens) + 2
    cache = _empty(fw, n_blocks, bs, d, seed=seed)
    table, at, ids = np.full((C, W), -1), 0, rng.permutation(n_blocks)
    for c, n in enumerate(lens):
        for j in range(-(-int(n) // bs)):
            table[c, j], at = ids[at], at + 1
    if garbage:              # what lies behind the last token: NaN codes
        for c, n in enumerate(lens):
            if n % bs:
                b = int(table[c, n // bs])
                cache.k[b, n % bs:, :] = 0x7F
                cache.v[b, :, n % bs:] = 0xFF
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    q = torch.tensor(rows(rng, (S, T, Hkv * G, d), False)).to(dt)
    return cache, table, q


def _attend(tf, cache, table, q, lens, dtype, scale=None, what=""):
    torch, fw = tf
    sc = None if scale is None else torch.tensor(scale, dtype=torch.float32, device="cuda")
    out = fw.cache_attention(q if q.is_cuda else q.cuda(), cache, _i32(torch, table), _i32(torch, lens), scale=sc)
    torch.cuda.synchronize()
    ref = O.cache_attention(q.double().cpu().numpy(), _host(cache), table, lens,
                            None if scale is None else np.float32(scale).astype(np.float64))
    n = max(int(x) for x in lens)
    w = check(out["o"].float().cpu().numpy(), out["lse"].cpu().numpy(), ref, dtype, cache.d, max(n, 1), what)
    record(f"decode {what}", o=w[0], lse=w[1])
    return out


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("bf16", 80), ("bf16", 1), ("bf16", 33), ("bf16", 192),
                                     ("bf16", 256), ("f32", 128), ("f32", 80), ("f32", 16), ("f32", 200), ("f32", 256)])
@pytest.mark.parametrize("T,G", [(1, 4), (3, 2), (5, 7)])
def test_decode_widths(tf, dtype, d, T, G):
    print(f"decode {dtype} d={d} T={T} G={G}", flush=True)
    lens = [1, 150, 64, 333]
    cache, table, q = _setup(tf, d + T, 2, T, 2, G, d, 64, lens, dtype)
    _attend(tf, cache, table, q, lens, dtype, what=f"{dtype} d={d} T={T} G={G}")


@pytest.mark.parametrize("bs", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_lengths_and_blocks(tf, bs, dtype):
    """Empty cells, one token, lengths at and beside every edge, more new positions than tokens."""
    lens = [0, 1, 2, 15, 16, 17, 63, 64, 65, 127, 129, 255, 256, 257, 400, 3]
    for T in (1, 4):
        print(f"decode lengths bs={bs} {dtype} T={T}", flush=True)
        cache, table, q = _setup(tf, bs, 4, T, 4, 3, 64, bs, lens, dtype)
        _attend(tf, cache, table, q, lens, dtype, what=f"lengths bs={bs} {dtype} T={T}")


@pytest.mark.parametrize("T,G", [(1, 1), (1, 8), (1, 16), (1, 17), (2, 8), (8, 4), (7, 8), (8, 8), (9, 8), (1, 70)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_rows(tf, T, G, dtype):
    """One to several row tiles of a cell."""
    print(f"decode rows T={T} G={G} {dtype}", flush=True)
    lens = [100, 37]
    cache, table, q = _setup(tf, T * G, 1, T, 2, G, 96, 32, lens, dtype)
    _attend(tf, cache, table, q, lens, dtype, what=f"rows T={T} G={G} {dtype}")


@pytest.mark.parametrize("dtype,d,T", [("bf16", 128, 1), ("bf16", 128, 3), ("f32", 64, 1), ("bf16", 64, 20)])
def test_decode_long_ragged_cells(tf, dtype, d, T):
    """Cells of very different lengths: parts on different workgroups, joined."""
    torch, fw = tf
    lens = [9000, 3, 0, 700, 2049, 512, 5000, 1]
    print(f"decode ragged {dtype} d={d} T={T}", flush=True)
    cache, table, q = _setup(tf, 3, 2, T, 4, 2, d, 64, lens, dtype, extra=5)
    out = _attend(tf, cache, table, q, lens, dtype, what=f"ragged {dtype} d={d} T={T}")
    assert out["_ws"] is not None


@pytest.mark.parametrize("scale", [[0.0, 0.5], [-0.3, 20.0]])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_scales(tf, scale, dtype):
    lens = [100, 200]
    cache, table, q = _setup(tf, 8, 1, 2, 2, 4, 64, 32, lens, dtype)
    _attend(tf, cache, table, q, lens, dtype, scale=scale, what=f"scale {scale} {dtype}")


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("f32", 32)])
@pytest.mark.parametrize("case", ["one long", "equal", "short and long", "all empty"])
def test_decode_shares_of_the_tiles(tf, dtype, d, case):
    """Workgroups that begin and end inside cells, at their edges, behind their tiles; cells in one part and in many."""
    rng = np.random.default_rng(7)
    S, Hkv = 40, 2
    lens = {"one long": [1] * 79 + [6000], "equal": [512] * 80, "short and long": [int(x) for x in rng.choice([0, 5, 64, 700, 2500], 80)],
            "all empty": [0] * 80}[case]
    print(f"shares {case} {dtype}", flush=True)
    extra = max(0, 2100 // 16 - max(lens) // 16)       # the table's row is long even where no cell is
    for T in (1, 3):
        cache, table, q = _setup(tf, 30 + T, S, T, Hkv, 2, d, 16, lens, dtype, extra=extra)
        out = _attend(tf, cache, table, q, lens, dtype, what=f"shares {case} {dtype} T={T}")
        assert out["_ws"] is not None


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_rising_logits(tf, dtype):
    """Scales at which the logits of later blocks exceed the first maximum by far."""
    torch, fw = tf
    lens = [700, 90]
    cache, table, q = _setup(tf, 31, 1, 1, 2, 4, 64, 16, lens, dtype)
    for c, n in enumerate(lens):
        for j in range(-(-n // 16)):
            cache.k_exp[int(table[c, j])] = 112 + min(j, 14)
    _attend(tf, cache, table, q, lens, dtype, what=f"rising {dtype}")


def test_decode_many_cells(tf):
    """More cells than threads of a workgroup."""
    rng = np.random.default_rng(0)
    S, Hkv = 75, 8
    lens = rng.integers(0, 90, S * Hkv)
    lens[77] = 1500
    cache, table, q = _setup(tf, 9, S, 1, Hkv, 2, 32, 16, lens, "bf16")
    _attend(tf, cache, table, q, lens, "bf16", what="many cells")


def test_decode_bad_pages_and_lengths(tf):
    """Blocks out of range are not seen; lengths beyond the table are clamped; negative ones are empty."""
    torch, fw = tf
    lens = [200, 100, 64, 48]
    cache, table, q = _setup(tf, 10, 2, 2, 2, 4, 64, 16, lens, "bf16")
    W = table.shape[1]
    table[0, 3], table[0, 7] = -1, 1 << 30
    table[1, :] = cache.k.shape[0]
    _attend(tf, cache, table, q, lens, "bf16", what="bad pages")
    wild = [1 << 30, -5, 64, 48]
    table[0, :] = np.arange(W) % cache.k.shape[0]
    _attend(tf, cache, table, q, wild, "bf16", what="wild lengths")
    # pages behind the last token are not looked at
    a = _attend(tf, cache, table, q, [30, 20, 10, 5], "bf16", what="short")
    table[0, 2:], table[1, 2:], table[2, 1:] = 99999, -99999, 7
    b = _attend(tf, cache, table, q, [30, 20, 10, 5], "bf16", what="short")
    assert torch.equal(a["o"], b["o"]) and torch.equal(a["lse"], b["lse"])


@pytest.mark.parametrize("dtype,G", [("bf16", 2), ("bf16", 7), ("f32", 2)])
def test_decode_nan_codes_reach_only_rows_that_see_them(tf, dtype, G):
    torch, fw = tf
    T, d = 4, 64
    lens = [70, 64]
    cache, table, q = _setup(tf, 11, 1, T, 2, G, d, 16, lens, dtype)
    clean = fw.cache_attention(q.cuda(), cache, _i32(torch, table), _i32(torch, lens))
    b = int(table[0, 68 // 16])
    cache.v[b, 5, 68 % 16] = 0x7F       # seen by the last two positions of the first cell
    got = fw.cache_attention(q.cuda(), cache, _i32(torch, table), _i32(torch, lens))
    torch.cuda.synchronize()
    hit = torch.zeros(got["o"].shape, dtype=torch.bool)
    hit[0, 2:, :G, 5] = True
    o, c = got["o"].cpu(), clean["o"].cpu()
    assert torch.equal(torch.isnan(o), hit)
    assert torch.equal(o[~hit], c[~hit]) and torch.equal(got["lse"], clean["lse"])
    cache.k[b, 69 % 16, 0] = 0xFF       # a key: the last position alone
    lost = fw.cache_attention(q.cuda(), cache, _i32(torch, table), _i32(torch, lens))["o"].cpu()
    assert torch.isnan(lost[0, 3, :G]).all() and torch.equal(lost[0, :2], c[0, :2]) and torch.equal(lost[0, :, G:], c[0, :, G:])


def test_decode_strided_queries(tf):
    torch, fw = tf
    S, T, Hkv, G, d = 3, 2, 2, 3, 80
    lens = [50, 80, 9, 33, 128, 1]
    for dtype in ("bf16", "f32"):
        cache, table, q = _setup(tf, 12, S, T, Hkv, G, d, 32, lens, dtype)
        wide = torch.zeros(T, S, Hkv * G + 3, d + 5, dtype=q.dtype, device="cuda")
        view = wide.transpose(0, 1)[:, :, 1:1 + Hkv * G, 3:3 + d]
        view.copy_(q.cuda())
        _attend(tf, cache, table, view, lens, dtype, what=f"strided {dtype}")


def test_decode_repeats_streams_graphs_and_no_lse(tf):
    torch, fw = tf
    for lens, W in (([3000, 17, 400, 0], 5), ([40, 17, 100, 0], 0)):
        cache, table, q = _setup(tf, 13, 2, 1, 2, 4, 128, 64, lens, "bf16", extra=W)
        q, t, n = q.cuda(), _i32(torch, table), _i32(torch, lens)
        a = fw.cache_attention(q, cache, t, n)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            b = fw.cache_attention(q, cache, t, n, want_lse=False)
        s.synchronize()
        assert b["lse"] is None and torch.equal(a["o"], b["o"])
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c = fw.cache_attention(q, cache, t, n)
        for r in range(3):           # lengths change between replays: nothing about them is on the host
            n.sub_(5 * r).clamp_(min=0)
            want = fw.cache_attention(q, cache, t, n)
            c["o"].zero_()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(want["o"], c["o"]) and torch.equal(want["lse"], c["lse"])


def test_cache_past_4_gib(tf):
    """Blocks whose bytes lie past 32-bit offsets."""
    torch, fw = tf
    bs, d = 256, 128
    n_blocks = (1 << 32) // (bs * d) + 40
    cache = fw.kv_cache(n_blocks, bs, d)
    last = [n_blocks - 1, n_blocks - 3, 5]
    rng = np.random.default_rng(14)
    n = 600
    slots = np.array([last[p // bs] * bs + p % bs for p in range(n)], np.int64)
    k, v = (torch.tensor(rng.standard_normal((n, d)).astype(np.float32)).bfloat16() for _ in range(2))
    fw.cache_store(cache, k.cuda(), v.cuda(), torch.tensor(slots).cuda())
    q = torch.tensor(rng.standard_normal((1, 1, 4, d)).astype(np.float32)).bfloat16()
    out = fw.cache_attention(q.cuda(), cache, _i32(torch, [last]), _i32(torch, [n]))
    torch.cuda.synchronize()
    small = fw.kv_cache(3, bs, d)
    for i, b in enumerate(last):
        for x, y in zip(small[:4], cache[:4]):
            x[i] = y[b]
    ref = O.cache_attention(q.double().numpy(), _host(small), [[0, 1, 2]], [n], None)
    check(out["o"].float().cpu().numpy(), out["lse"].cpu().numpy(), ref, "bf16", d, n)
    K, _, _ = O.cache_rows(_host(small), [0, 1, 2], n)
    assert np.all(np.abs(K - k.double().numpy()) <= 2.0 ** -4 * np.abs(k.double().numpy()) + 2.0 ** -9)


def test_cache_refusals(tf):
    torch, fw = tf
    cache = fw.kv_cache(4, 32, 64)
    q = torch.zeros(1, 1, 4, 64, dtype=torch.bfloat16, device="cuda")
    t, n = _i32(torch, [[0, 1], [2, 3]]), _i32(torch, [5, 6])
    x, s = torch.zeros(3, 64, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    fw.cache_attention(q, cache, t, n)
    calls = [lambda: fw.cache_attention(q.half(), cache, t, n), lambda: fw.cache_attention(q[..., :32], cache, t, n),
             lambda: fw.cache_attention(q, cache, t.long(), n), lambda: fw.cache_attention(q, cache, t, n[:1]),
             lambda: fw.cache_attention(q[:, :, :3], cache, t, n), lambda: fw.cache_attention(q, cache, t, n.cpu()),
             lambda: fw.cache_attention(q, cache._replace(v=cache.k[:, :, :32]), t, n),
             lambda: fw.cache_attention(q, cache._replace(k=cache.k.float()), t, n),
             lambda: fw.cache_attention(q, cache, t, n, scale=torch.ones(1, device="cuda")),
             lambda: fw.cache_store(cache, x, x, s.int()), lambda: fw.cache_store(cache, x, x[:2], s),
             lambda: fw.cache_store(cache, x[:, :32], x[:, :32], s), lambda: fw.cache_store(cache, x, x.bfloat16(), s),
             lambda: fw.block_tables(n, n, t, n, n[:1], 48, n_slots=0),
             lambda: fw.block_tables(n, n, t, n, n, 32, n_slots=0),
             lambda: fw.block_tables(n, n.long(), t, n, n[:1], 32, n_slots=0),
             lambda: fw.block_tables(n, n, t, n, n[:1], 32, n_slots=-1),
             lambda: fw.block_tables(n, n, t, n, n[:1], 32, n_slots=0, ws=torch.empty(1 << 20, dtype=torch.uint8)),
             lambda: fw.cache_attention(q, cache, t, n, ws=torch.empty(1 << 20, dtype=torch.uint8))]
    for i, f in enumerate(calls):
        with pytest.raises(fw.FwError):
            f()
            print("accepted", i)


# ---------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------

def test_prompt_eviction_cache_and_decoding(tf):
    """A prompt's attention, its window's scores, ContourKV's allocation, the kept rows into the 8-bit cache, and
    decoding steps over what each cell kept -- against float64 from the cache's own contents and, within the
    cache's 8 bits, from the rows that went in."""
    torch, fw = tf
    rng = np.random.default_rng(20)
    S, Hkv, G, d, n, bs = 2, 2, 4, 128, 400, 32
    Hq, C = Hkv * G, S * Hkv
    qkv = torch.tensor(rng.standard_normal((S * n, Hq + 2 * Hkv, d)).astype(np.float32)).bfloat16().cuda()
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    cu = torch.tensor([0, n, 2 * n], device="cuda")
    prompt = fw.prompt_attention(q, k, v, cu)
    # cells [sequence][head]: the last 16 positions' query rows score every key
    K = k.view(S, n, Hkv, d).transpose(1, 2).reshape(C, n, d).contiguous()
    V = v.view(S, n, Hkv, d).transpose(1, 2).reshape(C, n, d).contiguous()
    Q = q.view(S, n, Hkv, G, d)[:, -16:].permute(0, 2, 3, 1, 4).reshape(C, G * 16, d).contiguous()
    scores = fw.maxpool_scores(fw.dropped_mass_curve(Q, K)["importance"], 7)
    budget = C * 60
    kept = fw.ragged_compact(K, V, scores, budget, 8, Hkv)
    offsets = kept["offsets"]
    lens0 = torch.zeros(C, dtype=torch.int32, device="cuda")
    lens1 = (offsets[1:] - offsets[:-1]).int()
    table = torch.full((C, 20), -1, dtype=torch.int32, device="cuda")
    n_blocks = 40
    free, n_free = torch.randperm(n_blocks).int().cuda(), _i32(torch, [n_blocks])
    cache = fw.kv_cache(n_blocks, bs, d)
    up = fw.block_tables(lens0, lens1, table, free, n_free, bs, n_slots=budget)
    assert int(up["refused"]) == 0 and torch.equal(up["offsets"], offsets)
    fw.cache_store(cache, kept["k_out"], kept["v_out"], up["slots"])
    lens, stored = up["lens"], []
    for step in range(3):
        x = torch.tensor(rng.standard_normal((S, 1, Hq + 2 * Hkv, d)).astype(np.float32)).bfloat16().cuda()
        one = fw.block_tables(lens, lens + 1, table, free, n_free, bs, n_slots=C)
        fw.cache_store(cache, x[:, 0, Hq:Hq + Hkv].reshape(C, d), x[:, 0, Hq + Hkv:].reshape(C, d), one["slots"])
        lens = one["lens"]
        stored.append(x)
        out = fw.cache_attention(x[:, :, :Hq], cache, table, lens)
    torch.cuda.synchronize()
    ref = O.cache_attention(x[:, :, :Hq].double().cpu().numpy(), _host(cache), table.cpu().numpy(), lens.cpu().numpy(), None)
    check(out["o"].float().cpu().numpy(), out["lse"].cpu().numpy(), ref, "bf16", d, n, "end to end")
    # what each cell holds is what it kept, then the new rows
    kp, off = kept["kept_pos"].cpu().numpy(), offsets.cpu().numpy()
    for c in range(C):
        Kc, Vc, ok = O.cache_rows(_host(cache), table[c].cpu().numpy(), int(lens[c]))
        want = torch.cat([K[c][kp[off[c]:off[c + 1]]]] + [y[c // Hkv, :, Hq + c % Hkv] for y in stored]).double().cpu().numpy()
        assert ok.all() and np.all(np.abs(Kc - want) <= 2.0 ** -4 * np.abs(want) + 2.0 ** -8)
    # the prompt's own last rows, for the tokens that were kept or not, come from the full keys
    r = O.attend(q[n - 1, :G].double().cpu().numpy(), K[0].double().cpu().numpy(), V[0].double().cpu().numpy(), d ** -0.5, [n] * G)
    check(prompt["o"][n - 1, :G].float().cpu().numpy(), prompt["lse"][n - 1, :G].cpu().numpy(), r, "bf16", d, n)
    # the request ends: every block comes back
    fw.block_tables(lens, torch.zeros_like(lens), table, free, n_free, bs, n_slots=0)
    assert int(n_free) == n_blocks and torch.equal(free.sort().values, torch.arange(n_blocks, device="cuda").int())
    assert torch.all(table == -1)
