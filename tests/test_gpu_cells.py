"""fw_cache_fork, fw_cache_release and fw_cache_compact against the oracle, alone and together with the calls around
them."""
import numpy as np
import pytest

from oracle import cells as O
from oracle import serving as V
from tests.cells import compare, random_state

pytestmark = pytest.mark.gpu
CACHE = ("k", "v", "k_exp", "v_exp")


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


def _i32(torch, x):
    return None if x is None else _cuda(torch, x, torch.int32)


def _up(tf, s):
    torch, fw = tf
    cache = fw.KvCache(*(_cuda(torch, s[key]) for key in CACHE), s["d"])
    cells = fw.CacheCells(_i32(torch, s["table"]), _i32(torch, s["lens"]), _i32(torch, s["free_list"]),
                          _i32(torch, [s["n_free"]]), _i32(torch, s["shared"]))
    return cache, cells


def _down(cache, cells):
    n = lambda x: x.cpu().numpy()
    return dict(k=n(cache.k), v=n(cache.v), k_exp=n(cache.k_exp), v_exp=n(cache.v_exp), d=cache.d, table=n(cells.table),
                lens=n(cells.lens), free_list=n(cells.free_list), n_free=int(cells.n_free), shared=n(cells.shared))


def _fork(tf, s, src, dst, length=None):
    torch, fw = tf
    cache, cells = _up(tf, s)
    r = fw.cache_fork(cache, cells, _i32(torch, src), _i32(torch, dst), length=_i32(torch, length))
    torch.cuda.synchronize()
    want = O.fork(s, src, dst, length)
    compare(_down(cache, cells), want, s, "fork")
    assert int(r["refused"]) == want["refused"]
    O.invariants(want)
    return want


def _release(tf, s, new_len):
    torch, fw = tf
    cache, cells = _up(tf, s)
    r = fw.cache_release(cache, cells, _i32(torch, new_len))
    torch.cuda.synchronize()
    want = O.release(s, new_len)
    compare(_down(cache, cells), want, s, "release")
    assert int(r["refused"]) == want["refused"]
    O.invariants(want)
    return want


def _compact(tf, s, offsets, pos, which=None):
    torch, fw = tf
    cache, cells = _up(tf, s)
    r = fw.cache_compact(cache, cells, _cuda(torch, offsets, torch.int64), _i32(torch, pos), which=_i32(torch, which))
    torch.cuda.synchronize()
    want = O.compact(s, offsets, pos, which)
    compare(_down(cache, cells), want, s, "compact")
    assert int(r["refused"]) == want["refused"]
    O.invariants(want)
    return want


def _some(rng, s, cells, part=0.5, prefix=0.3):
    """Random kept positions of these cells; some keep a run at their front, some nothing."""
    pos, off = [], [0]
    for c in cells:
        n = int(s["lens"][c])
        k = int(round(n * part * rng.uniform(0, 2)))
        if rng.random() < prefix:
            got = list(range(min(k, n)))
        else:
            got = sorted(rng.permutation(n)[:min(k, n)].tolist())
        pos += got
        off.append(len(pos))
    return off, pos


SIZES = [(16, 20, 32), (32, 64, 64), (16, 80, 96), (64, 128, 128), (128, 160, 192), (256, 256, 256), (16, 256, 256), (256, 20, 32)]


@pytest.mark.parametrize("bs,d,dp", SIZES)
@pytest.mark.parametrize("spread", [3, 60])
def test_compact_widths_and_blocks(tf, bs, d, dp, spread):
    print(f"compact bs={bs} d={d} spread={spread}", flush=True)
    rng = np.random.default_rng(bs + d + spread)
    s = random_state(rng, [0, 1, bs, 2 * bs + 1, 3 * bs, 5 * bs - 1], bs, dp, d, spread=spread)
    cells = range(6)
    for part, prefix in ((0.5, 0.3), (0.05, 0.0), (1.0, 1.0), (0.9, 0.0)):
        _compact(tf, s, *_some(rng, s, cells, part, prefix))


def test_compact_by_hand(tf):
    rng = np.random.default_rng(1)
    s = random_state(rng, [40, 64, 17], 16, 32, 20)
    _compact(tf, s, [0, 0, 0, 0], [])                                        # everything goes
    _compact(tf, s, [0, 40, 104, 121], [*range(40), *range(64), *range(17)])  # everything stays
    _compact(tf, s, [0, 1, 2, 3], [39, 63, 16])                              # the last token alone
    _compact(tf, s, [0, 39, 102, 118], [*range(1, 40), *range(1, 64), *range(1, 17)])
    _compact(tf, s, [0, 20], list(range(10, 30)), which=[1])
    _compact(tf, s, [0, 3, 5, 6], [1, 2, 3, 7, 9, 4], which=[2, 0, 1])
    _compact(tf, s, [0], [])                                                 # no cell listed


def test_compact_refusals_on_the_device(tf):
    rng = np.random.default_rng(2)
    s = random_state(rng, [40, 64, 17], 16, 32, 20)
    for off, pos, which in (([0, 2, 3, 4], [5, 5, 1, 2], None), ([0, 2, 3, 4], [5, 4, 1, 2], None),
                            ([0, 2, 3, 4], [-1, 4, 1, 2], None), ([0, 2, 3, 4], [39, 40, 1, 2], None),
                            ([0, 2, 3, 5], [1, 4, 63, 2, 2 ** 30], None), ([0, 2, 3, 9], [1, 4, 63, 2], None),
                            ([-3, 2, 3, 4], [1, 4, 63, 2], None), ([0, 3, 2, 4], [1, 4, 5, 2], None),
                            ([0, 2 ** 40, 3, 4], [1, 4, 5, 2], None), ([0, 2, 3, 4], [1, 4, 5, 2], [1, 1, 0]),
                            ([0, 2, 3, 4], [1, 4, 5, 2], [3, -1, 0]), ([0, 2, 3, 4], [1, 4, 5, 2], [2 ** 30, -2 ** 31, 2]),
                            ([0, 65], list(range(65)), [1])):
        _compact(tf, s, off, pos, which)


def test_compact_where_values_become_subnormal_or_are_not_numbers(tf):
    """Blocks whose exponents differ by much meet in one block; NaN codes, zeros, the least and largest exponents."""
    rng = np.random.default_rng(3)
    s = random_state(rng, [64, 64, 48], 16, 32, 32)
    s["k_exp"][s["table"][0, :4]] = [100, 110, 107, 119]
    s["v_exp"][s["table"][0, :4]] = [253, 1, 130, 240]
    s["k_exp"][s["table"][1, :4]] = [1, 2, 3, 9]
    s["k"][s["table"][0, 1], 3, 5], s["v"][s["table"][0, 2], 7, 4] = 0x7F, 0xFF
    s["k"][s["table"][2, 1]] = 0
    s["v"][s["table"][2, 1]] = 0x80
    s["k"][s["table"][2, 2]] = 0x7F
    pos = [*range(1, 64, 3), *range(2, 64, 2), *range(17, 48)]
    _compact(tf, s, [0, 21, 52, 83], pos)


@pytest.mark.parametrize("bs,d,dp", SIZES)
def test_fork_and_release(tf, bs, d, dp):
    print(f"fork bs={bs} d={d}", flush=True)
    rng = np.random.default_rng(bs + d)
    s = random_state(rng, [0, 1, bs, 2 * bs + 1, 3 * bs - 1] + [0] * 9, bs, dp, d, n_blocks=30)
    s = _fork(tf, s, [1, 2, 3, 4, 3, 0], [5, 6, 7, 8, 9, 10])
    s = _fork(tf, s, [7, 8, 3], [11, 12, 13], length=[bs + 1, 2 * bs, -1])   # cells that share go on
    s = _release(tf, s, [0, 0, bs - 1, bs + 3, 99999, 1, 0, -5, bs, 2 * bs, 0, 1, 5, 7])
    s = _release(tf, s, [0] * 14)
    assert s["n_free"] == 30


def test_fork_refusals(tf):
    rng = np.random.default_rng(4)
    s = random_state(rng, [20, 33, 16, 0, 0, 0, 0, 0], 16, 32, 20, n_blocks=8)
    assert s["n_free"] == 2
    _fork(tf, s, [0, 1, 0, 2], [3, 4, 5, 6])            # two copies are left, the third is refused, the fourth needs none
    _fork(tf, s, [0, 0, 2], [3, 3, 3])                  # one cell three times
    _fork(tf, s, [0, 2, 7], [1, 2, 7])                  # cells that hold tokens; an empty cell that continues itself
    _fork(tf, s, [3, 0, 4], [4, 3, 5])                  # cells empty before the call are empty to all its pairs
    _fork(tf, s, [-1, 8, 0, 0], [3, 3, -1, 8])
    _fork(tf, s, [2 ** 31 - 1, 0], [3, -2 ** 31])
    _fork(tf, s, [], [])


def test_release_when_nothing_is_left(tf):
    rng = np.random.default_rng(5)
    s = random_state(rng, [40, 0, 0, 0], 16, 32, 20, n_blocks=5)
    s = _fork(tf, s, [0, 0], [1, 2])
    assert s["n_free"] == 0
    r = _release(tf, s, [20, 25, 40, 0])                # no block for either copy: both stay
    assert r["refused"] == 2
    r = _release(tf, s, [32, 0, 40, 0])                 # no copies needed
    assert r["refused"] == 0 and r["n_free"] == 2


def test_compaction_of_shared_cells(tf):
    rng = np.random.default_rng(6)
    s = random_state(rng, [100, 0, 0, 50, 0], 16, 32, 20, n_blocks=40)
    s = _fork(tf, s, [0, 0, 3], [1, 2, 4])
    a = _compact(tf, s, *_some(rng, s, range(5), 0.5, 0.0))
    _compact(tf, a, *_some(rng, a, range(5), 0.7, 0.5))
    off, pos = [0, 20, 60], [*range(20), *range(30, 70)]  # a part-filled block that stays, and others' blocks
    _compact(tf, s, off, pos, which=[0, 2])
    tight = random_state(rng, [100, 0], 16, 32, 20, n_blocks=9)
    tight = _fork(tf, tight, [0], [1])
    assert tight["n_free"] == 1
    r = _compact(tf, tight, [0, 40, 50], [*range(50, 90), *range(10, 20)])
    assert r["refused"] == 2                            # three blocks are too many; with one more they still are
    r = _compact(tf, tight, [0, 10, 50], [*range(10, 20), *range(50, 90)])
    assert r["refused"] == 1


@pytest.mark.parametrize("seed", range(8))
def test_any_calls_in_a_row(tf, seed):
    rng = np.random.default_rng(200 + seed)
    C, W = 12, 7
    bs, d, dp = SIZES[seed % 4]
    s = random_state(rng, [int(rng.integers(0, W * bs)) if c < 5 else 0 for c in range(C)], bs, dp, d, W=W, n_blocks=48)
    for i in range(8):
        what = rng.integers(0, 3)
        if what == 0:
            P = int(rng.integers(1, 7))
            s = _fork(tf, s, rng.integers(-1, C + 1, P), rng.integers(-1, C + 1, P),
                      None if rng.random() < 0.5 else rng.integers(-1, W * bs, P))
        elif what == 1:
            s = _release(tf, s, np.where(rng.random(C) < 0.4, rng.integers(0, W * bs, C), 9999))
        else:
            which = rng.permutation(C)[:int(rng.integers(1, C + 1))]
            s = _compact(tf, s, *_some(rng, s, which, 0.6), which=which)


@pytest.mark.parametrize("C,top", [(1, 3000), (700, 40), (1100, 17), (40, 400)])
def test_many_and_long_cells(tf, C, top):
    rng = np.random.default_rng(C)
    lens = rng.integers(0, top + 1, C)
    lens[-1] = top
    s = random_state(rng, lens.tolist() + [0] * C, 16, 32, 4, n_blocks=None)
    s["d"] = 4
    room = s["n_free"]
    t = random_state(rng, lens.tolist() + [0] * C, 16, 32, 4, n_blocks=len(s["shared"]) + C - room + 3)
    t = _fork(tf, t, np.arange(C), np.arange(C, 2 * C))
    t = _compact(tf, t, *_some(rng, t, range(C), 0.4))
    _release(tf, t, np.where(np.arange(2 * C) % 3 == 0, 0, rng.integers(0, top + 1, 2 * C)))


def test_more_blocks_than_one_run(tf):
    """Marked blocks in several runs of the collection."""
    rng = np.random.default_rng(7)
    s = random_state(rng, [16 * 300] * 50 + [0], 16, 32, 4, n_blocks=20000)
    _release(tf, s, rng.integers(0, 16 * 300, 51))
    s = _fork(tf, s, [3], [50])
    _release(tf, s, [0] * 51)


def test_blocks_that_are_none_do_no_harm(tf):
    """Entries out of range are left alone: nothing is read or written through them."""
    torch, fw = tf
    rng = np.random.default_rng(8)
    s = random_state(rng, [60, 60, 60, 0], 16, 32, 20, W=5)
    s["table"][0, 1], s["table"][1, 2], s["table"][2, 3] = -1, 10 ** 8, -9
    cache, cells = _up(tf, s)
    pos = torch.arange(1, 60, 2, dtype=torch.int32, device="cuda")
    fw.cache_compact(cache, cells, _cuda(torch, [0, 30], torch.int64), pos, which=_i32(torch, [0]))
    fw.cache_fork(cache, cells, _i32(torch, [1]), _i32(torch, [3]))
    fw.cache_release(cache, cells, _i32(torch, [3, 20, 50, 0]))
    torch.cuda.synchronize()
    got = _down(cache, cells)
    free = got["free_list"][:got["n_free"]]
    assert len(set(free.tolist())) == len(free) and free.min() >= 0 and free.max() < len(s["shared"])


@pytest.mark.parametrize("seed", range(4))
def test_what_entries_out_of_range_stand_for(tf, seed):
    """Tokens of such a block are zeros, what goes to one is lost, and it is never copied, counted or freed: as if each
    were a block of its own, of zeros, that nobody looks at afterwards.  All other blocks hold what they then would."""
    torch, fw = tf
    rng = np.random.default_rng(300 + seed)
    s = random_state(rng, [60, 60, 60, 0, 75], 16, 32, 20, W=5)
    n = len(s["shared"])
    bad = (0, 1, -1), (1, 2, 10 ** 8), (2, 3, -9), (4, 0, n), (4, 4, 2 ** 31 - 1)
    t = dict(s, table=s["table"].copy())
    more = lambda x, fill: np.concatenate([x, np.full((len(bad), *x.shape[1:]), fill, x.dtype)])
    for key, fill in (("k", 0), ("v", 0), ("k_exp", 1), ("v_exp", 1), ("shared", 0), ("free_list", -7)):
        t[key] = more(s[key], fill)
    for i, (c, j, b) in enumerate(bad):
        s["table"][c, j], t["table"][c, j] = b, n + i
    cache, cells = _up(tf, s)

    def check(want, was, r, what):
        torch.cuda.synchronize()
        got = _down(cache, cells)
        assert int(r["refused"]) == want["refused"] == 0, what
        cut = lambda x: dict(x, **{key: x[key][:n] for key in (*CACHE, "shared")})
        free = [b for b in want["free_list"][:want["n_free"]] if b < n]
        table = want["table"].copy()
        for i, (_, _, b) in enumerate(bad):
            table[table == n + i] = b
        compare(got, dict(cut(want), table=table, free_list=np.array(free), n_free=len(free)), cut(was), what)

    def again(x):
        """The stand-ins as the next call would read them: zeros, none of them free or shared."""
        free = [b for b in x["free_list"][:x["n_free"]] if b < n]
        x = dict(x, free_list=np.array(free + [-7] * (n + len(bad) - len(free)), np.int32), n_free=len(free))
        for key, fill in (("k", 0), ("v", 0), ("k_exp", 1), ("v_exp", 1), ("shared", 0)):
            x[key][n:] = fill
        return x

    off, pos = _some(rng, s, [0, 2, 4], 0.5, 0.0)
    r = fw.cache_compact(cache, cells, _cuda(torch, off, torch.int64), _i32(torch, pos), which=_i32(torch, [0, 2, 4]))
    a = O.compact(t, off, pos, [0, 2, 4])
    check(a, t, r, "compact")
    r = fw.cache_fork(cache, cells, _i32(torch, [1]), _i32(torch, [3]))
    a = again(a)
    b = O.fork(a, [1], [3])
    check(b, a, r, "fork")
    end = [3, 20, 50, 33, 17]
    r = fw.cache_release(cache, cells, _i32(torch, end))
    b = again(b)
    check(O.release(b, end), b, r, "release")


def test_the_loop_as_it_is_used(tf):
    """A prompt's keys turn, are stored, attended and scored; the cells are compacted, forked, grow and end."""
    torch, fw = tf
    g = torch.Generator(device="cuda").manual_seed(9)
    S, Hkv, G, d, bs, n = 2, 2, 2, 64, 16, 150
    C, Hq, blocks = S * Hkv, Hkv * G, 120
    rnd = lambda *x: torch.randn(*x, generator=g, device="cuda").bfloat16()
    cache, cells = fw.kv_cache(blocks, bs, d), fw.cache_cells(2 * C, 16, blocks)
    freq = 10000.0 ** (-torch.arange(0, d, 2, device="cuda") / d)
    q, k, v = rnd(S * n, Hq, d), rnd(S * n, Hkv, d), rnd(S * n, Hkv, d)
    pos = torch.arange(n, device="cuda").repeat(S)
    r = fw.rotate_heads(q, k, pos, freq, eps=1e-6)
    grow = lambda new, m: fw.block_tables(cells.lens, new, cells.table, cells.free_list, cells.n_free, bs, n_slots=m,
                                          lens=cells.lens)
    new = torch.tensor([n] * C + [0] * C, dtype=torch.int32, device="cuda")
    up = grow(new, C * n)
    by_cell = lambda x: x.view(S, n, Hkv, d).transpose(1, 2).reshape(C * n, d).contiguous()
    fw.cache_store(cache, by_cell(r["k"]), by_cell(v), up["slots"])
    first = cells._replace(table=cells.table[:C], lens=cells.lens[:C])
    win = r["q"].view(S, n, Hq, d)[:, n - 8:].contiguous()
    att = fw.cache_attention(win, cache, first.table, first.lens)
    sc = fw.cache_scores(win, cache, first.table, first.lens, att["lse"])["scores"]
    # every row that sees something gives its weights away whole: eight rows of each sequence's heads
    assert torch.allclose(sc.sum(1), torch.ones(C, device="cuda"), atol=1e-3)
    keep = torch.tensor([40, 50, 150, 7], dtype=torch.int32, device="cuda")
    sel = fw.cache_select(sc, first.lens, keep, recent=8, n_kept=247)
    before = _down(cache, cells)
    assert int(fw.cache_compact(cache, cells, sel["offsets"], sel["kept_pos"], which=torch.arange(C, dtype=torch.int32, device="cuda"))["refused"]) == 0
    after = _down(cache, cells)
    off, kept = sel["offsets"].tolist(), sel["kept_pos"].tolist()
    compare(after, O.compact(before, off, kept, range(C)), before, "compact")
    # attention over what is left, against the tokens as they were chosen
    att = fw.cache_attention(win[:, 7:], cache, first.table, first.lens)
    for c in range(C):
        K, V_, _ = V.cache_rows(after, after["table"][c], len(kept[off[c]:off[c + 1]]))
        o = V.attend(win[c // Hkv, 7, (c % Hkv) * G:(c % Hkv + 1) * G].double().cpu().numpy(), K, V_, d ** -0.5, [len(K)] * G)["o"]
        got = att["o"][c // Hkv, 0, (c % Hkv) * G:(c % Hkv + 1) * G].double().cpu().numpy()
        assert np.all(np.abs(got - o) <= 2.0 ** -7 * np.abs(o) + 1e-3)
    # two continuations of each sequence: the new cells share, grow by a token of their own, and end
    src = torch.arange(C, dtype=torch.int32, device="cuda")
    assert int(fw.cache_fork(cache, cells, src, src + C)["refused"]) == 0
    up = grow(cells.lens + 1, 2 * C)
    fw.cache_store(cache, rnd(2 * C, d), rnd(2 * C, d), up["slots"])
    s = _down(cache, cells)
    O.invariants(s)
    for c in range(C):
        a, b = V.cache_rows(s, s["table"][c], int(s["lens"][c]))[0], V.cache_rows(s, s["table"][C + c], int(s["lens"][c]))[0]
        assert np.array_equal(a[:-1 - (len(a) - 1) % bs], b[:-1 - (len(a) - 1) % bs]) and not np.array_equal(a[-1], b[-1])
    fw.cache_release(cache, cells, torch.zeros(2 * C, dtype=torch.int32, device="cuda"))
    assert int(cells.n_free) == blocks and not cells.shared.any()


def test_captured(tf):
    """A step that forks, compacts and releases, captured once and replayed on other contents and lengths."""
    torch, fw = tf
    rng = np.random.default_rng(10)
    s = random_state(rng, [100, 80, 0, 0], 16, 32, 20, n_blocks=30)
    cache, cells = _up(tf, s)
    src, dst = _i32(torch, [0, 1]), _i32(torch, [2, 3])
    which = _i32(torch, [2, 3])
    off = _cuda(torch, [0, 30, 55], torch.int64)
    pos = _i32(torch, [*range(3, 93, 3), *range(0, 75, 3)])
    end = _i32(torch, [9999, 9999, 0, 0])

    def step():
        return (fw.cache_fork(cache, cells, src, dst), fw.cache_compact(cache, cells, off, pos, which=which),
                fw.cache_release(cache, cells, end))
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    for i in range(4):
        s = _down(cache, cells)
        cells.lens[0] -= 0
        end[2] = 20 * (i % 2)
        g.replay()
        torch.cuda.synchronize()
        want = O.release(O.compact(O.fork(s, [0, 1], [2, 3]), off.tolist(), pos.tolist(), [2, 3]), end.tolist())
        got = _down(cache, cells)
        for key in ("table", "lens", "shared", "n_free"):
            assert np.array_equal(got[key], want[key]), (i, key)
        assert [int(x["refused"]) for x in out][2] == 0
        fw.cache_release(cache, cells, _i32(torch, [9999, 9999, 0, 0]))


@pytest.mark.parametrize("more", [1, 300, 200000])
def test_more_room_than_is_kept(tf, more):
    """kept_pos as cache_select leaves it where n_kept is an upper bound: -1 behind the last cell's, here also before the
    first one's."""
    rng = np.random.default_rng(17)
    s = random_state(rng, [600, 0, 33, 280, 0], 16, 32, 20, n_blocks=70)
    s = _fork(tf, s, [0], [4])
    off, pos = _some(rng, s, range(5), 0.6, 0.0)
    for before in (0, more):
        _compact(tf, s, [before + x for x in off], [-1] * before + pos + [-1] * more)
    which = [4, 2]
    off, pos = _some(rng, s, which, 0.6, 0.0)
    _compact(tf, s, off, pos + [-1] * more, which)


def test_captured_and_replayed_on_other_states(tf):
    """A step that forks, compacts and releases, captured once and replayed on other lengths, tables, codes, exponents,
    pairs and positions, some of which are refused."""
    torch, fw = tf
    rng = np.random.default_rng(16)
    dims = dict(bs=16, dp=32, d=20, W=8, n_blocks=30)
    plan = [([100, 80, 0, 0], [0, 1], [2, 3], [2, 3], [9999, 9999, 0, 0]),
            ([64, 17, 0, 0], [1, 0], [2, 3], [3, 2], [20, 9999, 5, 16]),
            ([120, 128, 0, 9], [0, 1], [2, 3], [2, 0], [64, 33, 9999, 0]),       # the second pair's cell holds tokens
            ([31, 100, 0, 0], [0, 0], [2, 2], [1, 2], [0, 48, 9999, 7]),         # one cell twice
            ([100, 80, 0, 0], [1, 5], [3, 2], [3, 3], [99, 80, 0, 11])]          # a cell that is none, a cell listed twice
    make = lambda lens: random_state(rng, lens, dims["bs"], dims["dp"], dims["d"], W=dims["W"], n_blocks=dims["n_blocks"])
    s = make(plan[0][0])
    cache, cells = _up(tf, s)
    arrays = dict(zip(CACHE, cache[:4]), table=cells.table, lens=cells.lens, free_list=cells.free_list, shared=cells.shared)
    src, dst, which, end = (_i32(torch, x) for x in plan[0][1:])
    off, pos = _cuda(torch, [0, 30, 55], torch.int64), _i32(torch, [*range(3, 93, 3), *range(0, 75, 3)])

    def step():
        return (fw.cache_fork(cache, cells, src, dst), fw.cache_compact(cache, cells, off, pos, which=which),
                fw.cache_release(cache, cells, end))
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    refusals = 0
    for i, (lens, *now) in enumerate(plan + plan[::-1]):
        s = make(lens)
        for key, x in arrays.items():
            x.copy_(_cuda(torch, s[key]))
        cells.n_free.fill_(s["n_free"])
        for x, y in zip((src, dst, which, end), now):
            x.copy_(_i32(torch, y))
        a = O.fork(s, *now[:2])
        cut = int(rng.integers(20, 36))
        kept = [sorted(rng.permutation(max(m, int(a["lens"][c])))[:m].tolist()) for c, m in zip(now[2], (cut, 55 - cut))]
        off.copy_(_cuda(torch, [0, cut, 55]))
        pos.copy_(_i32(torch, kept[0] + kept[1]))
        g.replay()
        torch.cuda.synchronize()
        b = O.compact(a, [0, cut, 55], kept[0] + kept[1], now[2])
        c = O.release(b, now[3])
        compare(_down(cache, cells), c, s, f"replay {i}")
        assert [int(x["refused"]) for x in out] == [x["refused"] for x in (a, b, c)], i
        refusals += a["refused"] + b["refused"] + c["refused"]
    assert refusals


@pytest.mark.parametrize("off", [[0, 256 * 10 ** 6, 256 * 10 ** 6, 256 * 10 ** 6], [0, 2, 2 ** 33, 2 ** 40], [-2 ** 62, -2 ** 40, -7, -1],
                                 [-2 ** 50, 0, 2, 4], [2 ** 62] * 4, [1, 2, 4, 4], [4, 4, 4, 4], [0, 1, 300000, 300001]])
def test_offsets_out_of_range(tf, off):
    """Ascending offsets that lie anywhere: their cells are refused, and the others served."""
    print(f"compact offsets={off}", flush=True)
    s = random_state(np.random.default_rng(13), [40, 64, 17], 16, 32, 20)
    _compact(tf, s, off, [3, 9, 1, 2])


def test_many_pairs_and_listed_cells(tf):
    """More cells than claims fit LDS, and more pairs than are asked for once."""
    rng = np.random.default_rng(14)
    C = 10000
    lens = np.zeros(C, int)
    lens[:40] = rng.integers(0, 60, 40)
    s = random_state(rng, lens, 16, 32, 4, n_blocks=6500)
    dst = 40 + rng.permutation(C - 40)[:5000]
    dst[[7, 4000, 4999]] = dst[6], dst[100], 3
    s = _fork(tf, s, rng.integers(0, 40, 5000), dst, rng.integers(-1, 70, 5000))
    which = rng.permutation(C)[:4500]
    which[[4200, 4300]] = which[2], C
    kept = [min(2, int(s["lens"][c])) if c < C else 1 for c in which]
    pos = [x for c, n in zip(which, kept) for x in sorted(rng.permutation(max(1, int(s["lens"][c]) if c < C else 1))[:n].tolist())]
    s = _compact(tf, s, np.cumsum([0] + kept).tolist(), pos, which)
    s = _release(tf, s, rng.integers(0, 40, C))
    _release(tf, s, [0] * C)


def test_a_stack_of_many_runs(tf):
    """Blocks whose numbers lie in more runs than are counted on the way."""
    torch, fw = tf
    rng = np.random.default_rng(15)
    n, lens = 300000, [500, 320, 33, 0, 0]
    s = random_state(rng, lens, 16, 32, 20)
    few = len(s["shared"])
    at = np.sort(rng.permutation(n)[:few])         # where the small cache's blocks lie in the large one
    t = dict(s, n_free=n - few + s["n_free"], shared=np.zeros(n, np.int32))
    for key in CACHE:
        t[key] = np.zeros((n, *s[key].shape[1:]), np.uint8)
        t[key][at] = s[key]
    rest = np.setdiff1d(np.arange(n), at)
    t["table"] = np.where(s["table"] >= 0, at[s["table"]], -1).astype(np.int32)
    t["free_list"] = np.full(n, -7, np.int32)
    t["free_list"][:t["n_free"]] = np.concatenate([rest, at[s["free_list"][:s["n_free"]]]])
    cache, cells = _up(tf, t)
    calls = (("fork", lambda: fw.cache_fork(cache, cells, _i32(torch, [0, 1]), _i32(torch, [3, 4])), lambda x: O.fork(x, [0, 1], [3, 4])),
             ("compact", lambda: fw.cache_compact(cache, cells, _cuda(torch, [0, 60, 90], torch.int64),
                                                  _i32(torch, [*range(2, 122, 2), *range(30)]), which=_i32(torch, [0, 2])),
              lambda x: O.compact(x, [0, 60, 90], [*range(2, 122, 2), *range(30)], [0, 2])),
             ("release", lambda: fw.cache_release(cache, cells, _i32(torch, [10, 300, 0, 123, 0])),
              lambda x: O.release(x, [10, 300, 0, 123, 0])),
             ("end", lambda: fw.cache_release(cache, cells, _i32(torch, [0] * 5)), lambda x: O.release(x, [0] * 5)))
    for what, run, oracle in calls:
        r = run()
        torch.cuda.synchronize()
        want, got = oracle(t), _down(cache, cells)
        assert int(r["refused"]) == want["refused"] == 0
        used = np.unique(np.concatenate([at, want["table"][want["table"] >= 0]]))
        other = np.setdiff1d(np.arange(n), used)
        for x in (got, want, t):
            assert not x["k"][other].any() and not x["v"][other].any()
        small = lambda x: dict(x, k=x["k"][used], v=x["v"][used], k_exp=x["k_exp"][used], v_exp=x["v_exp"][used])
        compare(small(got), small(want), small(t), what)
        O.invariants(want)
        at, t = used, want


def test_two_streams_with_workspaces_of_their_own(tf):
    torch, fw = tf
    rng = np.random.default_rng(11)
    states = [random_state(rng, [300, 200, 0, 0], 16, 32, 20, n_blocks=60) for _ in range(2)]
    ups = [_up(tf, s) for s in states]
    streams = [torch.cuda.Stream() for _ in range(2)]
    src, dst, end = _i32(torch, [0, 1]), _i32(torch, [2, 3]), _i32(torch, [100, 9999, 50, 0])
    torch.cuda.synchronize()
    for (cache, cells), st in zip(ups, streams):
        with torch.cuda.stream(st):
            fw.cache_fork(cache, cells, src, dst)
            fw.cache_release(cache, cells, end)
    torch.cuda.synchronize()
    for s, (cache, cells) in zip(states, ups):
        want = O.release(O.fork(s, [0, 1], [2, 3]), [100, 9999, 50, 0])
        compare(_down(cache, cells), want, s, "streams")


def test_refusals(tf):
    torch, fw = tf
    rng = np.random.default_rng(12)
    s = random_state(rng, [60, 20, 0], 16, 32, 20)
    cache, cells = _up(tf, s)
    i = _i32(torch, [0, 1, 2])
    off = _cuda(torch, [0, 1, 2, 3], torch.int64)
    for f in (lambda: fw.cache_fork(cache, cells, i, i[:2]), lambda: fw.cache_fork(cache, cells, i.long(), i),
              lambda: fw.cache_fork(cache, cells, i, i, length=i[:1]), lambda: fw.cache_fork(cache, cells, i.cpu(), i),
              lambda: fw.cache_release(cache, cells, i[:2]), lambda: fw.cache_release(cache, cells, i.float()),
              lambda: fw.cache_compact(cache, cells, off.int(), i), lambda: fw.cache_compact(cache, cells, off, i.long()),
              lambda: fw.cache_compact(cache, cells, off, i, which=i[:2]),
              lambda: fw.cache_compact(cache, cells, _cuda(torch, [0, 0, 0, 0, 0], torch.int64), i),
              lambda: fw.cache_compact(cache, cells._replace(table=cells.table.t()), off, i),
              lambda: fw.cache_compact(cache, cells._replace(free_list=cells.free_list[1:]), off, i),
              lambda: fw.cache_compact(cache, cells._replace(n_free=i), off, i),
              lambda: fw.cache_compact(cache, cells, off, i, ws=i)):
        with pytest.raises(fw.FwError):
            f()
    got = _down(cache, cells)
    compare(got, dict(O.copy_state(s)), s, "refused calls")
