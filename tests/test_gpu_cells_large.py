"""The operators around the cache past 32-bit offsets, on long and many cells, on other streams, and in graphs that share
a workspace.  What is compared with is the same call on a small copy, or plain indexing where codes move as they are."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tf():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2608_25230_amd import fw
    fw.lib()
    yield torch, fw
    torch.cuda.empty_cache()


def _gen(torch, seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _codes(torch, gen, n, a, b):
    return torch.randint(0, 0x7E, (n, a, b), generator=gen, device="cuda", dtype=torch.uint8)


def _cache(tf, gen, n, bs, dp, exp=120):
    """Every token holds the largest code, so that a block of any tokens keeps its exponent and their codes."""
    torch, fw = tf
    k, v = _codes(torch, gen, n, bs, dp), _codes(torch, gen, n, dp, bs)
    k[:, :, 0] = 0x7E
    v[:, 0] = 0x7E
    e = torch.full((n,), exp, dtype=torch.uint8, device="cuda")
    return fw.KvCache(k, v, e, e.clone(), dp)


def _grown(tf, gen, lens, bs, spare=0):
    """Cells of these lengths in blocks of no order."""
    torch, fw = tf
    need = [-(-n // bs) for n in lens]
    n_blocks = sum(need) + spare
    cells = fw.cache_cells(len(lens), max(need), n_blocks)
    cells.free_list.copy_(torch.randperm(n_blocks, generator=gen, device="cuda"))
    new = torch.tensor(lens, dtype=torch.int32, device="cuda")
    r = fw.block_tables(cells.lens, new, cells.table, cells.free_list, cells.n_free, bs, n_slots=0, lens=cells.lens)
    assert int(r["refused"]) == 0
    return cells, n_blocks


def _rows(torch, cache, table, pos, bs):
    b = table[torch.div(pos, bs, rounding_mode="floor").long()].long()
    at = (pos % bs).long()
    return cache.k[b, at], cache.v[b, :, at]


@pytest.mark.parametrize("lens,bs,dp", [([200001], 64, 128), ([30000] * 6 + [5] * 50, 16, 64), ([300 + 7 * (i % 200) for i in range(3000)], 64, 32),
                                        ([70000, 0, 1, 65536, 255, 256, 257], 256, 96)])
def test_compaction_of_long_and_many_cells(tf, lens, bs, dp):
    """Kept tokens are those rows, in order, call after call."""
    torch, fw = tf
    print(f"compact {len(lens)} cells up to {max(lens)} bs={bs} dp={dp}", flush=True)
    gen = _gen(torch, len(lens))
    cells, n_blocks = _grown(tf, gen, lens, bs)
    cache = _cache(tf, gen, n_blocks, bs, dp)
    for part in (0.7, 0.5, 0.97):
        now = cells.lens.tolist()
        k0, v0, t0 = cache.k.clone(), cache.v.clone(), cells.table.clone()
        was = cache._replace(k=k0, v=v0)
        pos = [torch.nonzero(torch.rand(n, generator=gen, device="cuda") < part).flatten().int() for n in now]
        off = torch.tensor([0] + [p.numel() for p in pos], device="cuda").cumsum(0)
        r = fw.cache_compact(cache, cells, off, torch.cat(pos))
        assert int(r["refused"]) == 0 and cells.lens.tolist() == [p.numel() for p in pos]
        for c in range(0, len(lens), max(1, len(lens) // 60)):
            p = pos[c]
            if p.numel() == 0:
                continue
            want = _rows(torch, was, t0[c], p, bs)
            got = _rows(torch, cache, cells.table[c], torch.arange(p.numel(), device="cuda", dtype=torch.int32), bs)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), (part, c)
        held = sum(-(-p.numel() // bs) for p in pos)
        assert int(cells.n_free) == n_blocks - held
        both = torch.cat([cells.free_list[:n_blocks - held], cells.table[cells.table >= 0]])
        assert torch.equal(both.sort().values, torch.arange(n_blocks, device="cuda", dtype=torch.int32))


@pytest.mark.parametrize("bs,dp", [(64, 192), (16, 256), (256, 256)])
def test_compaction_of_many_wide_chunks(tf, bs, dp):
    """More chunks than workgroups, at widths of which fewer workgroups fit the card than are launched."""
    lens = [40000 + 77 * i for i in range(8)] + [100, 0, 1]
    assert all(2 * (part * sum(lens) / 256) > 800 for part in (0.7, 0.7 * 0.5, 0.7 * 0.5 * 0.97))
    test_compaction_of_long_and_many_cells(tf, lens, bs, dp)


def test_blocks_past_32_bits(tf):
    """A cache of more than 2^32 bytes: the same scores, the same compaction, fork and release as in a small copy."""
    torch, fw = tf
    gen = _gen(torch, 1)
    bs, dp, n, used = 64, 128, 600000, 100
    small = _cache(tf, gen, used, bs, dp)
    big = fw.KvCache(torch.zeros(n, bs, dp, dtype=torch.uint8, device="cuda"), torch.zeros(n, dp, bs, dtype=torch.uint8, device="cuda"),
                     torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda"), dp)
    at = n - 1 - 7 * torch.arange(used, device="cuda")      # where the small cache's blocks lie in the large one
    for x, y in zip(big[:4], small[:4]):
        x[at] = y
    sc = fw.cache_cells(4, 24, used)
    new = torch.tensor([1500, 1000, 0, 0], dtype=torch.int32, device="cuda")
    fw.block_tables(sc.lens, new, sc.table, sc.free_list, sc.n_free, bs, n_slots=0, lens=sc.lens)
    bc = fw.cache_cells(4, 24, n)
    bc.table.copy_(torch.where(sc.table >= 0, at[sc.table.long()].int(), -1))
    bc.lens.copy_(sc.lens)
    left = int(sc.n_free)
    bc.free_list[:left] = at[sc.free_list[:left].long()].int()
    bc.n_free.fill_(left)
    q = torch.randn(2, 3, 4, dp, generator=gen, device="cuda").bfloat16()
    lse = fw.cache_attention(q, small, sc.table, sc.lens)["lse"]
    assert torch.equal(fw.cache_attention(q, big, bc.table, bc.lens)["lse"], lse)
    assert torch.equal(fw.cache_scores(q, big, bc.table, bc.lens, lse)["scores"], fw.cache_scores(q, small, sc.table, sc.lens, lse)["scores"])
    pairs = [torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 1], [2, 3], [1200, 900])]
    off = torch.tensor([0, 500, 700], device="cuda")
    pos = torch.cat([torch.arange(3, 1003, 2, device="cuda"), torch.arange(0, 800, 4, device="cuda")]).int()
    end = torch.tensor([400, 2000, 77, 300], dtype=torch.int32, device="cuda")
    for cache, cells in ((small, sc), (big, bc)):
        assert int(fw.cache_fork(cache, cells, *pairs[:2], length=pairs[2])["refused"]) == 0
        assert int(fw.cache_compact(cache, cells, off, pos, which=pairs[1])["refused"]) == 0
        assert int(fw.cache_release(cache, cells, end)["refused"]) == 0
    assert torch.equal(bc.lens, sc.lens) and int(bc.n_free) == int(sc.n_free) and torch.equal(bc.shared[at], sc.shared)
    for c in range(4):
        m = int(sc.lens[c])
        p = torch.arange(m, device="cuda", dtype=torch.int32)
        for x, y in zip(_rows(torch, big, bc.table[c], p, bs), _rows(torch, small, sc.table[c], p, bs)):
            assert torch.equal(x, y), c
    # its last blocks are the small one's in reverse, so those that went back lie in reverse order too
    assert torch.equal(bc.free_list[:int(bc.n_free)].sort().values, at[sc.free_list[:int(sc.n_free)].long()].int().sort().values)


def test_scores_and_rows_past_32_bits(tf):
    """A score matrix of more than 2^31 columns in all, and a projection of more than 2^31 numbers: the last rows as alone."""
    torch, fw = tf
    gen = _gen(torch, 2)
    C, n = 70000, 32000
    x = torch.zeros(C, n, device="cuda")
    x[-2:] = torch.rand(2, n, generator=gen, device="cuda")
    lens = torch.zeros(C, dtype=torch.int32, device="cuda")
    lens[-2:] = torch.tensor([n, n - 700], dtype=torch.int32, device="cuda")
    keep = torch.full((C,), 900, dtype=torch.int32, device="cuda")
    a = fw.cache_select(x, lens, keep, recent=5, n_kept=1800)
    b = fw.cache_select(x[-2:].clone(), lens[-2:].clone(), keep[-2:].clone(), recent=5, n_kept=1800)
    assert torch.equal(a["kept_pos"], b["kept_pos"]) and torch.equal(a["offsets"][-3:], b["offsets"])
    del x, a
    torch.cuda.empty_cache()
    T, H, d = 270000, 32, 256
    q = torch.zeros(T, H, d, dtype=torch.bfloat16, device="cuda")
    q[-3:] = torch.randn(3, H, d, generator=gen, device="cuda").bfloat16()
    pos, freq = torch.arange(T, device="cuda") * 1000, torch.rand(d // 2, generator=gen, device="cuda")
    want = fw.rotate_heads(q[-3:].clone(), None, pos[-3:].clone(), freq, eps=1e-6)["q"]
    got = fw.rotate_heads(q, None, pos, freq, eps=1e-6, out=(q, None))["q"]
    assert torch.equal(got[-3:], want) and not got[:-3:1000].any()
    del q, got
    torch.cuda.empty_cache()


def test_other_streams(tf):
    """Each call runs on the current stream, after what that stream was given before."""
    torch, fw = tf
    gen = _gen(torch, 3)
    cells, n_blocks = _grown(tf, gen, [900, 1400], 64, spare=30)
    cache = _cache(tf, gen, n_blocks, 64, 64)
    q = torch.randn(1, 4, 4, 64, generator=gen, device="cuda").bfloat16()
    pos, freq = torch.arange(4, device="cuda"), torch.rand(32, generator=gen, device="cuda")
    keep = torch.tensor([300, 500], dtype=torch.int32, device="cuda")

    def step(x):
        y = fw.rotate_heads(x[0], None, pos, freq)["q"][None]
        lse = fw.cache_attention(y, cache, cells.table, cells.lens)["lse"]
        s = fw.cache_scores(y, cache, cells.table, cells.lens, lse)["scores"]
        return fw.cache_select(s, cells.lens, keep, recent=8, n_kept=800)
    want = step(q)
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        late = torch.zeros_like(q)
        torch.cuda._sleep(50_000_000)
        late.copy_(q)
        got = step(late)
        r = fw.cache_compact(cache, cells, got["offsets"], got["kept_pos"])
    st.synchronize()
    assert torch.equal(got["kept_pos"], want["kept_pos"]) and int(r["refused"]) == 0 and cells.lens.tolist() == [300, 500]


def test_graphs_that_share_a_workspace(tf):
    """Two captured calls with one workspace, replayed in turns on one stream between eager calls that use it too."""
    torch, fw = tf
    gen = _gen(torch, 4)
    cells, n_blocks = _grown(tf, gen, [640, 1000, 0, 0], 16, spare=150)
    cache = _cache(tf, gen, n_blocks, 16, 32)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    src, dst, end = i32([0, 1]), i32([2, 3]), i32([9999, 9999, 0, 0])
    which, off = i32([2, 3]), torch.tensor([0, 200, 500], device="cuda")
    pos = torch.cat([torch.arange(0, 600, 3, device="cuda"), torch.arange(1, 901, 3, device="cuda")]).int()
    ws = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
    fork = lambda: fw.cache_fork(cache, cells, src, dst, ws=ws)["refused"]
    compact = lambda: fw.cache_compact(cache, cells, off, pos, which=which, ws=ws)["refused"]
    stop = lambda: fw.cache_release(cache, cells, end, ws=ws)["refused"]
    free = int(cells.n_free)
    fork(), compact(), stop()
    torch.cuda.synchronize()
    graphs = []
    for f in (fork, compact):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = f()
        graphs.append((g, out))
    for i in range(4):
        t = cells.table[:2].clone()
        for g, out in graphs:
            g.replay()
            torch.cuda.synchronize()
            assert int(out) == 0
        assert cells.lens.tolist() == [640, 1000, 200, 300] and torch.equal(cells.table[:2], t)
        for c, (s, p) in enumerate(((0, pos[:200]), (1, pos[200:]))):
            want = _rows(torch, cache, cells.table[s], p, 16)
            got = _rows(torch, cache, cells.table[2 + c], torch.arange(p.numel(), device="cuda", dtype=torch.int32), 16)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), (i, c)
        assert int(stop()) == 0 and int(cells.n_free) == free and not cells.shared.any()


def test_two_compactions_at_once(tf):
    """On two streams, each with more chunks than workgroups fit the card."""
    torch, fw = tf
    gen = _gen(torch, 5)
    bs, dp, lens = 64, 128, [9000 + 31 * i for i in range(60)]
    sides = []
    for _ in range(2):
        cells, n_blocks = _grown(tf, gen, lens, bs)
        cache = _cache(tf, gen, n_blocks, bs, dp)
        pos = [torch.nonzero(torch.rand(n, generator=gen, device="cuda") < 0.6).flatten().int() for n in lens]
        off = torch.tensor([0] + [p.numel() for p in pos], device="cuda").cumsum(0)
        was = cache._replace(k=cache.k.clone(), v=cache.v.clone())
        sides.append((torch.cuda.Stream(), cells, cache, pos, torch.cat(pos), off, was, cells.table.clone()))
    torch.cuda.synchronize()
    out = []
    for st, cells, cache, _, flat, off, _, _ in sides:
        with torch.cuda.stream(st):
            out.append(fw.cache_compact(cache, cells, off, flat))
    torch.cuda.synchronize()
    for (_, cells, cache, pos, _, _, was, table), r in zip(sides, out):
        assert int(r["refused"]) == 0
        for c in range(0, len(lens), 7):
            want = _rows(torch, was, table[c], pos[c], bs)
            got = _rows(torch, cache, cells.table[c], torch.arange(pos[c].numel(), device="cuda", dtype=torch.int32), bs)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), c
