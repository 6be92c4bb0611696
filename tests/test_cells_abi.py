"""Argument checks of rotation, scores, selection, fork, release and compaction that need no GPU."""
import ctypes
import os

import pytest

from paper_2608_25230_amd import fw
from tests.test_serving_abi import BAD_CACHES, _cache


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(fw.LIB_PATH):
        pytest.skip("libfw.so not built")
    return fw.lib()


def _heads(**kw):
    a = dict(dtype=1, q=4096, k=8192, T=10, Hq=4, Hkv=2, d=64, q_row=512, q_head=64, k_row=512, k_head=64, rot=64, pos=16,
             freq=16, interleaved=0, norm=1, eps=1e-6, w_dtype=0, q_weight=None, k_weight=None)
    a.update(kw)
    return ctypes.byref(fw.Heads(*a.values()))


def test_rotate_heads_validation(L):
    def call(h, qo=16384, qr=256, qh=64, ko=32768, kr=128, kh=64):
        return L.fw_rotate_heads(h, qo, qr, qh, ko, kr, kh, None, 0, None)
    assert call(None) == 1
    for null in ("q", "k", "pos", "freq"):
        assert call(_heads(**{null: None})) == 1, null
    assert call(_heads(), qo=None) == 1 and call(_heads(), ko=None) == 1
    assert call(_heads(dtype=2)) == 3 and call(_heads(q_weight=16, w_dtype=5)) == 3
    for bad in (dict(T=-1), dict(Hq=-1), dict(Hkv=-1), dict(d=0), dict(d=257), dict(T=(1 << 25) + 1), dict(T=1 << 25, Hq=30),
                dict(Hq=1 << 40), dict(rot=3), dict(rot=66), dict(rot=-2), dict(q_row=-1), dict(k_head=1 << 31),
                dict(eps=-1.0), dict(eps=float("nan"))):
        assert call(_heads(**bad)) == 2, bad
    # rows of an output that meet: heads or positions too close, every row in one place
    for bad in (dict(qh=63), dict(qr=255), dict(qr=0), dict(kh=0), dict(kr=-1), dict(kr=1 << 31), dict(qr=64, qh=64 * 9)):
        assert call(_heads(), **bad) == 2, bad
    # in its own place an output keeps its strides
    assert call(_heads(), qo=4096) == 2 and call(_heads(), ko=8192) == 2
    assert call(_heads(T=0, q=None, k=None, pos=None, freq=None)) == 0
    assert call(_heads(Hq=0, Hkv=0, q=None, k=None)) == 0
    assert L.fw_rotate_heads_workspace_size(_heads()) == 0


def test_cache_scores_validation(L):
    names = ("dtype", "q", "S", "T", "Hq", "Hkv", "q_seq", "q_tok", "q_head", "table", "W", "lens", "scale", "lse",
             "earlier", "scores", "n")
    base = dict(zip(names, (1, 16, 2, 1, 8, 2, 512, 512, 64, 16, 100, 16, None, 16, None, 16, 6400)))
    call = lambda c=None, **kw: L.fw_cache_scores(c or _cache(), *dict(base, **kw).values(), None, 0, None)
    assert L.fw_cache_scores(None, *base.values(), None, 0, None) == 1
    for bad in BAD_CACHES:
        assert call(c=_cache(**bad)) == 2, bad
    assert call(dtype=3) == 3
    for null in ("q", "table", "lens", "lse", "scores"):
        assert call(**{null: None}) == 1, null
    for bad in (dict(S=0), dict(T=0), dict(Hq=7), dict(Hkv=0), dict(W=0), dict(W=1 << 25), dict(S=1 << 22), dict(T=4097),
                dict(q_seq=-1), dict(q_head=1 << 31), dict(n=0), dict(n=1 << 31), dict(S=1 << 12, W=1 << 20)):
        assert call(**bad) == 2, bad
    assert L.fw_cache_scores_workspace_size(_cache(), 2, 1, 8, 2, 100) == 0


def test_cache_select_validation(L):
    names = ("C", "scores", "n", "lens", "keep", "recent", "n_kept", "offsets", "kept_pos", "ws", "ws_bytes")
    base = dict(zip(names, (4, 16, 100, 16, 16, 3, 50, 16, 16, 16, 1 << 40)))
    call = lambda **kw: L.fw_cache_select(*dict(base, **kw).values(), None)
    for null in ("scores", "lens", "keep", "offsets", "kept_pos"):
        assert call(**{null: None}) == 1, null
    for bad in (dict(C=0), dict(C=1 << 22), dict(n=0), dict(n=(1 << 31) - 65536), dict(C=1 << 12, n=1 << 23), dict(recent=-1), dict(n_kept=-1),
                dict(n_kept=1 << 40)):
        assert call(**bad) == 2, bad
    need = L.fw_cache_select_workspace_size(4, 100)
    if need:
        assert call(ws_bytes=need - 1) == 5 and call(ws=None) == 5


def _cells(**kw):
    a = dict(C=4, max_blocks=8, table=16, lens=16, free_list=16, n_free=16, shared=16)
    a.update(kw)
    return ctypes.byref(fw.Cells(*a.values()))


BAD_CELLS = (dict(C=0), dict(C=1 << 22), dict(max_blocks=0), dict(max_blocks=1 << 25))
NO_CELLS = ("table", "lens", "free_list", "n_free", "shared")


def _common(L, call, size):
    assert call(cache=None) == 1 and call(cells=None) == 1
    for bad in BAD_CACHES:
        assert call(cache=_cache(**bad)) == 2, bad
    for bad in BAD_CELLS:
        assert call(cells=_cells(**bad)) == 2 and size(_cache(), _cells(**bad)) == 0, bad
    for null in NO_CELLS:
        assert call(cells=_cells(**{null: None})) == 1, null
    assert call(refused=None) == 1
    need = size(_cache(), _cells())
    assert need > 0
    assert call(ws_bytes=need - 1) == 5 and call(ws=None) == 5


def test_cache_fork_validation(L):
    base = dict(cache=_cache(), cells=_cells(), P=3, src=16, dst=16, length=None, refused=16, ws=16, ws_bytes=1 << 40)
    call = lambda **kw: L.fw_cache_fork(*dict(base, **kw).values(), None)
    _common(L, call, lambda c, t: L.fw_cache_fork_workspace_size(c, t, 3))
    for null in ("src", "dst"):
        assert call(**{null: None}) == 1
    for bad in (dict(P=-1), dict(P=1 << 22)):
        assert call(**bad) == 2, bad


def test_cache_release_validation(L):
    base = dict(cache=_cache(), cells=_cells(), new_len=16, refused=16, ws=16, ws_bytes=1 << 40)
    call = lambda **kw: L.fw_cache_release(*dict(base, **kw).values(), None)
    _common(L, call, L.fw_cache_release_workspace_size)
    assert call(new_len=None) == 1


def test_cache_compact_validation(L):
    base = dict(cache=_cache(), cells=_cells(), P=3, which=None, offsets=16, n_kept=100, kept_pos=16, refused=16, ws=16,
                ws_bytes=1 << 40)
    call = lambda **kw: L.fw_cache_compact(*dict(base, **kw).values(), None)
    _common(L, call, lambda c, t: L.fw_cache_compact_workspace_size(c, t, 3, 100))
    for null in ("offsets", "kept_pos"):
        assert call(**{null: None}) == 1
    for bad in (dict(P=-1), dict(P=1 << 22, which=16), dict(P=5), dict(n_kept=-1), dict(n_kept=1 << 30),
                dict(n_kept=(1 << 30) - 512), dict(P=(1 << 22) - 1, which=16, n_kept=256)):
        assert call(**bad) == 2, bad


def test_host_tensors_and_unfit_arrays_are_refused(L):
    torch = pytest.importorskip("torch")
    z = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    i32 = torch.zeros(2, dtype=torch.int32)
    cache, cells = fw.kv_cache(3, 64, 64, device="cpu"), fw.cache_cells(2, 5, 3, device="cpu")
    assert cells.table.shape == (2, 5) and cells.free_list.tolist() == [2, 1, 0] and int(cells.n_free) == 3
    off = torch.zeros(3, dtype=torch.int64)
    for f in (lambda: fw.rotate_heads(z, z, None, None, eps=1e-6),
              lambda: fw.cache_scores(z[None], cache, cells.table, i32, torch.zeros(1, 4, 2)),
              lambda: fw.cache_select(torch.zeros(2, 9), i32, i32, n_kept=0),
              lambda: fw.cache_fork(cache, cells, i32, i32), lambda: fw.cache_release(cache, cells, i32),
              lambda: fw.cache_compact(cache, cells, off, i32)):
        with pytest.raises(fw.FwError) as e:
            f()
        assert e.value.status == 2
    # what the binding itself checks, on tensors of one device
    with pytest.raises(fw.FwError):
        fw._cells(cells._replace(shared=torch.zeros(4, dtype=torch.int32)), cache, torch.device("cpu"))
    with pytest.raises(fw.FwError):
        fw._cells(cells._replace(table=cells.table.long()), cache, torch.device("cpu"))
