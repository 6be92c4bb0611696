"""Argument checks of the serving entry points that need no GPU: everything is
refused on the host before any launch."""
import ctypes
import os

import pytest

from paper_2608_25230_amd import fw


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(fw.LIB_PATH):
        pytest.skip("libfw.so not built")
    return fw.lib()


def _packed(**kw):
    a = dict(dtype=1, q=16, k=16, v=16, Tq=10, Tk=10, B=1, Hq=4, Hkv=2, d=64, q_row=256, q_head=64, k_row=128, k_head=64,
             v_row=128, v_head=64, cu_q=16, cu_k=16, scale=None, causal=1)
    a.update(kw)
    return ctypes.byref(fw.Packed(*a.values()))


def test_prompt_attention_validation(L):
    call = lambda p, o=16, ws=16, n=1 << 40: L.fw_prompt_attention(p, o, None, ws, n, None)
    assert call(None) == 1
    for null in ("q", "k", "v", "cu_q", "cu_k"):
        assert call(_packed(**{null: None})) == 1, null
    assert call(_packed(), o=None) == 1
    assert call(_packed(dtype=2)) == 3
    for bad in (dict(B=0), dict(Hkv=0), dict(Hq=0), dict(Hq=3), dict(d=0), dict(d=257), dict(Tq=-1), dict(Tk=-1),
                dict(Tq=1 << 31), dict(Tk=1 << 31), dict(Tq=1 << 28, Hq=32), dict(q_row=-1), dict(k_head=1 << 31),
                dict(B=1 << 31), dict(B=1 << 30, Hkv=4, Hq=4), dict(Hq=1 << 40, Hkv=1 << 40)):
        assert call(_packed(**bad)) == 2, bad
        assert L.fw_prompt_attention_workspace_size(_packed(**bad)) == 0
    # few rows over many keys are split, and need a workspace
    few = dict(Tq=2, Tk=100000)
    need = L.fw_prompt_attention_workspace_size(_packed(**few))
    assert need > 0
    assert call(_packed(**few), n=need - 1) == 5 and call(_packed(**few), ws=None) == 5
    assert call(_packed(Tq=0, q=None)) == 0      # nothing to do


def test_block_tables_validation(L):
    names = ("C", "old", "new", "bs", "W", "table", "n_blocks", "free", "n_free", "n_slots", "slots", "offsets", "lens",
             "refused", "ws", "ws_bytes")
    base = dict(zip(names, (4, 16, 16, 64, 8, 16, 100, 16, 16, 10, 16, 16, 16, 16, 16, 1 << 40)))
    call = lambda **kw: L.fw_block_tables(*dict(base, **kw).values(), None)
    for null in ("old", "new", "table", "free", "n_free", "slots", "offsets", "lens", "refused"):
        assert call(**{null: None}) == 1, null
    for bad in (dict(C=0), dict(C=1 << 24), dict(bs=0), dict(bs=8), dict(bs=48), dict(bs=512), dict(W=0), dict(W=1 << 25),
                dict(n_blocks=0), dict(n_blocks=1 << 31), dict(n_slots=-1)):
        assert call(**bad) == 2, bad
    need = L.fw_block_tables_workspace_size(4)
    assert need > 0 and L.fw_block_tables_workspace_size(0) == 0
    assert call(ws_bytes=need - 1) == 5 and call(ws=None) == 5


def _cache(**kw):
    a = dict(k=256, v=256, k_exp=16, v_exp=16, n_blocks=10, d=64, block_size=64)
    a.update(kw)
    return ctypes.byref(fw.Cache(*a.values()))


BAD_CACHES = (dict(d=0), dict(d=257), dict(n_blocks=0), dict(n_blocks=1 << 31), dict(block_size=8), dict(block_size=96),
              dict(k=264), dict(v=1))


def test_cache_row(L):
    assert [L.fw_cache_row(d) for d in (0, 1, 32, 33, 80, 97, 128, 129, 200, 256, 257, -1)] == [
        0, 32, 32, 64, 96, 128, 128, 192, 256, 256, 0, 0]


def test_cache_store_validation(L):
    def call(c=None, dtype=1, k=16, k_row=64, v=16, v_row=64, N=5, slots=16):
        return L.fw_cache_store(c or _cache(), dtype, k, k_row, v, v_row, N, slots, None, 0, None)
    assert L.fw_cache_store(None, 1, 16, 64, 16, 64, 5, 16, None, 0, None) == 1
    for null in ("k", "v", "k_exp", "v_exp"):
        assert call(c=_cache(**{null: None})) == 1
    for bad in BAD_CACHES:
        assert call(c=_cache(**bad)) == 2, bad
    assert call(dtype=7) == 3
    for null in ("k", "v", "slots"):
        assert call(**{null: None}) == 1
    for bad in (dict(N=-1), dict(N=1 << 31), dict(k_row=-1), dict(v_row=1 << 31)):
        assert call(**bad) == 2, bad
    assert call(N=0, k=None, v=None, slots=None) == 0
    assert L.fw_cache_store_workspace_size(_cache(), 5) == 0


def test_cache_attention_validation(L):
    names = ("dtype", "q", "S", "T", "Hq", "Hkv", "q_seq", "q_tok", "q_head", "table", "W", "lens", "scale", "o", "lse",
             "ws", "ws_bytes")
    base = dict(zip(names, (1, 16, 2, 1, 8, 2, 512, 512, 64, 16, 100, 16, None, 16, None, 16, 1 << 40)))
    call = lambda c=None, **kw: L.fw_cache_attention(c or _cache(), *dict(base, **kw).values(), None)
    assert L.fw_cache_attention(None, *base.values(), None) == 1
    for bad in BAD_CACHES:
        assert call(c=_cache(**bad)) == 2, bad
    assert call(dtype=3) == 3
    for null in ("q", "table", "lens", "o"):
        assert call(**{null: None}) == 1, null
    for bad in (dict(S=0), dict(T=0), dict(Hq=0), dict(Hkv=0), dict(Hq=7), dict(W=0), dict(W=1 << 25), dict(S=1 << 24),
                dict(T=4097), dict(T=2048, Hq=8), dict(S=1 << 22, T=1024), dict(q_seq=-1), dict(q_tok=1 << 31),
                dict(S=1 << 12, W=1 << 20)):
        assert call(**bad) == 2, bad
    need = L.fw_cache_attention_workspace_size(_cache(), 2, 1, 8, 2, 100)
    assert need > 0
    assert call(ws_bytes=need - 1) == 5 and call(ws=None) == 5
    assert L.fw_cache_attention_workspace_size(_cache(), 2, 1, 8, 2, 4) == 0    # one part per cell
    assert L.fw_cache_attention_workspace_size(_cache(), 0, 1, 8, 2, 100) == 0


def test_grids_beyond_the_card_are_refused(L):
    """A grid holds 2^32 threads; sizes past that are refused before anything is launched."""
    for bad in (dict(B=1 << 24), dict(B=1 << 23, Hkv=2, Hq=2), dict(Tq=1 << 30, Hq=1, Hkv=1)):
        assert L.fw_prompt_attention(_packed(**bad), 16, None, 16, 1 << 40, None) == 2, bad
    assert L.fw_cache_store(_cache(), 1, 16, 64, 16, 64, 1 << 28, 16, None, 0, None) == 2
    for S, T, Hq, Hkv in ((1 << 22, 1, 1, 1), (1 << 20, 1, 4, 4), (1 << 20, 16, 4, 1), (1 << 14, 4096, 1, 1)):
        assert L.fw_cache_attention(_cache(), 1, 16, S, T, Hq, Hkv, 512, 512, 64, 16, 100, 16, None, 16, None, 16,
                                    1 << 60, None) == 2, (S, T, Hq, Hkv)
        assert L.fw_cache_attention_workspace_size(_cache(), S, T, Hq, Hkv, 100) == 0


def test_the_last_sizes_before_a_grid_is_full(L):
    """A grid holds fewer than 2^32 threads, its workgroups rounded up: sixteen rows of the store, four of the join."""
    for N in ((1 << 28) - 15, (1 << 28) - 1):
        for bs in (16, 256):
            assert L.fw_cache_store(_cache(block_size=bs), 1, 16, 64, 16, 64, N, 16, None, 0, None) == 2, N
    for S, T, Hq, Hkv in ((24573, 2731, 1, 1), (24573, 1, 2731, 1)):
        assert L.fw_cache_attention(_cache(), 1, 16, S, T, Hq, Hkv, 512, 512, 64, 16, 100, 16, None, 16, None, 16,
                                    1 << 60, None) == 2, (S, T, Hq, Hkv)
        assert L.fw_cache_attention_workspace_size(_cache(), S, T, Hq, Hkv, 100) == 0
    assert L.fw_cache_attention_workspace_size(_cache(), 16383, 4096, 1, 1, 100) > 0       # 2^26 - 4096 rows


def test_sequences_beyond_what_a_call_can_look_through_are_refused(L):
    """Each workgroup looks through the sequences: millions of them would take minutes."""
    for bad in (dict(B=1 << 23, Hkv=1, Hq=1), dict(B=1 << 17, Hkv=4, Hq=4), dict(B=1 << 18, Hkv=1, Hq=1),
                dict(B=1 << 16, Hkv=16, Hq=16), dict(Tq=1 << 22, B=1 << 17, Hkv=1, Hq=8)):
        assert L.fw_prompt_attention(_packed(**bad), 16, None, 16, 1 << 40, None) == 2, bad
        assert L.fw_prompt_attention_workspace_size(_packed(**bad)) == 0


def test_host_tensors_are_refused(L):
    torch = pytest.importorskip("torch")
    z = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    cu = torch.tensor([0, 4])
    i32 = torch.zeros(2, dtype=torch.int32)
    cache = fw.kv_cache(3, 64, 64, device="cpu")
    assert cache.k.shape == (3, 64, 64) and cache.v.shape == (3, 64, 64) and cache.block_size == 64
    for f in (lambda: fw.prompt_attention(z, z, z, cu),
              lambda: fw.block_tables(i32, i32, torch.zeros(2, 2, dtype=torch.int32), i32, i32[:1], 64, n_slots=0),
              lambda: fw.cache_store(cache, z[:, 0], z[:, 0], cu),
              lambda: fw.cache_attention(z[None], cache, torch.zeros(2, 2, dtype=torch.int32), i32)):
        with pytest.raises(fw.FwError) as e:
            f()
        assert e.value.status == 2
    with pytest.raises(fw.FwError):
        fw.kv_cache(3, 64, 300, device="cpu")
