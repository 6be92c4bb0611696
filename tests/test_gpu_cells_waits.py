"""A compaction whose waits are given up, as where something else writes into its workspace: the call says so, writes over
nothing that has not been read, and leaves every block free once or held.  The limit of the waits is set to none from
here, so that each is given up at once."""
import ctypes

import numpy as np
import pytest

from oracle import cells as O
from tests.cells import random_state, same_codes
from tests.test_gpu_cells import _compact, _down, _release, _up, tf  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture
def no_polls(tf):  # noqa: F811
    torch, fw = tf
    polls = ctypes.c_int32.in_dll(fw.lib(), "fw_compact_polls")
    was, polls.value = polls.value, 0
    yield
    torch.cuda.synchronize()
    polls.value = was


# lengths of the cells; of the first all tokens but one stay, of the second the last half, of the others all but the first.
# The last list makes more chunks than there are workgroups, so that they take several each.
@pytest.mark.parametrize("lens,bs,d,dp", [([700, 600, 0, 300], 16, 20, 32), ([520, 1, 900], 64, 128, 128), ([1000, 700], 256, 256, 256),
                                          ([2000, 1500, 300] + [3] * 400, 16, 4, 32)])
def test_waits_given_up(tf, no_polls, lens, bs, d, dp):  # noqa: F811
    torch, fw = tf
    print(f"waits given up: {len(lens)} cells, bs={bs} d={d}", flush=True)
    rng = np.random.default_rng(len(lens) + bs)
    s = random_state(rng, [*lens, 90], bs, dp, d)                  # the last cell is not listed
    pos = [[*range(5), *range(6, lens[0])], list(range(lens[1] // 2, lens[1]))] + [list(range(1, n)) for n in lens[2:]]
    off = np.cumsum([0] + [len(p) for p in pos])
    cache, cells = _up(tf, s)
    r = fw.cache_compact(cache, cells, torch.tensor(off, device="cuda"),
                         torch.tensor([x for p in pos for x in p], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert int(r["refused"]) == -1
    got, want = _down(cache, cells), O.compact(s, off.tolist(), [x for p in pos for x in p])
    for key in ("table", "lens", "shared"):
        assert np.array_equal(got[key], want[key]), key
    assert got["n_free"] == want["n_free"] and np.array_equal(got["free_list"][:got["n_free"]], want["free_list"][:want["n_free"]])
    O.invariants(got)
    # a chunk of 256 places either moved whole or kept its bytes: it moved if no chunk before it keeps tokens of its positions
    for c, p in enumerate(pos):
        for j in range(0, len(p), 256):
            part = range(j, min(j + 256, len(p)))
            inside = [i for i, x in enumerate(p) if j <= x < j + 256]
            fixed = next((i for i, x in enumerate(p) if i != x), len(p)) // bs * bs
            waits = any(i // 256 < j // 256 and i >= fixed for i in inside)
            for i in part:
                b, at = int(want["table"][c, i // bs]), i % bs
                for key in ("k", "v"):
                    row = lambda z: z[key][b, at] if key == "k" else z[key][b, :, at]
                    if waits:
                        assert np.array_equal(row(got), row(s)), (c, i, key)
                        assert got[key + "_exp"][b] == s[key + "_exp"][b]
                    else:
                        assert same_codes(row(got), row(want)).all(), (c, i, key)
                        assert got[key + "_exp"][b] == want[key + "_exp"][b]
    for key in ("k", "v"):                                        # the last cell's tokens
        for b in s["table"][-1, :-(-90 // bs)]:
            assert np.array_equal(got[key][b], s[key][b])
    assert _release(tf, got, [0] * (len(lens) + 1))["n_free"] == len(s["shared"])


def test_afterwards(tf):  # noqa: F811
    """With the limit as it is the same call is served."""
    s = random_state(np.random.default_rng(1), [700, 600], 16, 32, 20)
    assert _compact(tf, s, [0, 699, 1298], [*range(1, 700), *range(1, 600)])["refused"] == 0
