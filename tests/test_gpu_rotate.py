"""fw_rotate_heads against the oracle."""
import numpy as np
import pytest

from oracle import cells as O
from tests.serving import HALF

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tf():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2608_25230_amd import fw
    fw.lib()
    return torch, fw


def tolerance(y, mag, dtype, d, norm, angle):
    """Elementwise bound of |y - y*| for a pair whose magnitudes sum to `mag` after the norm.

    u = 2^-24.  The angle: reduced in float64, three roundings of 2^-53 of it, then rounded to float32 as at most one half
    turn's multiple, 2^-25 of pi; sine and cosine of that are off by 2 units of 2^-23 each.  Both products and their sum
    round three times.  The norm: d products and sums, the mean, eps, root and quotient change the factor by less than
    ((d + 3) / 2 + 4) u, the weight's product and the factor's two more.  The result is rounded once.
    """
    u = 2.0 ** -24
    e = 3 * 2.0 ** -53 * angle + np.pi * 2.0 ** -25 + 2.0 ** -22 + 3 * u
    if norm:
        e = e + ((d + 3) / 2 + 6) * u
    return e * mag * (1 + 2.0 ** -7) + HALF[dtype] * np.abs(y) * (1 + 2.0 ** -7) + 2.0 ** -126


def _run(tf, dtype, T, Hq, Hkv, d, rot, interleaved, eps, weights, far=1000, seed=0, how="fused"):
    torch, fw = tf
    print(f"rotate {dtype} T={T} Hq={Hq} Hkv={Hkv} d={d} rot={rot} {interleaved} eps={eps} w={weights} {how}", flush=True)
    rng = np.random.default_rng(seed + d + T)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    x = torch.tensor(rng.standard_normal((T, Hq + 2 * Hkv, d)) * 3, dtype=dt, device="cuda")
    if how == "odd":    # rows that no wide load fits
        y = torch.zeros(T, Hq + 2 * Hkv, d + 3, dtype=dt, device="cuda")[:, :, 1:d + 1]
        y.copy_(x)
        x = y
    q, k = x[:, :Hq], x[:, Hq:Hq + Hkv]
    pos = torch.tensor(rng.integers(-far, far + 1, T), device="cuda") if rot else None
    freq = torch.tensor(10000.0 ** (-np.arange(rot // 2) / max(rot // 2, 1)), dtype=torch.float32, device="cuda") if rot else None
    w = [None, None]
    if weights:
        w = [torch.tensor(1 + rng.standard_normal(d) * 0.3, dtype=torch.bfloat16 if weights == "bf16" else torch.float32,
                          device="cuda") for _ in range(2)]
    before = x.clone()
    ref = []
    for z, wt in ((q, w[0]), (k, w[1])):
        ref.append(O.rotate_heads(z.double().cpu().numpy(), None if pos is None else pos.cpu().numpy(),
                                  None if freq is None else freq.double().cpu().numpy(), eps=eps,
                                  weight=None if wt is None else wt.double().cpu().numpy(), interleaved=interleaved))
    out = None
    if how == "place":
        out = (q, k)
    if how == "heads":  # [H][T][d]
        out = tuple(torch.empty(n, T, d, dtype=dt, device="cuda").transpose(0, 1) for n in (Hq, Hkv))
    r = fw.rotate_heads(q, k, pos, freq, eps=eps, q_weight=w[0], k_weight=w[1], interleaved=interleaved, out=out)
    torch.cuda.synchronize()
    angle = far * 1.0 if rot else 0.0
    for got, want in zip((r["q"], r["k"]), ref):
        assert got.dtype is dt and got.shape == want["y"].shape
        tol = tolerance(want["y"], want["mag"], dtype, d, eps is not None, angle)
        e = np.abs(got.double().cpu().numpy() - want["y"]) / tol
        assert np.max(e, initial=0) <= 1, float(np.max(e))
    if how == "place":
        assert torch.equal(x[:, Hq + Hkv:], before[:, Hq + Hkv:])
    else:
        assert torch.equal(x, before)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,Hq,Hkv,d,rot", [(1, 1, 1, 128, 128), (5, 4, 2, 64, 64), (3, 6, 2, 80, 80), (7, 3, 1, 80, 40),
                                            (2, 2, 2, 256, 256), (2, 2, 1, 255, 254), (9, 1, 1, 1, 0), (4, 5, 1, 2, 2),
                                            (3, 2, 1, 7, 4), (2, 3, 1, 96, 36), (6, 2, 1, 129, 128), (3, 2, 2, 192, 64),
                                            (2, 1, 1, 200, 0)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_shapes(tf, dtype, T, Hq, Hkv, d, rot, interleaved):
    _run(tf, dtype, T, Hq, Hkv, d, rot, interleaved, None, None)
    _run(tf, dtype, T, Hq, Hkv, d, rot, interleaved, 1e-6, "bf16")
    _run(tf, dtype, T, Hq, Hkv, d, rot, interleaved, 1e-5, None)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("how", ["place", "heads", "odd"])
def test_layouts(tf, dtype, how):
    for d, rot in ((128, 128), (80, 40), (65, 64)):
        _run(tf, dtype, 9, 6, 2, d, rot, False, 1e-6, "f32", how=how)
        _run(tf, dtype, 9, 6, 2, d, rot, True, None, None, how=how)


@pytest.mark.parametrize("T", [4095, 4096, 4099])
def test_many_tokens(tf, T):
    """Both sides of the rule for tokens a workgroup."""
    _run(tf, "bf16", T, 3, 1, 32, 32, False, 1e-6, "bf16")


@pytest.mark.parametrize("T,Hq,Hkv,d", [(4101, 1, 0, 128), (37, 1, 1, 16), (4999, 2, 1, 256), (13, 3, 0, 20), (8193, 1, 1, 20), (3, 70, 3, 64)])
@pytest.mark.parametrize("eps", [None, 1e-6])
def test_tokens_of_a_workgroup(tf, T, Hq, Hkv, d, eps):
    """Few heads, so that a workgroup takes up to eight tokens, the last one fewer; many heads."""
    _run(tf, "bf16", T, Hq, Hkv, d, d, False, eps, eps is not None)


@pytest.mark.parametrize("far", [131072, 1 << 24, (1 << 31) - 1, 1 << 40])
def test_far_positions(tf, far):
    _run(tf, "f32", 40, 2, 1, 64, 64, False, None, None, far=far)


def test_queries_alone_and_none(tf):
    torch, fw = tf
    q = torch.randn(6, 3, 64, device="cuda")
    pos, freq = torch.arange(6, device="cuda"), torch.rand(32, device="cuda")
    a = fw.rotate_heads(q, q[:, :1], pos, freq)
    b = fw.rotate_heads(q, None, pos, freq)
    assert b["k"] is None and torch.equal(a["q"], b["q"])
    r = fw.rotate_heads(q[:0], q[:0], pos[:0], freq)
    assert r["q"].shape == (0, 3, 64)


def test_back_and_forth(tf):
    """A turn back by the opposite position gives the row again, and norms keep."""
    torch, fw = tf
    q = torch.randn(50, 4, 128, device="cuda")
    pos, freq = torch.randint(0, 100000, (50,), device="cuda"), torch.rand(64, device="cuda")
    there = fw.rotate_heads(q, None, pos, freq)["q"]
    back = fw.rotate_heads(there, None, -pos, freq)["q"]
    # two turns, each pair's sum of magnitudes at most sqrt(2) times its length, each off by what `tolerance` counts
    u = 2.0 ** -24
    pair = torch.hypot(q[..., :64], q[..., 64:]).repeat(1, 1, 2)
    e = np.pi * 2.0 ** -25 + 2.0 ** -22 + 4 * u + 3 * 2.0 ** -53 * 1e5
    assert ((back - q).abs() <= 2 * 2 ** 0.5 * 2 ** 0.5 * e * pair * 1.01 + 1e-37).all()


def test_values_that_are_not_finite_stay_in_their_rows(tf):
    torch, fw = tf
    for dt in (torch.bfloat16, torch.float32):
        q = torch.randn(8, 4, 128, device="cuda").to(dt)
        pos, freq = torch.arange(8, device="cuda"), torch.rand(64, device="cuda")
        clean = {e: fw.rotate_heads(q, None, pos, freq, eps=e)["q"] for e in (None, 1e-6)}
        q[3, 2, 5], q[6, 0, 127] = float("nan"), float("inf")
        for e in (None, 1e-6):
            r = fw.rotate_heads(q, None, pos, freq, eps=e)["q"]
            keep = torch.ones(8, 4, dtype=torch.bool, device="cuda")
            keep[3, 2] = keep[6, 0] = False
            assert torch.equal(r[keep], clean[e][keep])
            assert r[3, 2, 5].isnan() and r[3, 2, 69].isnan()
            if e is None:
                assert r[3, 2].isnan().sum() == 2 and not r[6, 0, 62].isnan()
            else:
                assert r[3, 2].isnan().all()


def test_zero_rows(tf):
    torch, fw = tf
    z = torch.zeros(3, 2, 64, device="cuda")
    pos, freq = torch.arange(3, device="cuda"), torch.rand(32, device="cuda")
    assert torch.equal(fw.rotate_heads(z, z, pos, freq, eps=1e-6)["k"], z)


def test_captured(tf):
    torch, fw = tf
    q = torch.randn(64, 8, 128, device="cuda").bfloat16()
    pos, freq = torch.arange(64, device="cuda"), torch.rand(64, device="cuda")
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        fw.rotate_heads(q, None, pos, freq, eps=1e-6)
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = fw.rotate_heads(q, None, pos, freq, eps=1e-6)["q"]
    for i in range(4):
        q.copy_(torch.randn(64, 8, 128, device="cuda"))
        pos.add_(1000 * i)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, fw.rotate_heads(q, None, pos, freq, eps=1e-6)["q"])


def test_refusals(tf):
    torch, fw = tf
    q = torch.randn(6, 3, 64, device="cuda")
    pos, freq = torch.arange(6, device="cuda"), torch.rand(32, device="cuda")
    w = torch.ones(64, device="cuda")
    for f in (lambda: fw.rotate_heads(q.half(), None, pos, freq), lambda: fw.rotate_heads(q, q[:5], pos, freq),
              lambda: fw.rotate_heads(q, q.bfloat16(), pos, freq), lambda: fw.rotate_heads(q, None, pos[:5], freq),
              lambda: fw.rotate_heads(q, None, pos.int(), freq), lambda: fw.rotate_heads(q, None, pos, freq.double()),
              lambda: fw.rotate_heads(q, None, pos, None), lambda: fw.rotate_heads(q, None, pos, freq, q_weight=w),
              lambda: fw.rotate_heads(q, None, pos, torch.rand(33, device="cuda")),
              lambda: fw.rotate_heads(q, None, pos, freq, eps=1e-6, q_weight=w[:63]),
              lambda: fw.rotate_heads(q, q, pos, freq, eps=1e-6, q_weight=w, k_weight=w.bfloat16()),
              lambda: fw.rotate_heads(q, None, pos, freq, eps=-1.0),
              lambda: fw.rotate_heads(q.transpose(1, 2), None, pos, freq),
              lambda: fw.rotate_heads(q, None, pos, freq, out=(q.transpose(0, 1), None)),
              lambda: fw.rotate_heads(q, None, pos, freq, out=(q[:1].expand(6, 3, 64), None)),
              lambda: fw.rotate_heads(q, q, pos, freq, out=(q, None)),
              lambda: fw.rotate_heads(q, None, pos.cpu(), freq)):
        with pytest.raises(fw.FwError):
            f()


def test_positions_and_freq_go_together(tf):
    torch, fw = tf
    q = torch.randn(6, 3, 64, device="cuda")
    pos, freq = torch.arange(6, device="cuda"), torch.rand(32, device="cuda")
    for given in ((pos, None), (None, freq)):
        with pytest.raises(fw.FwError) as e:
            fw.rotate_heads(q, None, *given)
        assert e.value.status == 2
    assert torch.equal(fw.rotate_heads(q, None, None, None)["q"], q)
