"""fw_prompt_attention against the float64 oracle: lengths, widths, head
layouts, strides, masks, non-finite values in hidden places, streams, graphs."""
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


def _inputs(torch, seed, lq, lk, Hq, Hkv, d, dtype, layout="plain", before=0, after=0):
    """Device tensors in the layout, and their values in float64.  before / after: rows outside the sequences."""
    rng = np.random.default_rng(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    Tq, Tk = before + sum(lq) + after, sum(lk)
    q, k, v = rows(rng, (Tq, Hq, d), False), rows(rng, (Tk, Hkv, d)), rows(rng, (Tk, Hkv, d), False)
    if layout == "broadcast":      # one key/value head seen as Hkv
        k, v = np.repeat(k[:, :1], Hkv, 1), np.repeat(v[:, :1], Hkv, 1)
    t = [torch.tensor(x).to(dt) for x in (q, k, v)]
    f64 = [x.double().numpy() for x in t]
    if layout == "plain":
        dev = [x.cuda() for x in t]
    elif layout == "fused":        # one projection's output
        assert Tq == Tk
        qkv = torch.cat(t, 1).cuda()
        dev = [qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]]
    elif layout == "heads":        # heads outermost
        dev = [x.transpose(0, 1).contiguous().cuda().transpose(0, 1) for x in t]
    elif layout == "odd":          # rows that start at odd elements
        dev = []
        for x in t:
            y = torch.zeros(x.shape[0], x.shape[1], d + 3, dtype=dt, device="cuda")
            y[:, :, 1:d + 1] = x.cuda()
            dev.append(y[:, :, 1:d + 1])
    else:
        dev = [t[0].cuda(), t[1][:, :1].cuda().expand(-1, Hkv, -1), t[2][:, :1].cuda().expand(-1, Hkv, -1)]
    cu_q = np.cumsum([before] + list(lq))
    cu_k = np.cumsum([0] + list(lk))
    to = lambda x: torch.tensor(x, dtype=torch.int64, device="cuda")
    return dev, f64, (to(cu_q), to(cu_k)), (cu_q, cu_k)


def _run(tf, seed, lq, lk, Hq, Hkv, d, dtype, causal=True, layout="plain", scale=None, ws=None):
    torch, fw = tf
    lk = lq if lk is None else lk
    dev, f64, cu, cun = _inputs(torch, seed, lq, lk, Hq, Hkv, d, dtype, layout)
    sc = None if scale is None else torch.tensor(scale, dtype=torch.float32, device="cuda")
    out = fw.prompt_attention(*dev, *cu, causal=causal, scale=sc, ws=ws)
    torch.cuda.synchronize()
    ref = O.prompt_attention(*f64, *cun, None if scale is None else np.float32(scale).astype(np.float64), causal)
    w = check(out["o"].float().cpu().numpy(), out["lse"].cpu().numpy(), ref, dtype, d, max(lk))
    record(f"prompt {dtype} lq={lq[:6]} lk={list(lk)[:6]} {Hq}/{Hkv} d={d} {layout}", o=w[0], lse=w[1])
    return dev, cu, out


LENGTHS = [
    ([1], None), ([64], None), ([65], None), ([129, 1, 0, 63], None), ([17, 200, 31, 128], None),
    ([300], None), ([2, 1, 70], [90, 1, 300]),       # later chunks of longer prompts
    ([70, 5, 40, 3], [10, 0, 41, 2]),                # fewer keys than queries: rows without a key
]


@pytest.mark.parametrize("lq,lk", LENGTHS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
def test_lengths(tf, lq, lk, dtype, causal):
    print(f"lengths {lq} {lk} {dtype} causal={causal}", flush=True)
    _run(tf, 1, lq, lk, 4, 2, 128 if dtype == "bf16" else 64, dtype, causal)


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("f32", 32)])
@pytest.mark.parametrize("B", [64, 65, 200])
def test_many_sequences(tf, dtype, d, B):
    """More sequences than a wave has lanes, empty ones among them, lengths of keys apart from those of queries."""
    print(f"sequences {B} {dtype}", flush=True)
    rng = np.random.default_rng(B)
    lq = [int(x) for x in rng.integers(0, 6, B)]
    lk = [int(x) for x in rng.integers(0, 9, B)]
    lq[B - 1], lk[B - 1], lq[63], lk[63] = 40, 70, 33, 20
    for causal in (True, False):
        _run(tf, B, lq, lk, 4, 2, d, dtype, causal)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
def test_a_row_does_not_depend_on_its_neighbours(tf, dtype, d):
    """The same bits for a sequence alone and beside others, whatever they hold."""
    torch, fw = tf
    dev, f64, cu, cun = _inputs(torch, 21, [90, 75, 60], [90, 75, 60], 4, 2, d, dtype)
    a = fw.prompt_attention(*dev, *cu)
    for x, lo, hi in ((dev[0], 0, 90), (dev[1], 165, 225), (dev[2], 0, 90), (dev[2], 165, 225)):
        x[lo:hi] = float("nan")
    b = fw.prompt_attention(*dev, *cu)
    torch.cuda.synchronize()
    assert torch.equal(a["o"][90:165], b["o"][90:165]) and torch.equal(a["lse"][90:165], b["lse"][90:165])
    q = dev[0].clone()
    q[100] *= 40.0          # one position's logits far above the others'
    c = fw.prompt_attention(q, dev[1], dev[2], *cu)
    torch.cuda.synchronize()
    keep = [i for i in range(90, 165) if i != 100]
    assert torch.equal(b["o"][keep], c["o"][keep]) and torch.equal(b["lse"][keep], c["lse"][keep])


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64)])
@pytest.mark.parametrize("order", ["rising", "falling", "jump"])
def test_logits_that_outgrow_the_first_maximum(tf, dtype, d, order):
    """Keys whose logits rise along the row by far more than an exponential's range, fall, or jump once."""
    torch, fw = tf
    print(f"maximum {order} {dtype} {d}", flush=True)
    n = 300
    dev, f64, cu, cun = _inputs(torch, 22, [n], [n], 2, 1, d, dtype)
    dt = dev[0].dtype
    ramp = {"rising": np.linspace(-150, 150, n), "falling": np.linspace(150, -150, n),
            "jump": np.where(np.arange(n) < 170, -40.0, 60.0)}[order]
    q, k = torch.zeros_like(dev[0]), dev[1].clone() * 0.1
    q[:, :, 0] = float(np.sqrt(d))
    k[:, 0, 0] = torch.tensor(ramp).to(dt).cuda()
    out = fw.prompt_attention(q, k, dev[2], *cu)
    torch.cuda.synchronize()
    ref = O.prompt_attention(q.double().cpu().numpy(), k.double().cpu().numpy(), f64[2], *cun, None, True)
    check(out["o"].float().cpu().numpy(), out["lse"].cpu().numpy(), ref, dtype, d, n, order)


@pytest.mark.parametrize("dtype,d", [("bf16", 8), ("bf16", 16), ("bf16", 64), ("bf16", 72), ("bf16", 80), ("bf16", 96),
                                     ("bf16", 128), ("bf16", 136), ("bf16", 192), ("bf16", 256), ("bf16", 1), ("bf16", 33),
                                     ("bf16", 100), ("f32", 1), ("f32", 7), ("f32", 32), ("f32", 80), ("f32", 128),
                                     ("f32", 130), ("f32", 256)])
def test_widths(tf, dtype, d):
    print(f"width {dtype} {d}", flush=True)
    _run(tf, 2, [77, 130, 5], None, 2, 1, d, dtype)


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (8, 8), (8, 2), (7, 1), (6, 2), (32, 2), (40, 1)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_heads(tf, Hq, Hkv, dtype):
    print(f"heads {Hq}/{Hkv} {dtype}", flush=True)
    _run(tf, 3, [33, 1, 70], None, Hq, Hkv, 64, dtype)


@pytest.mark.parametrize("layout", ["fused", "heads", "odd", "broadcast"])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 80)])
def test_strides(tf, layout, dtype, d):
    print(f"layout {layout} {dtype} {d}", flush=True)
    _run(tf, 4, [65, 40, 3], None, 4, 2, d, dtype, layout=layout)


def test_packed_odd_widths_in_one_projection(tf):
    """d = 33 in a fused projection: rows aligned to nothing."""
    _run(tf, 5, [90, 20], None, 3, 1, 33, "bf16", layout="fused")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [[0.0, 0.3], [-0.2, 5.0], [1e-30, 1.0]])
def test_scales(tf, dtype, scale):
    """Zero (equal weights), negative, and large scales (nearly one key per row)."""
    print(f"scale {scale} {dtype}", flush=True)
    _run(tf, 6, [100, 30], None, 4, 2, 64, dtype, scale=scale)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 40)])
@pytest.mark.parametrize("lq,lk", [([1], [5000]), ([3, 40], [4097, 2500]), ([5], [3]), ([2, 2], [6000, 0])])
def test_few_rows_of_many_keys(tf, dtype, d, lq, lk):
    """Ranges of keys on different workgroups, joined."""
    torch, fw = tf
    print(f"split {dtype} {lq} {lk}", flush=True)
    for causal in (True, False):
        _, _, out = _run(tf, 7, lq, lk, 4, 1, d, dtype, causal)
        if max(lk) > 2000:
            assert out["_ws"] is not None


def _same(torch, a, b):
    return torch.equal(a["o"].view(torch.int16 if a["o"].element_size() == 2 else torch.int32),
                       b["o"].view(torch.int16 if a["o"].element_size() == 2 else torch.int32)) and torch.equal(
                           a["lse"].view(torch.int32), b["lse"].view(torch.int32))


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 80), ("f32", 64)])
def test_rows_outside_the_sequences_are_left(tf, dtype, d):
    torch, fw = tf
    dev, f64, cu, cun = _inputs(torch, 8, [50, 21], [50, 21], 4, 2, d, dtype, before=3, after=9)
    L = fw.lib()
    o = torch.full_like(dev[0], 7.0)
    lse = torch.full(dev[0].shape[:2], 7.0, device="cuda")
    # the C entry point writes the caller's buffers
    q, k, v = dev
    import ctypes
    p = fw.Packed(fw.FW_BF16 if dtype == "bf16" else fw.FW_F32, q.data_ptr(), k.data_ptr(), v.data_ptr(), q.shape[0],
                  k.shape[0], 2, 4, 2, d, *q.stride()[:2], *k.stride()[:2], *v.stride()[:2], cu[0].data_ptr(),
                  cu[1].data_ptr(), None, 1)
    need = L.fw_prompt_attention_workspace_size(ctypes.byref(p))
    ws = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda")
    assert L.fw_prompt_attention(ctypes.byref(p), o.data_ptr(), lse.data_ptr(), ws.data_ptr(), need,
                                 torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    for part in (o[:3], o[-9:], lse[:3], lse[-9:]):
        assert torch.all(part == 7.0)
    ref = O.prompt_attention(*f64, *cun, None, True)
    check(o[3:-9].float().cpu().numpy(), lse[3:-9].cpu().numpy(), {key: x[3:-9] for key, x in ref.items()}, dtype, d, 50)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("bf16", 256), ("f32", 64)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_hidden_keys_and_values_do_not_touch_a_row(tf, dtype, d, bad):
    """A key or value that is not finite reaches the rows that see it and no others: later keys of the same tile,
    the next sequence's rows, every row before it."""
    torch, fw = tf
    print(f"hidden {dtype} {d} {bad}", flush=True)
    lq = [70, 100]
    dev, f64, cu, cun = _inputs(torch, 9, lq, lq, 2, 1, d, dtype)
    clean = fw.prompt_attention(*dev, *cu)
    q, k, v = (x.clone() for x in dev)
    v[40, 0, 3] = bad          # seen by rows 40 .. 69 of the first sequence, in column 3
    v[70 + 99, 0, 5] = bad     # seen by the very last row
    got = fw.prompt_attention(q, k, v, *cu)
    torch.cuda.synchronize()
    o, c = got["o"].float().cpu(), clean["o"].float().cpu()
    hit = torch.zeros(o.shape, dtype=torch.bool)
    hit[40:70, :, 3] = True
    hit[169, :, 5] = True
    assert torch.equal(~torch.isfinite(o), hit), int((~torch.isfinite(o) ^ hit).sum())
    assert torch.equal(o[~hit], c[~hit])
    if bad != bad:
        assert torch.isnan(o[hit]).all()
    else:
        assert torch.equal(o[hit], torch.full_like(o[hit], bad))
    assert torch.equal(got["lse"], clean["lse"])
    v[50, 0, 3] = -bad if bad == bad else bad    # infinities of both signs: NaN where both are seen
    both = fw.prompt_attention(q, k, v, *cu)["o"].float().cpu()
    assert torch.isnan(both[50:70, :, 3]).all() and torch.isfinite(both[:40]).all()
    k[60, 0] = bad             # rows that see key 60 are lost; the others keep their bits
    lost = fw.prompt_attention(q, k, dev[2], *cu)["o"].float().cpu()
    assert torch.equal(lost[:60], c[:60]) and torch.equal(lost[70:], c[70:])


def test_offsets_out_of_range_are_clamped(tf):
    """Offsets beyond the arrays read and write nothing outside them."""
    torch, fw = tf
    dev, f64, cu, cun = _inputs(torch, 10, [40, 20], [40, 20], 2, 1, 64, "bf16")
    good = fw.prompt_attention(*dev, *cu)
    cu_q = cu[0].clone()
    cu_q[2] = 1 << 40
    cu_k = cu[1].clone()
    cu_k[2] = 1 << 40
    wild = fw.prompt_attention(*dev, cu_q, cu_k)
    torch.cuda.synchronize()
    assert _same(torch, good, wild)
    fw.prompt_attention(*dev, torch.tensor([0, -5, 60], device="cuda"), cu[1])
    fw.prompt_attention(*dev, torch.tensor([50, 10, 60], device="cuda"), torch.tensor([9, 3, 60], device="cuda"))
    torch.cuda.synchronize()


def test_no_rows(tf):
    torch, fw = tf
    z = torch.zeros(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    kv = torch.zeros(5, 1, 64, dtype=torch.bfloat16, device="cuda")
    out = fw.prompt_attention(z, kv, kv, torch.tensor([0, 0], device="cuda"), torch.tensor([0, 5], device="cuda"))
    assert out["o"].shape == (0, 2, 64)
    q = torch.ones(4, 2, 64, dtype=torch.bfloat16, device="cuda")
    none = torch.zeros(0, 1, 64, dtype=torch.bfloat16, device="cuda")
    out = fw.prompt_attention(q, none, none, torch.tensor([0, 4], device="cuda"), torch.tensor([0, 0], device="cuda"))
    assert torch.all(out["o"] == 0) and torch.all(out["lse"] == float("-inf"))


def test_repeats_other_stream_and_graph(tf):
    """The same bits on every call, on a side stream, and on each replay of a captured call."""
    torch, fw = tf
    for lq, lk, dtype in (([100, 30, 1], None, "bf16"), ([3], [3000], "bf16"), ([40, 9], None, "f32")):
        dev, f64, cu, cun = _inputs(torch, 11, lq, lk or lq, 4, 2, 64, dtype)
        a = fw.prompt_attention(*dev, *cu)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            b = fw.prompt_attention(*dev, *cu)
        s.synchronize()
        assert _same(torch, a, b)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c = fw.prompt_attention(*dev, *cu)
        for r in range(3):
            c["o"].zero_()
            dev[0].mul_(1.0 if r == 0 else -1.0)
            want = fw.prompt_attention(*dev, *cu)
            g.replay()
            torch.cuda.synchronize()
            assert _same(torch, want, c), r


def test_long_sequence_sampled_rows(tf):
    """2,500 positions: every tile edge of a long causal row, against the oracle on sampled rows."""
    torch, fw = tf
    n, Hq, Hkv, d = 2500, 8, 2, 128
    dev, f64, cu, cun = _inputs(torch, 12, [n], [n], Hq, Hkv, d, "bf16")
    out = fw.prompt_attention(*dev, *cu)
    torch.cuda.synchronize()
    rng = np.random.default_rng(0)
    pick = np.unique(np.concatenate([[0, 1, 63, 64, 127, 128, n - 1], rng.integers(0, n, 40)]))
    o, lse = out["o"].float().cpu().numpy(), out["lse"].cpu().numpy()
    for h in range(Hq):
        ref = O.attend(f64[0][pick, h], f64[1][:, h // 4], f64[2][:, h // 4], d ** -0.5, pick + 1)
        check(o[pick, h], lse[pick, h], ref, "bf16", d, n, h)


def test_refusals(tf):
    torch, fw = tf
    dev, f64, cu, cun = _inputs(torch, 13, [8], [8], 4, 2, 64, "bf16")
    q, k, v = dev
    for bad in (dict(q=q.float()), dict(k=k.half()), dict(cu_q=cu[0].int()), dict(v=v[:, :, :32]),
                dict(q=q.cpu()), dict(cu_q=cu[0].cpu()), dict(scale=torch.ones(3, device="cuda")),
                dict(q=q[:, :3]), dict(cu_k=cu[1].repeat(2)), dict(q=q.transpose(1, 2)),
                dict(scale=torch.ones(2, dtype=torch.float64, device="cuda"))):
        a = dict(dict(q=q, k=k, v=v, cu_q=cu[0], cu_k=cu[1]), **bad)
        with pytest.raises(fw.FwError):
            fw.prompt_attention(**a)
