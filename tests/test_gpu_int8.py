"""8-bit products on the GPU against their formulas in 64 bits.

Quantisation is defined by roundings in float32, so its integers are known exactly:
s = max(max |x| / 127, 2^-120), q = rint(x * (1 / s)). Sums of the integers are
exact, and out = sum * (s_a * s_b) takes three roundings in float32 (the sum's
conversion, the product of the scales, the product), 2^-24 each, and one in bf16
(2^-8): tolerances below count those, relative to each value.
"""

from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import stage_oracle as O
from paper_2606_18600_amd import int8, synth
from paper_2606_18600_amd.harness import DeviceStage, torch_dtype, upload_weights
from tests.helpers import ocfg

pytestmark = pytest.mark.gpu

TD = {"f32": torch.float32, "bf16": torch.bfloat16}
TOL = {"f32": 3 * 2.0 ** -24 * (1 + 2.0 ** -20), "bf16": 3 * 2.0 ** -24 + 2.0 ** -8 * (1 + 2.0 ** -20)}


def _quantised(x: torch.Tensor):
    """(integers, scales) of the rows of x, by the formula, on the host."""
    v = x.detach().float().cpu().numpy()
    with np.errstate(invalid="ignore"):
        s = np.maximum(np.abs(v).max(axis=1) / np.float32(127), np.float32(2.0 ** -120))
        q = np.rint(v * (np.float32(1) / s)[:, None])
    return q, s.astype(np.float32)


def _reference(x, w):
    qx, sx = _quantised(x)
    qw, sw = _quantised(w)
    with np.errstate(invalid="ignore"):
        return (qx.astype(np.float64) @ qw.astype(np.float64).T) * (
            sx.astype(np.float64)[:, None] * sw.astype(np.float64))


def _close(y, ref, out):
    got = y.detach().double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    err = np.abs(got - ref)
    assert np.nanmax(err - TOL[out] * np.abs(ref)) <= 0, np.nanmax(err / (np.abs(ref) + 1e-300))


def _draw(seed, rows, k, dtype="f32"):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn((rows, k), generator=g, device="cuda")
    x[:, seed % k] *= 9.0
    return x.to(TD[dtype])


# rows around the tiles of 16, 64, 128, 192 and 256 rows; odd columns and depths; a depth
# below one k tile, between two and of many
@pytest.mark.parametrize("m,n,k,dtype,out", [
    (1, 1, 1, "f32", "f32"), (1, 512, 256, "bf16", "bf16"), (1, 33, 63, "bf16", "f32"),
    (2, 17, 65, "f32", "bf16"), (15, 48, 128, "bf16", "bf16"), (16, 49, 1000, "f32", "f32"),
    (17, 130, 640, "bf16", "f32"), (31, 257, 1217, "bf16", "bf16"), (33, 96, 4096, "f32", "f32"),
    (64, 1280, 8192, "bf16", "bf16"), (65, 300, 515, "bf16", "f32"), (96, 64, 192, "f32", "bf16"),
    (127, 1000, 384, "bf16", "bf16"), (128, 2048, 1024, "bf16", "f32"),
    (129, 513, 777, "f32", "f32"), (150, 1024, 5120, "bf16", "bf16"),
    (176, 3000, 256, "bf16", "f32"), (191, 255, 2048, "f32", "bf16"),
    (193, 256, 128, "bf16", "bf16"), (256, 256, 896, "bf16", "f32"),
    (257, 769, 1409, "f32", "f32"), (385, 1100, 320, "bf16", "bf16"),
    (700, 4099, 512, "bf16", "f32"), (1024, 2560, 129, "f32", "f32"),
    (1025, 1537, 2000, "bf16", "bf16"), (2600, 530, 640, "bf16", "f32"),
])
def test_linear(m, n, k, dtype, out):
    x, w = _draw(m + n, m, k, dtype), _draw(n + k, n, k, "bf16")
    y = int8.linear(x, int8.quantize(w), TD[out])
    assert y.shape == (m, n) and y.dtype == TD[out]
    _close(y, _reference(x, w), out)


@pytest.mark.parametrize("m", [1, 3, 16, 40, 100, 128, 160, 200, 300])
def test_linear_wide_and_deep(m):
    """Many columns (every CU has several tiles) and a depth of many k tiles, on a
    sample of columns; the sums pass 2^24, where float32 would lose them."""
    x, w = _draw(m, m, 28672, "bf16"), _draw(7, 4128, 28672, "bf16")
    w[5] = w[5].abs()
    x[0] = x[0].abs()
    y = int8.linear(x, int8.quantize(w), torch.float32)
    cols = torch.arange(5, 4128, 61, device="cuda")
    _close(y[:, cols], _reference(x, w[cols]), "f32")


@pytest.mark.parametrize("m,n,k", [
    (1, 57339, 700), (2, 50001, 3001), (16, 28671, 8192), (9, 128251, 130), (20, 57339, 1100),
    (33, 57339, 2000), (64, 10239, 5120), (64, 128251, 1000), (70, 128251, 250), (100, 57339, 2000),
    (125, 128251, 900), (128, 10239, 5120), (128, 8191, 8192), (130, 57339, 2000),
    (150, 28670, 4096), (165, 57339, 515), (190, 128251, 700), (40, 5121, 20000),
    (10, 12930, 9000), (1100, 40961, 200), (2050, 8200, 300), (2100, 20001, 160),
    (2200, 2555, 300), (300, 8191, 8192)])
def test_linear_many_columns(m, n, k):
    """Sizes that keep most of the chip at work, one or more for each kernel; all rows,
    a sample of columns with the first and the last."""
    x, w = _draw(m, m, k, "bf16"), _draw(n, n, k, "bf16")
    y = int8.linear(x, int8.quantize(w), torch.float32)
    assert y.shape == (m, n) and y.isfinite().all()
    cols = torch.cat([torch.arange(0, n, max(1, n // 150), device="cuda"),
                      torch.arange(n - 40, n, device="cuda")])
    _close(y[:, cols], _reference(x, w[cols]), "f32")


@pytest.mark.parametrize("m,n,k", [(1, 8190, 28671), (2, 5, 3), (3, 57339, 8191), (4, 10239, 5119),
                                   (4, 1279, 8190), (1, 16, 16), (3, 4100, 64), (4, 700, 100)])
@pytest.mark.parametrize("dtype,out", [("bf16", "f32"), ("f32", "f32"), ("bf16", "bf16"),
                                       ("f32", "bf16")])
def test_few_rows_are_quantised_on_the_way(m, n, k, dtype, out):
    """Up to four rows, in one launch: the same values as with quantised rows, also
    from rows with a gap between them, and rows of NaN and zeros beside others."""
    wide = _draw(m + 5, m, k + 9, dtype)
    x, w = wide[:, 3:3 + k], int8.quantize(_draw(n, n, k, "bf16"))
    y = int8.linear(x, w, TD[out])
    assert torch.equal(y, int8.product(int8.quantize(x), w, TD[out]))
    if m > 1:
        x[0, k // 2], x[1] = float("nan"), 0
        z = int8.linear(x, w, TD[out])
        assert z[0].isnan().all() and (z[1] == 0).all() and torch.equal(z[2:], y[2:])


@pytest.mark.parametrize("m,n,k", [(5, 40, 200), (70, 100, 384), (300, 520, 256), (1030, 64, 130)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides_and_addresses(m, n, k, dtype):
    """Rows with a gap between them that start at any address of their type, an
    output inside a larger one (whose other values stay), a transposed input."""
    wide = _draw(m, m, k + 7, dtype)
    x = wide[:, 3:3 + k]
    w = _draw(n, n, k, dtype)
    ref = _reference(x, w)
    big = torch.full((m, n + 9), -7.0, dtype=TD[dtype], device="cuda")
    y = int8.product(int8.quantize(x), int8.quantize(w.t().contiguous().t()), out=big[:, 5:5 + n])
    _close(y, ref, dtype)
    assert (big[:, :5] == -7).all() and (big[:, 5 + n:] == -7).all()
    assert torch.equal(int8.linear(x.contiguous(), int8.quantize(w)), y)


# rows around the numbers that a block takes at once, longer than its registers hold
@pytest.mark.parametrize("m", [255, 256, 257, 511, 514, 1027])
@pytest.mark.parametrize("k", [63, 9001, 40003])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_of_a_block(m, k, dtype):
    x, w = _draw(m, m, k, dtype), _draw(k, 40, k, dtype)
    _close(int8.linear(x, int8.quantize(w), torch.float32), _reference(x, w), "f32")


@pytest.mark.parametrize("m", [3, 40, 300])
def test_offsets_beyond_32_bits(m):
    """Rows far apart: elements past 2^32 of the activations and of the result."""
    k, n = 333, 80
    ld = (1 << 32) // (m - 1) // 64 * 64 + 64
    x = torch.empty(ld * (m - 1) + k, dtype=torch.bfloat16, device="cuda").as_strided((m, k), (ld, 1))
    out = torch.empty(ld * (m - 1) + n, dtype=torch.float32,
                      device="cuda").as_strided((m, n), (ld, 1))
    x.copy_(_draw(m, m, k, "bf16"))
    w = _draw(m + 1, n, k)
    wq = int8.quantize(w)
    ref = _reference(x, w)
    _close(int8.product(int8.quantize(x), wq, out=out), ref, "f32")
    _close(int8.linear(x, wq, torch.float32), ref, "f32")


def test_leading_dimensions_and_empty():
    x, w = _draw(3, 24, 320, "bf16"), int8.quantize(_draw(4, 90, 320, "bf16"))
    y = int8.linear(x, w)
    assert torch.equal(int8.linear(x.view(2, 3, 4, 320), w), y.view(2, 3, 4, 90))
    assert int8.linear(x[:0], w).shape == (0, 90)
    assert int8.linear(x[0], w).shape == (90,)
    assert torch.equal(int8.linear(x[0], w), y[0])
    # an expanded row (stride 0)
    assert torch.equal(int8.linear(x[:1].expand(5, 320), w), y[:1].expand(5, 90))


@pytest.mark.parametrize("rows", [3, 1500])
def test_quantised_weights_of_the_caller(rows):
    """pack_weight of the formula's integers gives what quantize gives."""
    w = _draw(11, rows, 450, "f32")
    q, s = _quantised(w)
    qd, sd = torch.from_numpy(q.astype(np.int8)).cuda(), torch.from_numpy(s).cuda()
    x = int8.quantize(_draw(12, 40, 450, "bf16"))
    y = int8.product(x, int8.quantize(w), torch.float32)
    assert torch.equal(int8.product(x, int8.pack_weight(qd, sd), torch.float32), y)
    gap = torch.zeros((rows, 467), dtype=torch.int8, device="cuda")
    gap[:, 5:455] = qd
    assert torch.equal(int8.product(x, int8.pack_weight(gap[:, 5:455], sd), torch.float32), y)


@pytest.mark.parametrize("m", [4, 200, 1100])
def test_rows_of_zeros_tiny_and_not_finite(m):
    """A row of zeros gives zeros, one of the smallest values what the floor of
    the scale leaves, one with a NaN or an infinity NaN throughout, and none touches
    another row; the same in the weights."""
    x, w = _draw(21, m, 300), _draw(22, 70, 300)
    x[0] = 0
    x[1] = 2.0 ** -149
    x[2, 17], x[3, 299] = float("nan"), float("-inf")
    w[60], w[61, 3], w[62, 0] = 0, float("inf"), float("nan")
    ref = _reference(x, w)
    y = int8.linear(x, int8.quantize(w))
    _close(y, ref, "f32")
    assert (y[0, :60] == 0).all() and y[2].isnan().all() and y[3].isnan().all()
    assert y[4:, :61].isfinite().all() and y[:, 61:63].isnan().all()


def test_largest_sums():
    """All values at the ends of the range: the int32 sums' largest magnitude at the
    largest depth."""
    k = 131072
    x = torch.ones((3, k), device="cuda")
    x[1] = -1
    w = torch.ones((20, k), device="cuda")
    y = int8.linear(x, int8.quantize(w), torch.float32)
    _close(y, _reference(x, w), "f32")


@pytest.mark.parametrize("m", [1, 100, 513])
def test_captured_and_replayed(m):
    """A captured call, replayed on new inputs in the same tensors, with eager calls
    in between."""
    w = int8.quantize(_draw(31, 700, 900, "bf16"))
    x = _draw(32, m, 900, "bf16")
    int8.linear(x, w)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = int8.linear(x, w)
    for seed in range(40, 45):
        x.copy_(_draw(seed, m, 900, "bf16"))
        graph.replay()
        eager = int8.linear(x, w)
        torch.cuda.synchronize()
        assert torch.equal(y, eager)


def test_streams():
    """Two streams with work of their own, not synchronised with each other."""
    w = int8.quantize(_draw(51, 1000, 2000, "bf16"))
    xs = [_draw(52 + i, 90 + 200 * i, 2000, "bf16") for i in range(2)]
    want = [int8.linear(x, w) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    got = [[] for _ in xs]
    for _ in range(4):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i].append(int8.linear(xs[i], w))
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(a, y) for y in b)


# ---- LM head ---------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n_hidden,rows", [(40, [39, 0, 17, 17, 5]), (40, None),
                                           (200, list(range(199, 2, -1))), (1, [0])])
def test_lm_head(dtype, n_hidden, rows):
    """Against the formula in 64 bits. The kernel's normed values are off by a
    relative 2^-19 at most (a sum of `hidden` squares by threads, waves and block in
    float32, a root, a division and two products: under 32 roundings), so a value
    within 127 * 2^-18 of a border between two integers may take either: its weight
    bounds what that does to a logit. Everything else is within 2^-18 of the sum of
    the magnitudes."""
    seed, shape, V = 71, synth.TINY, 1003
    rng = np.random.default_rng(seed)
    td = torch_dtype(dtype)
    x = torch.from_numpy(rng.standard_normal((n_hidden, shape.hidden))).to("cuda", td)
    g = torch.from_numpy(rng.uniform(0.5, 1.5, shape.hidden)).to("cuda", td)
    w = torch.from_numpy(rng.standard_normal((V, shape.hidden)) / 16).to("cuda", td)
    layer = [upload_weights(synth.host_layer_weights(shape, seed, 0), dtype)]
    st = DeviceStage(shape, dtype, 0, layer, 8, 256, 4)
    try:
        y = st.lm_head(g, int8.quantize(w), x, rows=rows).double().cpu().numpy()
    finally:
        st.close()
    sel = list(range(n_hidden)) if rows is None else rows
    x64, g64 = x.double().cpu().numpy()[sel], g.double().cpu().numpy()
    h = x64 / np.sqrt((x64 ** 2).mean(1, keepdims=True) + shape.rms_eps) * g64
    s = np.abs(h).max(1, keepdims=True) / 127
    level = h / s
    q = np.rint(level)
    qw, sw = _quantised(w)
    qw, sw = qw.astype(np.float64), sw.astype(np.float64)
    ref = (q @ qw.T) * s * sw
    near = np.abs(np.abs(level - np.floor(level)) - 0.5) < 127 * 2.0 ** -18
    slack = (near @ np.abs(qw).T + 2.0 ** -18 * (np.abs(q) @ np.abs(qw).T)) * s * sw
    assert (np.abs(y - ref) <= slack).all(), np.max(np.abs(y - ref) / slack)
    # ... and close to the head in 64 bits: each value is off by half a step at most
    full = O.lm_head(ocfg(shape), x64, g64, w.double().cpu().numpy())
    steps = 0.5 * s * np.abs(w.double().cpu().numpy()).sum(1) + \
        (0.5 * sw) * (np.abs(q) * s).sum(1, keepdims=True) * (1 + 2.0 ** -10)
    assert (np.abs(y - full) <= steps + 2.0 ** -18 * np.abs(full) + slack).all()


def test_lm_head_refuses():
    from paper_2606_18600_amd.stage import STAGE_ERR_INVALID_ARG, StageError
    shape = synth.TINY
    st = DeviceStage(shape, "bf16", 0, [upload_weights(synth.host_layer_weights(shape, 1, 0), "bf16")],
                     8, 64, 4)
    try:
        x = torch.zeros((10, shape.hidden), dtype=torch.bfloat16, device="cuda")
        g = torch.ones(shape.hidden, dtype=torch.bfloat16, device="cuda")
        w = int8.quantize(torch.ones((100, shape.hidden), device="cuda"))
        narrow = int8.quantize(torch.ones((100, shape.hidden - 1), device="cuda"))
        for head, rows in ((w, [0, 10]), (w, [-1]), (narrow, [0])):
            with pytest.raises(StageError) as e:
                st.lm_head(g, head, x, rows=rows)
            assert e.value.code == STAGE_ERR_INVALID_ARG
        assert st.lm_head(g, w, x, rows=[]).shape == (0, 100)
    finally:
        st.close()
