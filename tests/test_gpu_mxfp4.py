"""The operators on MXFP4 matrices against their definition in 64 bits (mxfp4_ref)."""
import numpy as np
import pytest
import torch

import mxfp4_ref as ref
import paper_2604_13519_b200 as ts

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _strided(a, dtype, stride):
    """a (numpy) as the left columns of a wider buffer whose other columns hold 77."""
    full = torch.full((a.shape[0], stride), 77.0, dtype=dtype, device="cuda")
    full[:, :a.shape[1]] = torch.from_numpy(np.asarray(a, dtype=np.float64)).to(dtype).cuda()
    return full, full[:, :a.shape[1]]


def _f64(t):
    return t.double().cpu().numpy()


def _matrix(rng, rows, cols):
    return rng.standard_normal((rows, cols)) * 2.0 ** rng.integers(-6, 7, (rows, 1))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (1, 31, 0), (3, 32, 0), (5, 33, 0), (7, 100, 4), (2, 4096, 0), (129, 250, 6),
                                           (64, 1024, 8), (1, 8192 + 8, 0), (333, 96, 1)])
def test_quantise(dtype, rows, cols, pad):
    rng = np.random.default_rng(rows * 1000 + cols)
    full, x = _strided(_matrix(rng, rows, cols), TYPES[dtype], cols + pad)
    codes, scales = ts.ts_mxfp4_quantise(x)
    want_codes, want_scales = ref.quantise(_f64(x))
    assert np.array_equal(scales.cpu().numpy(), want_scales)
    assert np.array_equal(codes.cpu().numpy(), want_codes)


@pytest.mark.parametrize("dtype", TYPES)
def test_quantise_borders_and_odd_values(dtype):
    """Every multiple of a sixteenth up to 8 in blocks of every scale of the type, both signs: all borders between two codes, exactly and
    next to them; then zeros, the type's smallest and largest numbers, infinities, NaN."""
    rows = []
    for e in range(-140, 127, 3):
        for first in range(0, 129, 31):
            block = np.arange(first, first + 32) / 16.0
            block[0] = 7.0
            rows.append(np.ldexp(block * np.where(np.arange(32) % 3 == 0, -1, 1), e))
    fin = torch.finfo(TYPES[dtype])
    for special in ([0.0, -0.0], [fin.max, 1.0], [-fin.max, fin.max * 0.75], [fin.tiny, -fin.tiny / 2], [fin.smallest_normal, 0.0],
                    [np.inf, 1.0], [-np.inf, 2.0], [np.nan, 3.0], [np.nan, np.inf]):
        rows.append(np.array(special + [0.0] * 30))
    _, x = _strided(np.stack(rows), TYPES[dtype], 32)
    codes, scales = ts.ts_mxfp4_quantise(x)
    want_codes, want_scales = ref.quantise(_f64(x))
    assert np.array_equal(scales.cpu().numpy(), want_scales)
    assert np.array_equal(codes.cpu().numpy(), want_codes)


def test_only_the_bad_block_is_lost():
    x = torch.ones(2, 96, device="cuda")
    x[0, 40] = float("nan")
    codes, scales = ts.ts_mxfp4_quantise(x)
    v = ts.ts_mxfp4_dequantise(codes, scales, 96, torch.float32)
    assert torch.isnan(v[0, 32:64]).all() and torch.equal(v[0, :32], x[0, :32]) and torch.equal(v[0, 64:], x[0, 64:])
    assert torch.equal(v[1], x[1])


@pytest.mark.parametrize("dtype", TYPES)
def test_dequantise_every_code_and_scale(dtype):
    scales = torch.arange(256, dtype=torch.uint8).view(256, 1).repeat(1, 16).cuda()      # 256 rows, 16 blocks: all code bytes
    codes = torch.arange(256, dtype=torch.uint8).view(1, 256).repeat(256, 1).cuda()
    v = ts.ts_mxfp4_dequantise(codes, scales, 512, TYPES[dtype])
    want = torch.from_numpy(ref.values(codes.cpu().numpy(), scales.cpu().numpy(), 512)).to(TYPES[dtype])
    assert torch.equal(torch.isnan(v.cpu()), torch.isnan(want))
    assert torch.equal(v.cpu().nan_to_num(0.5), want.nan_to_num(0.5))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (4, 33, 0), (5, 127, 3), (130, 256, 8)])
def test_dequantise_into_a_wider_buffer(dtype, rows, cols, pad):
    rng = np.random.default_rng(rows + cols)
    codes = torch.from_numpy(rng.integers(0, 256, (rows, 16 * ((cols + 31) // 32)), dtype=np.uint8)).cuda()
    scales = torch.from_numpy(rng.integers(112, 140, (rows, (cols + 31) // 32), dtype=np.uint8)).cuda()
    full = torch.full((rows, cols + pad), 77.0, dtype=TYPES[dtype], device="cuda")
    ts.ts_mxfp4_dequantise(codes, scales, cols, TYPES[dtype], out=full[:, :cols])
    want = torch.from_numpy(ref.values(codes.cpu().numpy(), scales.cpu().numpy(), cols)).to(TYPES[dtype])
    assert torch.equal(full[:, :cols].cpu(), want) and (full[:, cols:] == 77).all()


def _weights(rng, n, k, lo=112, hi=126):
    nb = (k + 31) // 32
    codes = rng.integers(0, 256, (n, 16 * nb), dtype=np.uint8)
    scales = rng.integers(lo, hi, (n, nb), dtype=np.uint8)
    return codes, scales, ts.Mxfp4Matrix(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), k)


def _check(y, x, w, k, y_dtype):
    """Products are exact, but what is left out of x: less than 2^-20 of the largest of 32 neighbours.  Sums are fp32: an addition is off
    by at most 2^-23 of what has been added up (truncation), k of them by k 2^-23 of the sum of the magnitudes; then one rounding to
    y's type, half a step of it (and half of its smallest number, where the result is below its normal ones)."""
    x, y = _f64(x), _f64(y)
    want, mag = x @ w.T, np.abs(x) @ np.abs(w).T
    fin = torch.finfo(y_dtype)
    pad = np.pad(np.abs(x), ((0, 0), (0, -k % 32))).reshape(x.shape[0], -1, 32).max(-1)
    top = np.repeat(pad, 32, axis=1)[:, :k]
    room = mag * (k * 2.0 ** -23) + top @ np.abs(w).T * 2.0 ** -20
    room = room + (np.abs(want) + room) * fin.eps / 2 + float(fin.tiny) * fin.eps / 2
    assert np.isfinite(y).all()
    assert (np.abs(y - want) <= room).all(), float(np.max(np.abs(y - want) / np.maximum(room, 1e-300)))
    # and by far not at the edge of that bound where many terms are added: as near as sums of this length are
    if want.size > 100:
        assert np.linalg.norm(y - want) <= (fin.eps / 2 + 1e-5) * np.linalg.norm(want) + 1e-30


SHAPES = [(1, 1, 1), (1, 128, 128), (1, 129, 33), (2, 100, 32), (3, 256, 160), (8, 128, 1000), (9, 300, 257), (16, 384, 512), (17, 130, 96),
          (31, 640, 2048), (33, 257, 128), (48, 128, 384), (64, 512, 640), (65, 200, 256), (80, 384, 1024), (127, 129, 520),
          (128, 256, 256), (129, 640, 192), (200, 1000, 300), (300, 256, 4096), (1, 4096, 4096), (5, 6144, 4096),
          (8, 40000, 128), (9, 38000, 300), (30, 39000, 700), (113, 38000, 200), (60, 39000, 640), (150, 19000, 3000), (301, 4096, 6000)]


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("x_type,y_type", [("bf16", "bf16"), ("f16", "f16"), ("f32", "f32"), ("bf16", "f32")])
def test_product(m, n, k, x_type, y_type):
    rng = np.random.default_rng(m * 100003 + n * 101 + k)
    codes, scales, w = _weights(rng, n, k)
    _, x = _strided(rng.standard_normal((m, k)), TYPES[x_type], k)
    y = ts.ts_mxfp4_product(w, x, TYPES[y_type])
    w.check()
    _check(y, x, ref.values(codes, scales, k), k, TYPES[y_type])


@pytest.mark.parametrize("x_type", TYPES)
@pytest.mark.parametrize("xpad,ypad", [(8, 4), (3, 0), (0, 1), (5, 3)])
def test_product_of_strided_rows_writes_nothing_beside_them(x_type, xpad, ypad):
    rng = np.random.default_rng(xpad + 10 * ypad)
    m, n, k = 19, 200, 264
    codes, scales, w = _weights(rng, n, k)
    _, x = _strided(rng.standard_normal((m, k)), TYPES[x_type], k + xpad)
    full = torch.full((m + 2, n + ypad), 77.0, dtype=TYPES[x_type], device="cuda")
    ts.ts_mxfp4_product(w, x, out=full[1:m + 1, :n])
    w.check()
    assert (full[0] == 77).all() and (full[m + 1] == 77).all() and (full[:, n:] == 77).all()
    _check(full[1:m + 1, :n], x, ref.values(codes, scales, k), k, TYPES[x_type])


def test_product_over_the_whole_range_of_scales():
    """Scales of 2^-127 to 2^127 in one matrix (a row each, so that no row's sum mixes them), NaN where the byte is 255."""
    rng = np.random.default_rng(5)
    n, k = 256, 128
    codes = rng.integers(0, 256, (n, 64), dtype=np.uint8)
    scales = np.repeat(np.arange(256, dtype=np.uint8)[:, None], 4, axis=1)
    w = ts.Mxfp4Matrix(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), k)
    x = np.zeros((3, k))
    x[0], x[1, ::7], x[2] = 2.0 ** -8 * rng.integers(1, 8, k), 0.25, 2.0 ** -9
    _, xt = _strided(x, torch.bfloat16, k)
    y = _f64(ts.ts_mxfp4_product(w, xt, torch.float32))
    want = x @ ref.values(codes, scales, k).T
    assert np.isnan(y[:, 255]).all()
    # all terms of a sum are multiples of one power of two and few: exact in fp32, but for results beyond its smallest and largest numbers
    size = np.abs(want[:, :255])
    normal, large = (size >= 2.0 ** -120) & (size < 2.0 ** 125), size >= 2.0 ** 125
    assert np.array_equal(y[:, :255][normal], want[:, :255][normal])
    assert np.abs(y[:, :255] - want[:, :255])[size < 2.0 ** -120].max() <= 2.0 ** -125
    assert (np.isinf(y[:, :255][large]) | (np.abs(y[:, :255][large] / want[:, :255][large] - 1) < 1e-6)).all()


def test_infinities_and_nan_make_their_rows_nan():
    rng = np.random.default_rng(6)
    _, _, w = _weights(rng, 200, 256)
    for rows in (5, 12):
        for dtype in TYPES.values():
            x = torch.randn(rows, 256, device="cuda", generator=torch.Generator("cuda").manual_seed(1)).to(dtype)
            good = ts.ts_mxfp4_product(w, x, torch.float32)
            x[1, 7] = float("inf")
            x[3, 100] = float("nan")
            y = ts.ts_mxfp4_product(w, x, torch.float32)
            fine = [r for r in range(rows) if r not in (1, 3)]
            assert torch.equal(y[fine], good[fine])
            assert torch.isnan(y[[1, 3]]).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_whose_elements_differ_widely(dtype):
    """Blocks with one large element and many small ones: what of the small ones is left out is bounded by the largest (2^-20 of it, the
    remainder behind the last plane, with every weight at most 6 scales)."""
    rng = np.random.default_rng(11)
    n, k = 128, 512
    codes, scales, w = _weights(rng, n, k, 120, 121)
    fin = torch.finfo(TYPES[dtype])
    for spread in (8, 14, 20, 30):
        a = rng.standard_normal((6, k)) * 2.0 ** rng.integers(-spread, 1, (6, k))
        a[:, ::32] = 1.0
        a[1] *= min(2.0 ** 100, float(fin.max) / 16)
        a[2] *= max(2.0 ** -100, float(fin.tiny) * 64)
        _, x = _strided(a, TYPES[dtype], k)
        y, xv, wv = _f64(ts.ts_mxfp4_product(w, x, torch.float32)), _f64(x), ref.values(codes, scales, k)
        top = np.repeat(np.abs(xv).reshape(6, -1, 32).max(-1), 32, axis=1)
        room = (np.abs(xv) * k * 2.0 ** -23 + top * 2.0 ** -20) @ np.abs(wv).T + 2.0 ** -140
        assert (np.abs(y - xv @ wv.T) <= room).all()


@pytest.mark.parametrize("n,k", [(128, 256), (640, 2048), (4096, 4096), (1000, 777), (40000, 256), (38100, 1000)])
@pytest.mark.parametrize("x_type", TYPES)
def test_a_row_s_result_does_not_depend_on_the_others(n, k, x_type):
    rng = np.random.default_rng(n)
    _, _, w = _weights(rng, n, k)
    x = torch.randn(64, k, device="cuda", generator=torch.Generator("cuda").manual_seed(n)).to(TYPES[x_type])
    whole = ts.ts_mxfp4_product(w, x, torch.float32)
    if x_type == "f32":
        x, whole = x[:32], ts.ts_mxfp4_product(w, x[:32], torch.float32)
    for m in (1, 2, 7, 8, 9, 16, 17, 31, 33, 40, 48, 63):
        assert torch.equal(ts.ts_mxfp4_product(w, x[:m], torch.float32), whole[:m]), m
    assert torch.equal(ts.ts_mxfp4_product(w, x[13:14].contiguous(), torch.float32), whole[13:14])


def test_empty_sides():
    e8 = lambda *s: torch.empty(*s, dtype=torch.uint8, device="cuda")
    w = ts.Mxfp4Matrix(e8(5, 0), e8(5, 0), 0)
    y = ts.ts_mxfp4_product(w, torch.empty(3, 0, device="cuda"))
    assert tuple(y.shape) == (3, 5) and (y == 0).all()
    _, _, w = _weights(np.random.default_rng(0), 5, 32)
    assert tuple(ts.ts_mxfp4_product(w, torch.empty(0, 32, device="cuda")).shape) == (0, 5)
    codes, scales = ts.ts_mxfp4_quantise(torch.empty(0, 64, device="cuda"))
    assert tuple(codes.shape) == (0, 32) and tuple(scales.shape) == (0, 2)
    assert tuple(ts.ts_mxfp4_dequantise(codes, scales, 64, torch.float32).shape) == (0, 64)


def test_captured_and_on_another_stream():
    rng = np.random.default_rng(8)
    _, _, w = _weights(rng, 384, 512)
    x = torch.randn(12, 512, device="cuda")
    ws, y = w.workspace(12, torch.float32), torch.empty(12, 384, device="cuda")
    want = ts.ts_mxfp4_product(w, x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ts.ts_mxfp4_product(w, x, out=y, workspace=ws, stream=side)
    side.synchronize()
    assert torch.equal(y, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        codes, scales = ts.ts_mxfp4_quantise(x)
        back = ts.ts_mxfp4_dequantise(codes, scales, 512, torch.float32)
        ts.ts_mxfp4_product(w, x, out=y, workspace=ws)
        z = ts.ts_mxfp4_product(w, back, workspace=ws)
    for seed in (1, 2):
        x.copy_(torch.randn(12, 512, generator=torch.Generator().manual_seed(seed)))
        y.zero_()
        g.replay()
        assert torch.equal(y, ts.ts_mxfp4_product(w, x))
        assert torch.equal(z, ts.ts_mxfp4_product(w, ts.ts_mxfp4_dequantise(*ts.ts_mxfp4_quantise(x), 512, torch.float32)))
    w.check()


def test_quantise_lay_out_multiply_together():
    """A matrix from bf16 into four bits, laid out and multiplied with: against the matrix's own values in 64 bits, and near the
    unquantised product (the relative error of an element is at most a quarter, of a sum of many about a tenth)."""
    rng = np.random.default_rng(9)
    a = torch.from_numpy(rng.standard_normal((1024, 2048)) * 0.02).to(torch.bfloat16).cuda()
    codes, scales = ts.ts_mxfp4_quantise(a)
    w = ts.Mxfp4Matrix(codes, scales, 2048)
    x = torch.from_numpy(rng.standard_normal((40, 2048))).to(torch.bfloat16).cuda()
    y = ts.ts_mxfp4_product(w, x, torch.float32)
    w.check()
    _check(y, x, ref.values(codes.cpu().numpy(), scales.cpu().numpy(), 2048), 2048, torch.float32)
    full = _f64(x) @ _f64(a).T
    assert np.linalg.norm(_f64(y) - full) < 0.25 * np.linalg.norm(full)


def test_a_matrix_laid_out_just_before_is_read_as_laid_out():
    """lay_out and product back to back, the same memory each time with another matrix: with one row (a launch that makes its own
    planes) and with several, enough k-blocks for a ring to be filled at once."""
    rng = np.random.default_rng(12)
    n, k = 4096, 1024
    packs = [(torch.from_numpy(rng.integers(0, 256, (n, k // 2), dtype=np.uint8)).cuda(), torch.full((n, k // 32), 120 + i, dtype=torch.uint8, device="cuda"))
             for i in range(4)]
    w = ts.Mxfp4Matrix(*packs[0], k)
    fresh = [ts.Mxfp4Matrix(*p, k) for p in packs]
    for m in (1, 2, 9, 40):
        x = torch.randn(m, k, device="cuda").to(torch.bfloat16)
        ws = w.workspace(m, x.dtype)
        want = [ts.ts_mxfp4_product(f, x, torch.float32) for f in fresh]
        got = []
        for _ in range(10):
            for p in packs:
                ts.binding._check(ts.binding.lib().ts_mxfp4_lay_out(p[0].data_ptr(), p[1].data_ptr(), n, k, w.data.data_ptr(),
                                                                     torch.cuda.current_stream().cuda_stream))
                got.append(ts.ts_mxfp4_product(w, x, torch.float32, workspace=ws))
        for i, y in enumerate(got):
            assert torch.equal(y, want[i % 4]), (m, i)


def test_products_on_two_streams_at_once():
    rng = np.random.default_rng(13)
    _, _, a = _weights(rng, 39000, 512)      # dealt out in runs: its CTAs wait for one another
    _, _, b = _weights(rng, 39000, 512)
    x = [torch.randn(20, 512, device="cuda") for _ in range(2)]
    want = [ts.ts_mxfp4_product(w, v) for w, v in zip((a, b), x)]
    streams, ws = [torch.cuda.Stream() for _ in range(2)], [w.workspace(20, torch.float32) for w in (a, b)]
    torch.cuda.synchronize()
    got = []
    for _ in range(20):
        for w, v, st, scratch in zip((a, b), x, streams, ws):
            got.append(ts.ts_mxfp4_product(w, v, workspace=scratch, stream=st))
    torch.cuda.synchronize()
    a.check()
    b.check()
    for i, y in enumerate(got):
        assert torch.equal(y, want[i % 2])


def test_the_first_call_may_be_captured():
    import os
    import subprocess
    import sys
    code = """
import torch, paper_2604_13519_b200 as ts
x = torch.randn(3, 512, device="cuda").to(torch.bfloat16)
codes, scales = torch.randint(0, 256, (640, 256), dtype=torch.uint8, device="cuda"), torch.full((640, 16), 120, dtype=torch.uint8, device="cuda")
w = ts.Mxfp4Matrix(codes, scales, 512)
ws = w.workspace(3, x.dtype)
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    y, one = ts.ts_mxfp4_product(w, x, workspace=ws), ts.ts_mxfp4_product(w, x[:1], workspace=ws)
    v = ts.ts_mxfp4_dequantise(*ts.ts_mxfp4_quantise(x), 512, torch.float32)
g.replay()
w.check()
assert torch.equal(y, ts.ts_mxfp4_product(w, x)) and torch.equal(one, y[:1])
assert torch.equal(v, ts.ts_mxfp4_dequantise(*ts.ts_mxfp4_quantise(x), 512, torch.float32))
print("captured")
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "captured" in r.stdout, r.stderr[-2000:]


def test_refusals_on_the_device():
    _, _, w = _weights(np.random.default_rng(14), 200, 64)
    x = torch.randn(20, 64, device="cuda")
    ws = w.workspace(20, x.dtype)
    full = torch.zeros(20, 200, device="cuda")
    for bad in (dict(workspace=ws[:64]), dict(workspace=ws[1:]), dict(workspace=ws.cpu()), dict(out=full[:19]), dict(out=full, dtype=torch.float16),
                dict(out=full.t().contiguous().t())):
        with pytest.raises((ts.TsError, ValueError)):
            ts.ts_mxfp4_product(w, x, **bad)
    for bad in (x[:, :32], x.t(), x.double(), x.cpu(), x[None]):
        with pytest.raises((ValueError, TypeError)):
            ts.ts_mxfp4_product(w, bad)
    codes, scales = ts.ts_mxfp4_quantise(x)
    for c, s, cols in ((codes[:, :16], scales, 64), (codes, scales[:5], 64), (codes, scales, 65), (codes.cpu(), scales, 64)):
        with pytest.raises(ValueError):
            ts.ts_mxfp4_dequantise(c, s, cols, torch.float32)


@pytest.mark.parametrize("x_type", TYPES)
def test_few_rows_many_times(x_type):
    """One to eight rows over matrices of many k-blocks, the ring several times full: every call the same result."""
    rng = np.random.default_rng(15)
    for n, k in ((6144, 4096), (24576, 1024), (128, 12288)):
        _, _, w = _weights(rng, n, k)
        x = torch.randn(64, k, device="cuda").to(TYPES[x_type])
        whole = ts.ts_mxfp4_product(w, x[:32], torch.float32)
        for m in (1, 2, 3, 5, 8):
            for _ in range(20):
                assert torch.equal(ts.ts_mxfp4_product(w, x[:m], torch.float32), whole[:m]), (n, k, m)
        w.check()


@pytest.mark.parametrize("m,n,k", [(33, 39000, 2100), (80, 77900, 2100), (113, 39000, 2100), (225, 2049, 1000), (700, 10100, 2100), (1500, 4900, 2111),
                                   (8200, 1030, 2100), (1000, 41000, 300)])
@pytest.mark.parametrize("x_type", TYPES)
def test_many_rows(m, n, k, x_type):
    """Rows in one and several chunks, odd numbers of tiles, runs that begin and end anywhere; twice on the same memory, once captured."""
    rng = np.random.default_rng(m + n + k)
    codes, scales, w = _weights(rng, n, k)
    _, x = _strided(rng.standard_normal((m, k)), TYPES[x_type], k + 5)
    held = torch.full((m + 2, n + 3), 9., device="cuda")
    y = held[1:m + 1, :n]
    ws = w.workspace(m, TYPES[x_type])
    ts.ts_mxfp4_product(w, x, out=y, workspace=ws)
    w.check()
    _check(y, x, ref.values(codes, scales, k), k, torch.float32)
    first = y.clone()
    ws.fill_(255)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        ts.ts_mxfp4_product(w, x, out=y, workspace=ws)
    for _ in range(3):
        y.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, first)
    w.check()
    assert (held[0] == 9).all() and (held[-1] == 9).all() and (held[:, n:] == 9).all()


def test_many_rows_on_two_streams_beside_few():
    """Products by pairs of CTAs on two streams, on a third one products in runs of single CTAs and of few rows."""
    rng = np.random.default_rng(15)
    _, _, a = _weights(rng, 10100, 2100)
    _, _, b = _weights(rng, 39000, 512)
    x = [torch.randn(700, 2100, device="cuda").bfloat16(), torch.randn(650, 2100, device="cuda").bfloat16(), torch.randn(20, 512, device="cuda"),
         torch.randn(3, 512, device="cuda")]
    m = [a, a, b, b]
    want = [ts.ts_mxfp4_product(w, v) for w, v in zip(m, x)]
    streams, ws = [torch.cuda.Stream() for _ in range(3)], [w.workspace(v.shape[0], v.dtype) for w, v in zip(m, x)]
    torch.cuda.synchronize()
    got = []
    for _ in range(10):
        for i in range(4):
            got.append(ts.ts_mxfp4_product(m[i], x[i], workspace=ws[i], stream=streams[min(i, 2)]))
    torch.cuda.synchronize()
    a.check()
    b.check()
    for i, y in enumerate(got):
        assert torch.equal(y, want[i % 4])
