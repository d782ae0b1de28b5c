"""The operators on MXFP4 matrices where their index arithmetic and their precision are at an edge."""
import numpy as np
import pytest
import torch

import mxfp4_ref as ref
import paper_2604_13519_b200 as ts

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
# what the planes of a type leave out of an element, relative to the largest magnitude of its 32 neighbours: behind the last plane (2, 3, 5)
# half of the smallest e4m3 number, 2^-10, where the largest was scaled to 2^7 and every plane is sixteen times as fine as the one before
LOSS = {"bf16": 2.0 ** -21, "f16": 2.0 ** -25, "f32": 2.0 ** -33}

# (rows, columns, columns between rows, elements ahead of the first): rows that begin anywhere, of one and of many warps, with ends
# on both sides of a multiple of 256
RAGGED = [(37, 1001, 0, 0), (9, 2047, 4, 0), (5, 8190, 0, 0), (6, 225, 2, 1), (6, 255, 2, 1), (6, 256, 1, 1), (6, 257, 0, 1), (6, 481, 1, 3),
          (2, 4096, 0, 1), (1, 5000, 0, 7), (300, 513, 0, 5)]


def _inside(rows, cols, pad, first, dtype):
    """A buffer of 77s and a view into it."""
    full = torch.full((first + rows * (cols + pad) + 64,), 77.0, dtype=dtype, device="cuda")
    return full, full.as_strided((rows, cols), (cols + pad, 1), first)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,pad,first", RAGGED)
def test_quantise_rows_of_any_alignment(rows, cols, pad, first, dtype):
    rng = np.random.default_rng(rows * 10000 + cols)
    _, x = _inside(rows, cols, pad, first, TYPES[dtype])
    x.copy_(torch.from_numpy(rng.standard_normal((rows, cols)) * 2.0 ** rng.integers(-6, 7, (rows, 1))))
    codes, scales = ts.ts_mxfp4_quantise(x)
    want_codes, want_scales = ref.quantise(x.double().cpu().numpy())
    assert np.array_equal(scales.cpu().numpy(), want_scales)
    assert np.array_equal(codes.cpu().numpy(), want_codes)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,pad,first", RAGGED)
def test_dequantise_into_rows_of_any_alignment(rows, cols, pad, first, dtype):
    rng = np.random.default_rng(rows * 10000 + cols)
    nb = (cols + 31) // 32
    codes = torch.from_numpy(rng.integers(0, 256, (rows, 16 * nb), dtype=np.uint8)).cuda()
    scales = torch.from_numpy(rng.integers(112, 140, (rows, nb), dtype=np.uint8)).cuda()
    full, y = _inside(rows, cols, pad, first, TYPES[dtype])
    ts.ts_mxfp4_dequantise(codes, scales, cols, TYPES[dtype], out=y)
    want = torch.from_numpy(ref.values(codes.cpu().numpy(), scales.cpu().numpy(), cols)).to(TYPES[dtype])
    assert torch.equal(y.cpu(), want)
    y.fill_(77.0)
    assert (full == 77).all()


def _one_hot(rng, n, k, scale=127):
    """A matrix with one element other than zero in each row: its column and value per row."""
    code, at = rng.integers(1, 8, n) + 8 * rng.integers(0, 2, n), rng.integers(0, k, n)
    codes = np.zeros((n, (k + 31) // 32 * 16), dtype=np.uint8)
    codes[np.arange(n), at // 2] = code << (4 * (at & 1))
    scales = np.full((n, (k + 31) // 32), scale, dtype=np.uint8)
    w = ts.Mxfp4Matrix(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda(), k)
    return at, ref.SIZES[code & 7] * np.where(code & 8, -1.0, 1.0) * 2.0 ** (scale - 127), w


def _top(x):
    """Per element the largest magnitude of its 32 neighbours."""
    rows, k = x.shape
    return np.repeat(np.abs(np.pad(x, ((0, 0), (0, -k % 32)))).reshape(rows, -1, 32).max(-1), 32, axis=1)[:, :k]


@pytest.mark.parametrize("x_type", TYPES)
@pytest.mark.parametrize("m,n,k", [(1, 256, 256), (2, 130, 100), (4, 256, 512), (8, 200, 256), (24, 256, 256), (100, 256, 256), (20, 39000, 256)])
@pytest.mark.parametrize("spread", [0, 6, 20])
def test_every_plane_counts(m, n, k, x_type, spread):
    """One weight per row of the matrix: nothing is added up but an element's planes, each of them an exact product, in fp32 with a rounding
    (2^-24 of at most 9/8 of the result) per addition.  Beyond that the result may miss what the planes leave out; a plane less
    would leave out sixteen times that, or with fp32 rows 2^-19 of the largest neighbour.  Elements of bf16 and fp16 rows down to 2^-13 of
    their largest neighbour come out exactly."""
    rng = np.random.default_rng(m * 1000 + n + spread)
    at, w, matrix = _one_hot(rng, n, k)
    a = rng.standard_normal((m, k)) * 2.0 ** -rng.integers(0, spread + 1, (m, k))
    x = torch.from_numpy(a).to(TYPES[x_type]).cuda()
    y = ts.ts_mxfp4_product(matrix, x, torch.float32).double().cpu().numpy()
    matrix.check()
    x = x.double().cpu().numpy()
    top, want = _top(x)[:, at], x[:, at] * w
    adds = {"bf16": 1, "f16": 2, "f32": 4}[x_type]
    assert (np.abs(y - want) <= adds * 1.125 * 2.0 ** -24 * np.abs(want) + LOSS[x_type] * top * np.abs(w)).all()
    if x_type != "f32":
        large = np.abs(x[:, at]) >= 2.0 ** -13 * top
        assert large.any() and np.array_equal(y[large], want[large])


@pytest.mark.parametrize("x_type", ["bf16", "f32"])
@pytest.mark.parametrize("exponent", [-100, -112, -117, -120, -126, -130])
def test_rows_near_the_smallest_numbers(exponent, x_type):
    """The planes' scales end at 2^-127, so that what is left out of a block is never less than 2^-10 of that; weights of 2^100 bring it
    back to where it shows."""
    rng = np.random.default_rng(-exponent)
    at, w, matrix = _one_hot(rng, 256, 256, 227)
    x = torch.from_numpy(rng.standard_normal((5, 256)) * 2.0 ** exponent).to(TYPES[x_type]).cuda()
    y = ts.ts_mxfp4_product(matrix, x, torch.float32).double().cpu().numpy()
    x = x.double().cpu().numpy()
    top, want = _top(x)[:, at], x[:, at] * w
    assert np.abs(want).max() > 0
    room = 4 * 1.125 * 2.0 ** -24 * np.abs(want) + np.maximum(LOSS[x_type] * top, 2.0 ** -137) * np.abs(w)
    assert (np.abs(y - want) <= room).all()


@pytest.mark.parametrize("x_type", TYPES)
@pytest.mark.parametrize("m,n,k", [(1, 300, 200), (5, 640, 1000), (90, 257, 300), (20, 39000, 130)])
def test_results_of_every_type_are_the_same_sums_rounded(m, n, k, x_type):
    rng = np.random.default_rng(n)
    codes = torch.from_numpy(rng.integers(0, 256, (n, 16 * ((k + 31) // 32)), dtype=np.uint8)).cuda()
    scales = torch.from_numpy(rng.integers(112, 122, (n, (k + 31) // 32), dtype=np.uint8)).cuda()
    w = ts.Mxfp4Matrix(codes, scales, k)
    _, x = _inside(m, k, 3, 1, TYPES[x_type])
    x.copy_(torch.from_numpy(rng.standard_normal((m, k))))
    sums = ts.ts_mxfp4_product(w, x, torch.float32)
    w.check()
    for dtype in TYPES.values():
        for pad, first in ((0, 0), (1, 1), (4, 8)):
            full, y = _inside(m, n, pad, first, dtype)
            ts.ts_mxfp4_product(w, x, out=y)
            assert torch.equal(y, sums.to(dtype))
            y.fill_(77.0)
            assert (full == 77).all()


@pytest.mark.parametrize("x_type", TYPES)
@pytest.mark.parametrize("rows,n,k", [(70, 200, 4100), (300, 1000, 700), (130, 19000, 1100), (66, 38100, 700), (9, 38100, 1000)])
def test_a_workspace_serves_fewer_rows_too(rows, n, k, x_type):
    """Exactly as much memory as is asked for, and behind it a guard that stays as it is."""
    rng = np.random.default_rng(rows)
    codes = torch.from_numpy(rng.integers(0, 256, (n, 16 * ((k + 31) // 32)), dtype=np.uint8)).cuda()
    w = ts.Mxfp4Matrix(codes, torch.full((n, (k + 31) // 32), 120, dtype=torch.uint8, device="cuda"), k)
    x = torch.randn(rows, k, device="cuda", generator=torch.Generator("cuda").manual_seed(n)).to(TYPES[x_type])
    size = w.workspace(rows, TYPES[x_type]).numel()
    held = torch.full((size + 4096,), 123, dtype=torch.uint8, device="cuda")
    for m in sorted({1, 3, 8, rows // 4, rows // 2, rows - 1, rows}):
        if m:
            y = ts.ts_mxfp4_product(w, x[:m], torch.float32, workspace=held[:size])
            assert torch.equal(y, ts.ts_mxfp4_product(w, x[:m].clone(), torch.float32))
    w.check()
    assert (held[size:] == 123).all()
