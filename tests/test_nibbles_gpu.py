"""Matrices in 4 bits on the GPU against their float64 definitions (oracle/layer.py).

Tolerances, S = sum of |a||b| over an output's products, v its exact value:
  quantise, restore: exact, both.
  fp32 product: the products are exact and each of the K additions is off by at most one unit in the last place of a
      partial sum <= S: K * 2^-23 * S (+ the bias's).
  bf16 product of 4-bit matrices: half a step of the result, 2^-8 |v|, on those sums.
  bf16 product of an e4m3 matrix: the scaled instruction also cuts each product toward zero to 2^(E - 13), E the exponent of the
      largest of its run of 8: 2^-10 * S in all.
"""

import numpy as np
import pytest

from oracle import layer as O

from .test_codes_gpu import _az, _coded, _data, _host, _rng, _strided

pytestmark = pytest.mark.gpu


def _four(rng, rows, cols, pad=0, junk=0xFF):
    """An Fp4Matrix of random data, with junk past its columns, and its exact values."""
    az, torch = _az()
    codes, scales = O.quantize(_data(rng, rows, cols).numpy())
    p = O.packed(codes)
    if cols % 2:
        p[:, -1] |= 0xF0  # the unused half of the last byte
    whole = torch.full((rows + 1, -(-cols // 32) * 16 + pad), junk, dtype=torch.uint8, device="cuda")
    whole[:rows, :p.shape[1]] = torch.from_numpy(p).cuda()
    sw = torch.full((rows + 1, -(-scales.shape[1] // 4) * 4 + pad // 4), junk, dtype=torch.uint8, device="cuda")
    sw[:rows, :scales.shape[1]] = torch.from_numpy(scales).cuda()
    return az.Fp4Matrix(whole[:rows], sw[:rows], cols), O.value(codes, scales)


SHAPES = [(1, 1), (1, 32), (2, 31), (3, 33), (5, 16), (7, 1000), (128, 128), (129, 257), (300, 40), (257, 640), (1, 20001)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("pad,offset", [(0, 0), (3, 1)])
def test_quantize_equals_the_definition(rows, cols, dtype, transposed, pad, offset):
    az, torch = _az()
    x = _data(_rng(rows, cols, 1), rows, cols, dtype)
    xd, _ = _strided(x, pad, offset=offset)

    def target(rows, cols):
        codes = torch.full((rows + 2, -(-cols // 32) * 16 + 32), 0xAB, dtype=torch.uint8, device="cuda")
        scales = torch.full((rows + 2, -(-cols // 128) * 4 + 4), 0xCD, dtype=torch.uint8, device="cuda")
        return codes, scales, az.Fp4Matrix(codes[:rows], scales[:rows], cols)

    def check(codes, scales, x):
        rows, cols = x.shape
        c, s = O.quantize(x)
        p = O.packed(c)
        got, gs = codes.cpu().numpy(), scales.cpu().numpy()
        assert np.array_equal(got[:rows, :p.shape[1]], p) and np.array_equal(gs[:rows, :s.shape[1]], s)
        assert np.all(got[:rows, p.shape[1]:] == 0xAB) and np.all(got[rows:] == 0xAB)  # nothing past the matrix is written
        assert np.all(gs[:rows, s.shape[1]:] == 0xCD) and np.all(gs[rows:] == 0xCD)

    q, qt = target(rows, cols), target(cols, rows)
    az.quantize_tensors(xd, q[2], qt[2] if transposed else None)
    torch.cuda.synchronize()
    check(q[0], q[1], x.double().numpy())
    if transposed:
        check(qt[0], qt[1], x.double().numpy().T)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("transposed", [False, True])
def test_quantize_special_values(dtype, transposed):
    az, torch = _az()
    x = np.zeros((140, 300))
    x[0, :4] = [np.inf, 1.0, np.nan, 5.0]
    x[0, 40] = -np.inf
    x[1, 130:134] = 3.3e38, -1e38, 1.0, 1e-30           # the largest values
    x[2, :3] = 1e-45, -1e-40, 1e-38                     # sub-normal ones
    x[3, :5] = 6 * 2.0 ** -9, 1.0, 2.0 ** -12, -0.0, 3e-9  # an exact power boundary
    x[4, :2] = np.nextafter(np.float32(6), np.float32(np.inf)), 17
    x[5, :32] = np.arange(32) / 4.0 - 2.0               # ties
    x[6, 32:64] = 6.0
    x[6, 33:50] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5.0, 0.1, -0.1, 0.0]
    x[139, 299] = -2.5
    t = torch.from_numpy(x.astype(np.float32))
    t = t.to(torch.bfloat16) if dtype == "bf16" else t
    q, qt = az.Fp4Matrix.empty(140, 300), az.Fp4Matrix.empty(300, 140)
    az.quantize_tensors(t.cuda(), q, qt if transposed else None)
    for m, y in ((q, t.double().numpy()),) + (((qt, t.double().numpy().T),) if transposed else ()):
        c, s = O.quantize(y)
        p = O.packed(c)
        assert np.array_equal(m.codes.cpu().numpy()[:, :p.shape[1]], p)
        assert np.array_equal(m.scales.cpu().numpy()[:, :s.shape[1]], s)
        assert s.min() >= 2 and s[s < 255].max() <= 252
        back = torch.empty(y.shape, device="cuda")
        az.dequantize_tensors(m, back)
        assert np.array_equal(_host(back), O.value(c, s), equal_nan=True)


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad,offset", [(0, 0), (5, 3)])
def test_dequantize_is_exact(rows, cols, dtype, pad, offset):
    az, torch = _az()
    q, want = _four(_rng(rows, cols, 2), rows, cols, pad=16)
    x, whole = _strided(torch.zeros((rows, cols), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32), pad, fill=9.0, offset=offset)
    az.dequantize_tensors(q, x)
    assert np.array_equal(_host(x), want)
    assert int((whole != 9.0).sum()) <= rows * cols


MM = [(1, 1, 1), (1, 16, 32), (2, 33, 40), (16, 16, 128), (17, 130, 129), (3, 5, 1000), (40, 257, 300), (64, 100, 2048), (130, 300, 513),
      (33, 1000, 96), (257, 129, 257), (300, 520, 640), (1, 300, 8192), (100, 64, 5000), (520, 530, 130)]


def _check(got, a, b, bias, out, kind):
    v, size = a @ b.T, np.abs(a) @ np.abs(b.T)
    extra = 0.0
    if bias is not None:
        v, extra = v + bias, np.abs(bias) * 2.0 ** -23
    k = a.shape[1]
    bound = k * 2.0 ** -23 * size + extra
    if out == "bf16":
        bound = 2.0 ** -8 * (np.abs(v) + bound) + bound + (2.0 ** -10 * size if kind == "e4m3" else 0.0)
    assert np.all(np.abs(got - v) <= bound * (1 + 1e-9)), float(np.max(np.abs(got - v) / np.maximum(bound, 1e-300)))


@pytest.mark.parametrize("m,n,k", MM)
@pytest.mark.parametrize("kind", ["e2m1", "e4m3", "e4m3 tiles"])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_product(m, n, k, kind, out):
    az, torch = _az()
    rng = _rng(m, n, k)
    a, va = _four(rng, m, k, pad=16) if kind == "e2m1" else _coded(rng, m, k, 128 if "tiles" in kind else 1, pad=16)
    b, vb = _four(rng, n, k, pad=32)
    bias = rng.standard_normal(n).astype(np.float32) if m % 2 else None
    c, whole = _strided(torch.zeros((m, n), dtype=torch.bfloat16 if out == "bf16" else torch.float32), 3, fill=9.0, offset=1)
    az.matmul_tensors(a, b, c, bias=torch.from_numpy(bias).cuda() if bias is not None else None)
    _check(_host(c), va, vb, bias, out, kind[:4])
    rows = whole[1:1 + m * (n + 3)].view(m, n + 3)
    assert bool((rows[:, n:] == 9.0).all()) and float(whole[0]) == 9.0  # nothing beside the rows is written


@pytest.mark.parametrize("kind", ["e2m1", "e4m3"])
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(2, 40, 300), (200, 300, 700)])
def test_scales_that_are_nan_reach_their_results_alone(m, n, k, kind, out):
    az, torch = _az()
    rng = _rng(m, n, k, 5)
    a, va = _four(rng, m, k) if kind == "e2m1" else _coded(rng, m, k)
    b, vb = _four(rng, n, k)
    b.scales[n - 3, 1] = 255
    a.scales[m - 1, 0] = 255
    c = torch.empty((m, n), dtype=torch.bfloat16 if out == "bf16" else torch.float32, device="cuda")
    az.matmul_tensors(a, b, c)
    bad = np.zeros((m, n), bool)
    bad[:, n - 3] = bad[m - 1] = True
    assert np.array_equal(np.isnan(_host(c)), bad)


@pytest.mark.parametrize("m,n,k", [(16, 16, 4096), (300, 300, 2048)])
def test_products_of_4_bits_are_exact(m, n, k):
    """Whole numbers below 2^24 in every partial sum: each of the instruction's sums has to be exact."""
    az, torch = _az()
    rng = _rng(m, n, k, 6)
    codes = [rng.integers(0, 16, (r, k)).astype(np.uint8) for r in (m, n)]
    scales = [rng.integers(127, 130, (r, k // 32)).astype(np.uint8) for r in (m, n)]
    vals = [O.value(c, s) for c, s in zip(codes, scales)]
    mats = [az.Fp4Matrix(torch.from_numpy(O.packed(c)).cuda(), torch.from_numpy(s).cuda(), k) for c, s in zip(codes, scales)]
    assert np.max(np.abs(vals[0]) @ np.abs(vals[1]).T) * 4 < 2.0 ** 24
    c = torch.empty((m, n), device="cuda")
    az.matmul_tensors(*mats, c)
    assert np.array_equal(_host(c), vals[0] @ vals[1].T)
