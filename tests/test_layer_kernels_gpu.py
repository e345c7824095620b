"""Every kernel of the products with 4-bit matrices, in one part and in several, on numbers whose sums are exact: results are
compared for equality.

Entries are whole numbers of at most 3 times 2^-1, 1 or 2 (one of them a 128 x 128 block), which e2m1 and e4m3 hold exactly.
A product is a multiple of 1/4 of at most 36, so that K <= 2^16 of them, in whatever order, are exact in fp32 (4 * 36 * K
< 2^24); and the scaled instruction, which cuts at 2^(E - 13) with 2^E <= 32 the largest product's binade, cuts
nothing.  An fp32 result is the exact one, a bf16 result its nearest bf16 value.
"""

import pytest

from .test_codes_kernels_gpu import TILES, _az, _coded, _dot, _generator, _launched, _rows, _whole

pytestmark = pytest.mark.gpu


def _four(x, pad=0):
    """x as an Fp4Matrix with set bits past its columns and rows, among codes and scales."""
    az, torch = _az()
    rows, cols = x.shape
    codes = torch.full((rows + 1, -(-cols // 32) * 16 + 16 * pad), 0xFF, dtype=torch.uint8, device="cuda")
    scales = torch.full((rows + 1, -(-cols // 128) * 4 + 4 * pad), 0xFF, dtype=torch.uint8, device="cuda")
    m = az.Fp4Matrix(codes[:rows], scales[:rows], cols)
    az.quantize_tensors(x, m)
    return m


# kind of a, results, rows of a, of b, columns, and what runs them: (rows of a tile, parts of the columns); 16 is the kernel of few rows
PRODUCTS = [("e2m1", "bf16", (1, 17, 629), 16, 1), ("e2m1", "bf16", (747, 841, 735), 32, 1),
            ("e2m1", "bf16", (1, 3331, 28527), 32, 8), ("e2m1", "bf16", (1073, 3807, 627), 64, 1),
            ("e2m1", "bf16", (2985, 19, 29715), 64, 8), ("e2m1", "bf16", (2155, 2973, 639), 128, 1),
            ("e2m1", "bf16", (4315, 149, 8243), 128, 7), ("e2m1", "bf16", (2137, 4289, 625), 256, 1),
            ("e2m1", "f32", (1, 17, 651), 16, 1), ("e2m1", "f32", (161, 3539, 759), 32, 1),
            ("e2m1", "f32", (1, 3613, 28017), 32, 8), ("e2m1", "f32", (773, 4855, 603), 64, 1),
            ("e2m1", "f32", (4619, 79, 5325), 64, 7), ("e2m1", "f32", (3967, 1801, 611), 128, 1),
            ("e2m1", "f32", (3523, 133, 10561), 128, 7), ("e2m1", "f32", (2047, 4499, 607), 256, 1),
            ("e4m3", "bf16", (1, 17, 687), 16, 1), ("e4m3", "bf16", (85, 4117, 625), 32, 1),
            ("e4m3", "bf16", (17, 3329, 7193), 32, 8), ("e4m3", "bf16", (1579, 1995, 639), 64, 1),
            ("e4m3", "bf16", (3431, 17, 8569), 64, 8), ("e4m3", "bf16", (3923, 1569, 639), 128, 1),
            ("e4m3", "bf16", (3447, 169, 12689), 128, 8), ("e4m3", "f32", (1, 17, 623), 16, 1),
            ("e4m3", "f32", (33, 4037, 623), 32, 1), ("e4m3", "f32", (19, 3417, 3141), 32, 7),
            ("e4m3", "f32", (2761, 1161, 603), 64, 1), ("e4m3", "f32", (4421, 17, 3463), 64, 7),
            ("e4m3", "f32", (4087, 1595, 619), 128, 1), ("e4m3", "f32", (3233, 129, 13257), 128, 8),
            ("e4m3", "bf16", (7417, 3397, 605), 256, 1), ("e4m3", "bf16", (33, 70, 9001), 16, 1),
            ("e4m3", "f32", (17, 1001, 10001), 16, 1), ("e2m1", "f32", (33, 70, 9001), 16, 1),
            ("e2m1", "bf16", (17, 1001, 10001), 16, 1)]


@pytest.mark.parametrize("kind,out,shape,tile,parts", PRODUCTS)
@pytest.mark.parametrize("pad,bias,sa", [(0, True, 1), (3, False, 128)])
def test_products_are_exact_on_whole_numbers(kind, out, shape, tile, parts, pad, bias, sa):
    az, torch = _az()
    m, n, k = shape
    g = _generator(m, n, k, pad)
    x, w = _whole(g, m, k), _whole(g, n, k)
    a = _four(x, pad) if kind == "e2m1" else _coded(x, sa, 16 * pad, pad)
    b = _four(w, pad + 1)
    bs = _whole(g, 1, n)[0].contiguous() if bias else None
    dt = torch.float32 if out == "f32" else torch.bfloat16
    o, whole = _rows(m, n, dt, n + pad, pad)
    o.fill_(float("nan"))
    size = az.az_nibbles_matmul_workspace if kind == "e2m1" else az.az_codes_nibbles_matmul_workspace
    ws = torch.full((max(size(a.c, b.c, az.AZ_F32 if out == "f32" else az.AZ_BF16), 16),), 0xFF, dtype=torch.uint8, device="cuda")
    ran = _launched(lambda: az.matmul_tensors(a, b, o, bias=bs, workspace=ws))
    want = _dot(x, w)
    if bias:
        want += bs.double()
    assert torch.equal(o, want.float().to(dt))
    o.fill_(7.0)
    assert bool((whole == 7.0).all())
    f32, number = str(out == "f32").lower(), 4 if kind == "e2m1" else 0
    exact = str(out == "f32" and kind == "e4m3").lower()
    if tile == 16:
        assert [r[0] for r in ran] == [f"az_nibble_direct<{number},{exact},{f32}>"]
    else:
        sums = "true" if parts > 1 else f32
        assert [(r[0], r[1][1]) for r in ran[:1]] == [(f"az_nibble_tiled<{number},{TILES[tile]},{exact},{sums}>", parts)]
        assert [r[0] for r in ran[1:]] == ([f"az_join_products<{f32}>"] if parts > 1 else [])


@pytest.mark.parametrize("kind,out,shape,tile,parts", PRODUCTS)
def test_products_of_any_numbers(kind, out, shape, tile, parts):
    """Normal numbers with a scale each row, by the 2-norm: fp32 sums of K terms in a random walk are off by at most sqrt(K) 2^-24
    <= 1e-5 of it; a bf16 rounding by at most 2^-8, the scaled instruction with an e4m3 operand by 3e-5.  And a second call gives
    the same bits."""
    az, torch = _az()
    m, n, k = shape
    g = _generator(m, n, k, 9)
    x = torch.randn((m, k), generator=g, device="cuda") * torch.exp(torch.randn((m, 1), generator=g, device="cuda"))
    w = torch.randn((n, k), generator=g, device="cuda")
    a = az.Fp4Matrix.empty(m, k) if kind == "e2m1" else az.CodeMatrix.empty(m, k)
    b = az.Fp4Matrix.empty(n, k)
    az.quantize_tensors(x, a)
    az.quantize_tensors(w, b)
    az.dequantize_tensors(a, x)
    az.dequantize_tensors(b, w)
    o = torch.empty((m, n), dtype=torch.float32 if out == "f32" else torch.bfloat16, device="cuda")
    az.matmul_tensors(a, b, o)
    again = torch.empty_like(o)
    az.matmul_tensors(a, b, again)
    assert torch.equal(o.view(torch.uint8), again.view(torch.uint8))
    want = _dot(x, w)
    off = float((o.double() - want).norm() / want.norm())
    assert off <= (1e-5 if out == "f32" else 2.0 ** -8 + 1e-5 + (3e-5 if kind == "e4m3" else 0.0))


# a product's row strides at their limits: tiles up to 2^22 bytes of codes and scales, the kernel of few rows up to 2^27 and 2^26
@pytest.mark.parametrize("m,ld,ld_scales,few", [(4000, (1 << 22) - 16, 64, False), (4000, 1 << 22, 64, True), (4000, 2064, (1 << 22) - 4, False),
                                                (4000, 2064, 1 << 22, True), (20, (1 << 27) - 16, (1 << 26) - 4, True)])
@pytest.mark.parametrize("kind", ["e2m1", "e4m3"])
def test_far_rows(m, ld, ld_scales, few, kind):
    az, torch = _az()
    n, k = 300, 1100
    g = _generator(m, ld, ld_scales)
    x, w = _whole(g, m, k), _whole(g, n, k)
    a = _four(x) if kind == "e2m1" else _coded(x)
    rows = 300 if m == 4000 else 17
    w = w[:rows].contiguous()
    near = _four(w)
    codes = torch.empty((rows - 1) * ld + 16 * 35, dtype=torch.uint8, device="cuda").as_strided((rows, 560), (ld, 1))
    scales = torch.empty((rows - 1) * ld_scales + 36, dtype=torch.uint8, device="cuda").as_strided((rows, 36), (ld_scales, 1))
    codes.copy_(near.codes[:, :560])
    scales.copy_(near.scales[:, :36])
    b = az.Fp4Matrix(codes, scales, k)
    o = torch.empty((m, rows), device="cuda")
    ran = _launched(lambda: az.matmul_tensors(a, b, o))
    assert torch.equal(o, _dot(x, w).float())
    assert ("direct" in ran[0][0]) == few
