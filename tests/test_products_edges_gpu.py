"""Products of matrices that end inside a tile, and the join of parts by either of its ways, on whole numbers whose sums are exact
(as in test_codes_kernels_gpu.py): results are compared for equality.
"""

import pytest

from .test_codes_kernels_gpu import _az, _coded, _dot, _generator, _launched, _rows, _whole
from .test_layer_kernels_gpu import _four

pytestmark = pytest.mark.gpu


def _operand(kind, x):
    return _four(x) if kind == "e2m1" else _coded(x)


def _apart(m, ld, ld_scales):
    """The same matrix in rows `ld` bytes apart (4 bits: scales `ld_scales`), its memory's end the last row's."""
    az, torch = _az()

    def far(t, width, ld):
        v = torch.empty((m.rows - 1) * ld + width, dtype=torch.uint8, device="cuda").as_strided((m.rows, width), (ld, 1))
        v.copy_(t[:, :width])
        return v

    if isinstance(m, az.CodeMatrix):
        return az.CodeMatrix(far(m.codes, -(-m.cols // 16) * 16, ld), m.scales, m.cols, m.scale_rows)
    return az.Fp4Matrix(far(m.codes, -(-m.cols // 32) * 16, ld), far(m.scales, -(-m.cols // 128) * 4, ld_scales), m.cols)


FAR = (1 << 22) - 16  # the widest rows that tiles take


# kinds of a and b, sizes, and which of them has fewer rows than the kernel's tile
@pytest.mark.parametrize("a,b,shape,short", [("e2m1", "e2m1", (1, 3331, 28527), "a"), ("e4m3", "e2m1", (17, 3329, 7193), "a"),
                                             ("e4m3", "e4m3", (33, 3301, 8205), "a"), ("e2m1", "e2m1", (2985, 19, 29715), "b"),
                                             ("e4m3", "e2m1", (3431, 17, 8569), "b"), ("e4m3", "e4m3", (2985, 19, 29715), "b")])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_tiles_of_few_rows_that_lie_far_apart(a, b, shape, short, out):
    az, torch = _az()
    m, n, k = shape
    g = _generator(m, n, k)
    x, w = _whole(g, m, k), _whole(g, n, k)
    p, q = _operand(a, x), _operand(b, w)
    if short == "a":
        p = _apart(p, FAR, (1 << 22) - 4)
    else:
        q = _apart(q, FAR, (1 << 22) - 4)
    dt = torch.float32 if out == "f32" else torch.bfloat16
    o, whole = _rows(m, n, dt, n + 3, 1)
    ran = _launched(lambda: az.matmul_tensors(p, q, o))
    assert "tiled" in ran[0][0]
    assert torch.equal(o, _dot(x, w).float().to(dt))
    o.fill_(7.0)
    assert bool((whole == 7.0).all())


# few rows, of a and of b, in the last group of sixteen; the columns end inside the last run of steps of a wave
@pytest.mark.parametrize("a,b", [("e2m1", "e2m1"), ("e4m3", "e2m1"), ("e4m3", "e4m3")])
@pytest.mark.parametrize("shape", [(1, 17, 1300), (3, 33, 2049), (17, 31, 8192 + 900)])
def test_few_rows_that_lie_far_apart(a, b, shape):
    az, torch = _az()
    m, n, k = shape
    g = _generator(m, n, k, 2)
    x, w = _whole(g, m, k), _whole(g, n, k)
    p, q = _apart(_operand(a, x), 1 << 24, 1 << 20), _apart(_operand(b, w), 1 << 24, 1 << 20)
    o = torch.empty((m, n), device="cuda")
    ran = _launched(lambda: az.matmul_tensors(p, q, o))
    assert "direct" in ran[0][0]
    assert torch.equal(o, _dot(x, w).float())


# rows of results on both sides of the rule for four columns a thread (a multiple of four, 256 or more)
@pytest.mark.parametrize("m,n,k", [(1100, 252, 9001), (1100, 255, 9001), (1100, 256, 9001), (1100, 258, 9001), (1100, 260, 9001),
                                   (100, 1024, 20000), (100, 1027, 20000), (100, 1028, 20000), (100, 1880, 20000), (2985, 19, 29715)])
@pytest.mark.parametrize("a,b", [("e2m1", "e2m1"), ("e4m3", "e2m1"), ("e4m3", "e4m3")])
@pytest.mark.parametrize("out,pad,bias", [("f32", 0, True), ("bf16", 3, True), ("bf16", 0, False), ("f32", 5, False)])
def test_joined_parts(m, n, k, a, b, out, pad, bias):
    az, torch = _az()
    g = _generator(m, n, k, 3)
    x, w = _whole(g, m, k), _whole(g, n, k)
    p, q = _operand(a, x), _operand(b, w)
    bs = _whole(g, 1, n + 1)[0, 1:] if bias else None  # (four bytes past an aligned address)
    dt = torch.float32 if out == "f32" else torch.bfloat16
    o, whole = _rows(m, n, dt, n + pad, pad)
    ran = _launched(lambda: az.matmul_tensors(p, q, o, bias=bs))
    assert [r[0] for r in ran[1:]] == [f"az_join_products<{str(out == 'f32').lower()}>"]
    want = _dot(x, w)
    if bias:
        want += bs.double()
    assert torch.equal(o, want.float().to(dt))
    o.fill_(7.0)
    assert bool((whole == 7.0).all())
