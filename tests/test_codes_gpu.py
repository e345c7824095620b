"""Coded matrices on the GPU against their float64 definitions (oracle/codes.py).

Tolerances, S = sum of |a||b| over an output's products, v its exact value:
  quantise, restore: exact, both.
  fp32 product: the products are exact; each of the K additions, of whatever order, is off
      by at most one unit in the last place of a partial sum <= S: K * 2^-23 * S (+ the bias's).
  bf16 product: half a step of the result, 2^-8 |v|; the scaled e4m3 instruction cuts each
      product toward zero to 2^(E - 13), E the exponent of the largest of its run of 8:
      at most 8 * 2^-13 of that product, so 2^-10 * S in all; and fp32 sums as above.
  weight gradient: fp32 sums of exact products over the rows, as the fp32 product.
"""

import numpy as np
import pytest

from oracle import codes as O

pytestmark = pytest.mark.gpu


def _az():
    import torch

    import paper_2609_37447_amd as az
    return az, torch


def _rng(*seed):
    return np.random.Generator(np.random.PCG64(list(seed)))


def _data(rng, rows, cols, dtype="f32"):
    """fp32 values over many binades; bf16 ones are rounded first."""
    import torch
    x = rng.standard_normal((rows, cols)) * np.exp2(rng.integers(-6, 7, (rows, 1 + (cols - 1) // 128)).repeat(128, 1)[:, :cols])
    x[rng.random((rows, cols)) < 0.1] = 0.0
    t = torch.from_numpy(x.astype(np.float32))
    return t.to(torch.bfloat16) if dtype == "bf16" else t


def _strided(t, pad, dev="cuda", fill=None, offset=0):
    """t on the device in rows `pad` elements longer than it, from `offset` elements on."""
    import torch
    rows, cols = t.shape
    whole = torch.full((rows * (cols + pad) + offset + 8,), 0 if fill is None else fill, dtype=t.dtype, device=dev)
    view = whole[offset:offset + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    view.copy_(t)
    return view, whole


def _coded(rng, rows, cols, scale_rows=1, pad=0, junk=0x7F):
    """A CodeMatrix of random data, with junk in the columns past cols, and its exact values."""
    az, torch = _az()
    codes, scales = O.quantize(_data(rng, rows, cols).numpy(), scale_rows)
    ld = -(-cols // 16) * 16 + pad
    whole = torch.full((rows + 1, ld), junk, dtype=torch.uint8, device="cuda")
    whole[:rows, :cols] = torch.from_numpy(codes).cuda()
    m = az.CodeMatrix(whole[:rows], torch.from_numpy(scales).cuda(), cols, scale_rows)
    return m, O.value(codes, scales, scale_rows)


def _host(t):
    return t.double().cpu().numpy()


# --------------------------------------------------------------------------- #
# Quantising and restoring
# --------------------------------------------------------------------------- #
SHAPES = [(1, 1), (1, 128), (2, 127), (3, 129), (5, 16), (7, 1000), (128, 128), (129, 257), (300, 40), (257, 640), (1, 20001)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("form", ["rows", "tiles", "transposed"])
@pytest.mark.parametrize("pad,offset", [(0, 0), (3, 1), (16, 0)])
def test_quantize_equals_the_definition(rows, cols, dtype, form, pad, offset):
    az, torch = _az()
    x = _data(_rng(rows, cols, 1), rows, cols, dtype)
    sr = 1 if form == "rows" else 128
    want_c, want_s = O.quantize(x.double().numpy(), sr)
    xd, _ = _strided(x, pad, offset=offset)
    ld = -(-cols // 16) * 16 + 16
    codes = torch.full((rows + 2, ld), 0xAB, dtype=torch.uint8, device="cuda")
    scales = torch.full(want_s.shape, 0xCD, dtype=torch.uint8, device="cuda")
    q = az.CodeMatrix(codes[:rows], scales, cols, sr)
    qt = None
    if form == "transposed":
        ldt = -(-rows // 16) * 16 + 32
        codes_t = torch.full((cols + 2, ldt), 0xAB, dtype=torch.uint8, device="cuda")
        scales_t = torch.full(want_s.T.shape, 0xCD, dtype=torch.uint8, device="cuda")
        qt = az.CodeMatrix(codes_t[:cols], scales_t, rows, 128)
    az.quantize_tensors(xd, q, qt)
    torch.cuda.synchronize()
    got = codes.cpu().numpy()
    assert np.array_equal(got[:rows, :cols], want_c)
    assert np.array_equal(scales.cpu().numpy(), want_s)
    assert np.all(got[:, cols:] == 0xAB) and np.all(got[rows:] == 0xAB)  # nothing past the matrix is written
    if qt is not None:
        got = codes_t.cpu().numpy()
        assert np.array_equal(got[:cols, :rows], want_c.T)
        assert np.array_equal(scales_t.cpu().numpy(), want_s.T)
        assert np.all(got[:, rows:] == 0xAB) and np.all(got[cols:] == 0xAB)


@pytest.mark.parametrize("scale_rows", [1, 128])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantize_special_values(scale_rows, dtype):
    az, torch = _az()
    x = np.zeros((140, 300))
    x[0, :4] = [np.inf, -np.inf, np.nan, 5.0]           # non-finite entries beside finite ones
    x[1, 130:134] = 3.3e38, -1e38, 1.0, 1e-30            # the largest values
    x[2, :3] = 1e-45, -1e-40, 1e-38                      # sub-normal ones
    x[3, :5] = 448 * 2.0 ** -9, 1.0, 2.0 ** -12, -0.0, 3e-9  # an exact power boundary
    x[4, :2] = np.nextafter(np.float32(448), np.float32(np.inf)), 17
    x[5, :16] = 448.0
    x[5, 16:128] = np.arange(112) / 8.0 + 1 / 16         # ties
    x[139, 299] = -2.5
    x[130:140, 256:] += np.where(np.arange(44) % 3 == 0, np.nan, 0.0)  # a block with NaN throughout
    t = torch.from_numpy(x.astype(np.float32))
    t = t.to(torch.bfloat16) if dtype == "bf16" else t
    want_c, want_s = O.quantize(t.double().numpy(), scale_rows)
    q = az.CodeMatrix.empty(140, 300, scale_rows)
    az.quantize_tensors(t.cuda(), q)
    back = torch.empty((140, 300), device="cuda")
    az.dequantize_tensors(q, back)
    assert np.array_equal(q.codes.cpu().numpy()[:, :300], want_c)
    assert np.array_equal(q.scales.cpu().numpy(), want_s)
    assert want_s.min() >= 10 and want_s.max() <= 246
    want = O.value(want_c, want_s, scale_rows)
    assert np.array_equal(_host(back), want, equal_nan=True)
    assert np.array_equal(np.isnan(want), ~np.isfinite(t.double().numpy()))


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale_rows,pad,offset", [(1, 0, 0), (1, 5, 3), (128, 8, 0)])
def test_dequantize_is_exact(rows, cols, dtype, scale_rows, pad, offset):
    az, torch = _az()
    q, want = _coded(_rng(rows, cols, 2), rows, cols, scale_rows, pad=16)
    t = torch.zeros((rows, cols), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32)
    x, whole = _strided(t, pad, fill=7.0, offset=offset)
    az.dequantize_tensors(q, x)
    assert np.array_equal(_host(x), want)
    x.fill_(7.0)
    assert bool((whole == 7.0).all())  # and nothing past the rows was written


def test_every_code_and_scale_is_restored():
    az, torch = _az()
    codes = np.tile(np.arange(256, dtype=np.uint8), (237, 1))
    scales = np.repeat(np.arange(10, 247, dtype=np.uint8)[:, None], 2, axis=1)
    q = az.CodeMatrix(torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda())
    want = O.value(codes, scales)
    for dt in (torch.float32, torch.bfloat16):
        x = torch.empty((237, 256), dtype=dt, device="cuda")
        az.dequantize_tensors(q, x)
        assert np.array_equal(_host(x), want, equal_nan=True)


# --------------------------------------------------------------------------- #
# The product
# --------------------------------------------------------------------------- #
def _check(got, want, size, terms, bf16, cut=0.0):
    tol = terms * 2.0 ** -23 * size + (2.0 ** -8 * np.abs(want) if bf16 else 0.0) + cut * size
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4].tolist(), float(np.abs(got - want)[bad].max()))
    if want.size >= 64:  # and as a whole, by the 2-norm: bf16's half steps are uniform, 2^-8 / sqrt 3 at most
        rel = np.linalg.norm(got - want) / max(np.linalg.norm(want), 1e-300)
        assert rel <= (2.0 ** -8 if bf16 else 1e-5), rel


PRODUCTS = [(1, 1, 1), (1, 16, 128), (1, 300, 129), (2, 17, 4000), (3, 17, 129), (15, 33, 127), (16, 100, 1024), (17, 64, 300),
            (33, 47, 90), (64, 100, 1000), (64, 257, 2048), (65, 130, 257), (128, 128, 128), (130, 250, 640), (200, 1880, 384),
            (256, 256, 512), (257, 300, 1111), (300, 1000, 16), (513, 515, 1296), (1, 4672, 8192), (1000, 130, 2000)]


@pytest.mark.parametrize("m,n,k", PRODUCTS)
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("sa,sb,pad,bias", [(1, 128, 0, True), (1, 1, 16, False), (128, 128, 3, True)])
def test_matmul(m, n, k, out, sa, sb, pad, bias):
    az, torch = _az()
    rng = _rng(m, n, k)
    a, av = _coded(rng, m, k, sa, pad=16 * (pad % 2))
    b, bv = _coded(rng, n, k, sb, pad=16 * (pad % 3))
    bs = rng.standard_normal(n).astype(np.float32) if bias else None
    dt = torch.float32 if out == "f32" else torch.bfloat16
    o, whole = _strided(torch.zeros((m, n), dtype=dt), pad, fill=7.0, offset=pad)
    az.matmul_tensors(a, b, o, bias=torch.from_numpy(bs).cuda() if bias else None)
    got = _host(o)
    want = av @ bv.T + (0.0 if bs is None else bs.astype(np.float64))
    size = np.abs(av) @ np.abs(bv).T + (0.0 if bs is None else np.abs(bs))
    _check(got, want, size, k + 1, out == "bf16", 2.0 ** -10 if out == "bf16" else 0.0)
    o.fill_(7.0)
    assert bool((whole == 7.0).all())


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("m", [5, 70, 300])
def test_matmul_nan_stays_in_its_row_and_column(out, m):
    az, torch = _az()
    rng = _rng(7, m)
    a, _ = _coded(rng, m, 300)
    b, _ = _coded(rng, 40, 300)
    a.codes[3, 299] = 0x7F
    b.scales[11, 1] = 255
    o = torch.empty((m, 40), dtype=torch.float32 if out == "f32" else torch.bfloat16, device="cuda")
    az.matmul_tensors(a, b, o)
    bad = np.isnan(_host(o))
    want = np.zeros((m, 40), bool)
    want[3] = True
    want[:, 11] = True
    assert np.array_equal(bad, want)


@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_matmul_far_apart_scales(out):
    # blocks of a at 2^-60 and 2^60 against blocks of b the other way round: every product counts
    az, torch = _az()
    rng = _rng(8)
    up = np.where(np.arange(512) // 128 % 2 == 0, 60.0, -60.0)
    xa, xb = rng.standard_normal((70, 512)) * 2.0 ** up, rng.standard_normal((90, 512)) * 2.0 ** -up
    ms = []
    for x in (xa, xb):
        q = az.CodeMatrix.empty(x.shape[0], 512)
        az.quantize_tensors(torch.from_numpy(x.astype(np.float32)).cuda(), q)
        ms.append((q, O.value(q.codes.cpu().numpy(), q.scales.cpu().numpy())))
    o = torch.empty((70, 90), dtype=torch.float32 if out == "f32" else torch.bfloat16, device="cuda")
    az.matmul_tensors(ms[0][0], ms[1][0], o)
    av, bv = ms[0][1], ms[1][1]
    _check(_host(o), av @ bv.T, np.abs(av) @ np.abs(bv).T, 513, out == "bf16", 2.0 ** -10 if out == "bf16" else 0.0)


# --------------------------------------------------------------------------- #
# The weight's gradient
# --------------------------------------------------------------------------- #
GRADS = [(1, 1, 1), (1, 64, 128), (2, 3, 129), (31, 70, 90), (64, 64, 64), (65, 129, 257), (200, 1880, 100), (333, 17, 1000),
         (1000, 256, 256), (1024, 130, 640), (4097, 40, 33), (300, 513, 520), (5000, 136, 264)]


@pytest.mark.parametrize("m,n,k", GRADS)
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("bias,add,pad,offset", [(True, False, 0, 0), (False, True, 8, 0), (True, True, 3, 1)])
def test_weight_grad(m, n, k, out, bias, add, pad, offset):
    az, torch = _az()
    rng = _rng(m, n, k, 3)
    x, xv = _coded(rng, m, k, pad=16 * (pad % 2))
    dy = _data(rng, m, n, "bf16")
    dyd, _ = _strided(dy, pad, fill=float("nan"), offset=offset)
    dt = torch.float32 if out == "f32" else torch.bfloat16
    w0 = torch.from_numpy(rng.standard_normal((n, k)).astype(np.float32)).to(dt)
    b0 = torch.from_numpy(rng.standard_normal(n).astype(np.float32))
    dw, whole = _strided(w0, pad, fill=7.0, offset=offset)
    db = b0.cuda() if bias else None
    if not add:
        dw.fill_(float("nan"))
        if bias:
            db.fill_(float("nan"))
    ws = torch.full((max(az.az_codes_weight_grad_workspace(m, n, k), 16),), 0xFF, dtype=torch.uint8, device="cuda")
    az.weight_grad_tensors(dyd, x, dw, db=db, accumulate=add, workspace=ws)
    y = dy.double().numpy()
    want = y.T @ xv + (w0.double().numpy() if add else 0.0)
    size = np.abs(y).T @ np.abs(xv) + (np.abs(w0.double().numpy()) if add else 0.0)
    _check(_host(dw), want, size, m + 1, out == "bf16")
    if bias:
        wb = y.sum(0) + (b0.double().numpy() if add else 0.0)
        sb = np.abs(y).sum(0) + (np.abs(b0.double().numpy()) if add else 0.0)
        _check(_host(db), wb, sb, m + 1, False)
    dw.fill_(7.0)
    assert bool((whole == 7.0).all())


@pytest.mark.parametrize("add", [False, True])
def test_weight_grad_of_no_rows(add):
    az, torch = _az()
    x = az.CodeMatrix.empty(0, 40)
    dy = torch.empty((0, 24), dtype=torch.bfloat16, device="cuda")
    dw, db = torch.full((24, 40), 3.0, device="cuda"), torch.full((24,), 3.0, device="cuda")
    az.weight_grad_tensors(dy, x, dw, db=db, accumulate=add)
    assert bool((dw == (3.0 if add else 0.0)).all()) and bool((db == (3.0 if add else 0.0)).all())


def test_weight_grad_against_differences():
    # loss = sum(dy * (x W^T + b)) in float64, moved along single weights and biases
    az, torch = _az()
    rng = _rng(9)
    x, xv = _coded(rng, 50, 70)
    dy = _data(rng, 50, 30, "bf16")
    dw, db = torch.empty((30, 70), device="cuda"), torch.empty((30,), device="cuda")
    az.weight_grad_tensors(dy.cuda(), x, dw, db=db)
    y, w, b = dy.double().numpy(), rng.standard_normal((30, 70)), rng.standard_normal(30)
    size = np.abs(y).T @ np.abs(xv)

    def loss(w, b):
        return float((y * (xv @ w.T + b)).sum())

    for i, j in rng.integers(0, 30, (12, 2)):
        e = np.zeros_like(w)
        e[i, 2 * j] = 0.5
        diff = loss(w + e, b) - loss(w - e, b)
        assert abs(diff - float(dw[i, 2 * j])) <= 51 * 2.0 ** -23 * size[i, 2 * j] + 1e-9 * abs(loss(w, b))
        e = np.zeros_like(b)
        e[i] = 0.5
        diff = loss(w, b + e) - loss(w, b - e)
        assert abs(diff - float(db[i])) <= 51 * 2.0 ** -23 * np.abs(y[:, i]).sum() + 1e-9 * abs(loss(w, b))


# --------------------------------------------------------------------------- #
# Together, on streams and in graphs
# --------------------------------------------------------------------------- #
class _Layer:
    """A dense head's step: save the input in 8 bits, product, policy, and back."""

    def __init__(self, m, n, k, seed):
        az, torch = _az()
        rng = _rng(m, n, k, seed)
        self.az, self.m, self.n, self.k = az, m, n, k
        self.x = _data(rng, m, k, "bf16").cuda()
        self.w = torch.from_numpy((rng.standard_normal((n, k)) * 0.1).astype(np.float32)).cuda()
        self.b = torch.from_numpy(rng.standard_normal(n).astype(np.float32)).cuda()
        self.legal = torch.from_numpy((rng.random((m, n)) < 0.3).astype(np.uint8)).cuda()
        self.legal[0] = 0
        self.target = torch.from_numpy(rng.random((m, n)).astype(np.float32)).cuda() * self.legal
        self.xq, self.wq = az.CodeMatrix.empty(m, k), az.CodeMatrix.empty(n, k, 128)
        self.wt, self.dq = az.CodeMatrix.empty(k, n, 128), az.CodeMatrix.empty(m, n)
        self.z, self.p = torch.empty((m, n), device="cuda"), torch.empty((m, n), device="cuda")
        self.dy = torch.empty((m, n), dtype=torch.bfloat16, device="cuda")
        self.dw, self.db = torch.empty((n, k), device="cuda"), torch.empty((n,), device="cuda")
        self.dx = torch.empty((m, k), dtype=torch.bfloat16, device="cuda")
        self.ws = torch.empty((max(16, az.az_codes_weight_grad_workspace(m, n, k), az.az_logits_policy_workspace(m, n),
                                   az.az_codes_matmul_workspace(self.xq.c, self.wq.c, az.AZ_F32),
                                   az.az_codes_matmul_workspace(self.dq.c, self.wt.c, az.AZ_BF16)),),
                              dtype=torch.uint8, device="cuda")

    def step(self):
        az = self.az
        az.quantize_tensors(self.x, self.xq)
        az.quantize_tensors(self.w, self.wq, self.wt)
        az.matmul_tensors(self.xq, self.wq, self.z, bias=self.b, workspace=self.ws)
        az.policy_tensors(self.z, self.p, mask=self.legal, workspace=self.ws)
        self.dy.copy_((self.p - self.target) / self.m)
        az.weight_grad_tensors(self.dy, self.xq, self.dw, db=self.db, workspace=self.ws)
        az.quantize_tensors(self.dy, self.dq)
        az.matmul_tensors(self.dq, self.wt, self.dx, workspace=self.ws)

    def outputs(self):
        return [t.clone() for t in (self.xq.codes, self.wt.codes, self.z, self.p, self.dw, self.db, self.dx)]


@pytest.mark.parametrize("m,n,k", [(3, 40, 200), (96, 300, 520)])
def test_a_dense_head_forward_and_back(m, n, k):
    L = _Layer(m, n, k, 4)
    L.step()
    xc, xs = O.quantize(_host(L.x))
    wc, wsc = O.quantize(_host(L.w), 128)
    xv, wv = O.value(xc, xs), O.value(wc, wsc, 128)
    z = xv @ wv.T + _host(L.b)
    _check(_host(L.z), z, np.abs(xv) @ np.abs(wv).T + np.abs(_host(L.b)), k + 1, False)
    p = O.policy(_host(L.z), L.legal.cpu().numpy())
    assert np.abs(_host(L.p) - p).max() <= 1e-5
    dy = _host(L.dy)
    _check(_host(L.dw), dy.T @ xv, np.abs(dy).T @ np.abs(xv), m + 1, False)
    _check(_host(L.db), dy.sum(0), np.abs(dy).sum(0), m + 1, False)
    dv = O.value(*O.quantize(dy))
    _check(_host(L.dx), dv @ wv, np.abs(dv) @ np.abs(wv), n + 1, True, 2.0 ** -10)


def test_equal_calls_give_equal_bits_on_any_stream():
    import torch
    L = _Layer(130, 200, 700, 5)
    L.step()
    torch.cuda.synchronize()
    first = L.outputs()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        L.step()
    s.synchronize()
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(first, L.outputs()))


def test_a_captured_step_replays():
    import torch
    L = _Layer(70, 260, 390, 6)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        L.step()
    torch.cuda.current_stream().wait_stream(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        L.step()
    for i in range(4):
        L.x.copy_(_data(_rng(60 + i), 70, 390, "bf16"))
        g.replay()
        torch.cuda.synchronize()
        replayed = L.outputs()
        L.step()  # the program's own eager work between the replays
        torch.cuda.synchronize()
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(replayed, L.outputs())), i


def test_two_layers_at_once_on_two_streams():
    import torch
    layers = [_Layer(90, 200, 600, 7), _Layer(40, 500, 300, 8)]
    want = []
    for L in layers:
        L.step()
        torch.cuda.synchronize()
        want.append(L.outputs())
    streams = [torch.cuda.Stream() for _ in layers]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        for L, s in zip(layers, streams):
            with torch.cuda.stream(s):
                L.step()
    torch.cuda.synchronize()
    for L, w in zip(layers, want):
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(w, L.outputs()))


def test_no_rows_launch_nothing():
    az, torch = _az()
    b, _ = _coded(_rng(1), 20, 50)
    az.quantize_tensors(torch.empty((0, 50), device="cuda"), az.CodeMatrix.empty(0, 50))
    az.dequantize_tensors(az.CodeMatrix.empty(0, 50), torch.empty((0, 50), device="cuda"))
    az.matmul_tensors(az.CodeMatrix.empty(0, 50), b, torch.empty((0, 20), device="cuda"))
    az.matmul_tensors(b, az.CodeMatrix.empty(0, 50), torch.empty((20, 0), device="cuda"))
    torch.cuda.synchronize()


def test_tensor_checks():
    az, torch = _az()
    a, _ = _coded(_rng(1), 20, 50)
    b, _ = _coded(_rng(2), 30, 50)
    good = torch.empty((20, 30), device="cuda")
    for out in (torch.empty((20, 31), device="cuda"), good.half(), good.cpu(), good.t().contiguous().t()):
        with pytest.raises(ValueError):
            az.matmul_tensors(a, b, out)
    with pytest.raises(ValueError):
        az.matmul_tensors(a, b, good, bias=torch.empty((31,), device="cuda"))
    with pytest.raises(az.AzError):
        az.matmul_tensors(a, az.CodeMatrix.empty(30, 51), good)
    with pytest.raises(ValueError):
        az.quantize_tensors(torch.empty((20, 51), device="cuda"), a)
    with pytest.raises(ValueError):
        az.weight_grad_tensors(torch.empty((21, 30), dtype=torch.bfloat16, device="cuda"), a, torch.empty((30, 50), device="cuda"))
    with pytest.raises(az.AzError):
        az.weight_grad_tensors(torch.empty((20, 30), dtype=torch.bfloat16, device="cuda"), az.CodeMatrix.empty(20, 50, 128),
                               torch.empty((30, 50), device="cuda"))
    with pytest.raises(ValueError):
        az.CodeMatrix(torch.zeros((4, 32), dtype=torch.uint8, device="cuda"), torch.zeros((4, 2), dtype=torch.uint8, device="cuda"))
    # the last row's chunks have to be there as well
    scales = torch.zeros((4, 1), dtype=torch.uint8, device="cuda")
    short = torch.zeros((3 * 32 + 20,), dtype=torch.uint8, device="cuda")
    with pytest.raises(ValueError):
        az.CodeMatrix(short.as_strided((4, 20), (32, 1)), scales)
    with pytest.raises(ValueError):
        az.CodeMatrix(short[:20].clone().view(1, 20), scales[:1])
    az.CodeMatrix(torch.zeros((4, 32), dtype=torch.uint8, device="cuda")[:, :20], scales)
    with pytest.raises(az.AzError):  # rows that are not 16-byte chunks apart
        az.dequantize_tensors(az.CodeMatrix(torch.zeros((4, 20), dtype=torch.uint8, device="cuda").as_strided((3, 4), (20, 1)), scales[:3]),
                              torch.zeros((3, 4), device="cuda"))


# --------------------------------------------------------------------------- #
# Offsets past 32 bits
# --------------------------------------------------------------------------- #
def _decoded(codes, scales):
    """Values of a coded matrix with a scale for each row's blocks, float64, on its device."""
    import torch
    table = torch.tensor(O.TABLE, device=codes.device)
    s = torch.tensor([2.0 ** (b - 127) for b in range(256)], dtype=torch.float64, device=codes.device)
    return table[codes.long()] * s[scales.long()].repeat_interleave(128, dim=1)[:, :codes.shape[1]]


def test_offsets_past_32_bits():
    az, torch = _az()
    rows, cols = 36000, 131072  # 4.7 GB of codes
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.randn((rows, cols), generator=g, device="cuda", dtype=torch.bfloat16)
    q = az.CodeMatrix.empty(rows, cols)
    az.quantize_tensors(x, q)
    tail = az.CodeMatrix.empty(100, cols)
    az.quantize_tensors(x[-100:].clone(), tail)
    assert torch.equal(q.codes[-100:], tail.codes) and torch.equal(q.scales[-100:], tail.scales)
    # restored into the 9.4 GB it came from
    az.dequantize_tensors(q, x)
    assert torch.equal(x[-100:].double(), _decoded(tail.codes, tail.scales))
    del x
    # as the weights of a product, by the kernels of few and of more rows
    tv = _decoded(tail.codes, tail.scales)
    for m in (2, 40, 200):
        a = az.CodeMatrix.empty(m, cols)
        az.quantize_tensors(torch.randn((m, cols), generator=g, device="cuda"), a)
        out = torch.empty((m, rows), device="cuda")
        az.matmul_tensors(a, q, out)
        av = _decoded(a.codes, a.scales)
        want = torch.mm(av, tv.t().contiguous())
        assert bool(((out[:, -100:].double() - want).abs() <= cols * 2.0 ** -23 * torch.mm(av.abs(), tv.abs().t().contiguous())).all())
        other = torch.empty((rows, m), device="cuda")  # and as the activations
        az.matmul_tensors(q, a, other)
        assert bool(((other[-100:].t().double() - want).abs() <= cols * 2.0 ** -23 * torch.mm(av.abs(), tv.abs().t().contiguous())).all())
    # as a saved activation: only the last rows have a gradient
    dy = torch.zeros((rows, 24), device="cuda", dtype=torch.bfloat16)
    dy[-100:] = torch.randn((100, 24), generator=g, device="cuda").to(torch.bfloat16)
    dw, small = torch.empty((24, cols), device="cuda"), torch.empty((24, cols), device="cuda")
    az.weight_grad_tensors(dy, q, dw)
    az.weight_grad_tensors(dy[-100:].clone(), tail, small)
    y = dy[-100:].double()
    size = torch.mm(y.t().abs().contiguous(), tv.abs())
    want = torch.mm(y.t().contiguous(), tv)
    assert bool(((dw.double() - want).abs() <= 200 * 2.0 ** -23 * size).all())
    assert bool(((small.double() - want).abs() <= 200 * 2.0 ** -23 * size).all())


def test_outputs_past_32_bits():
    az, torch = _az()
    m, n = 40000, 30000  # 4.8 GB of fp32 results
    a, av = _coded(_rng(31), m, 20)
    b, bv = _coded(_rng(32), n, 20)
    out = torch.full((m, n), float("nan"), device="cuda")
    az.matmul_tensors(a, b, out)
    got = _host(out[-70:, -300:])
    _check(got, av[-70:] @ bv[-300:].T, np.abs(av[-70:]) @ np.abs(bv[-300:]).T, 21, False)
    assert bool(torch.isfinite(out.sum(dim=1)).all())
