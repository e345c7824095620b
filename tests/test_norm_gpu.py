"""The root-mean-square norm and its gradients on the GPU against their float64 definitions (oracle/layer.py).

Tolerances, E = 2^-24 (half a step of fp32):
  sum: exact, an fp32 sum rounded to the type.
  y: r, h r and (h r) w are rounded once each (sums are fp64): 3 E |y|, in bf16 2^-8 |y| more; below 2^-126 steps are 2^-149.
  codes: of an fp32 y that is at hand, exactly its definition's; otherwise an e4m3 step of a value that is 3 E off.
  dx = r (g - u m) + dsum: at most nine roundings reach the term of u m (u 2, m 3, the product, the
      difference, r, the last product) and the sum is one more: 10 E r (|g| + |u| mean|g u|) + E |dx|.
  dweight: 3 roundings a term (r, u, the product) and one for each of at most rows + 64 additions, in units of sum |dy u|.
"""

import numpy as np
import pytest

from oracle import codes as C
from oracle import layer as O

from .test_codes_gpu import _az, _rng, _strided

pytestmark = pytest.mark.gpu
E = 2.0 ** -24
SHAPES = [(1, 1), (1, 16), (3, 17), (2, 127), (5, 128), (33, 129), (4, 255), (70, 512), (9, 513), (3, 1024), (5, 1025), (2, 2049),
          (3, 4096), (7, 5000), (2, 8192), (2, 16384), (3, 16385), (2, 40001), (300, 40)]


def _data(rng, rows, cols, dtype, size=1.0):
    import torch
    t = torch.from_numpy((size * rng.standard_normal((rows, cols)) * np.exp(rng.standard_normal((1, cols)))).astype(np.float32))
    return t.to(torch.bfloat16) if dtype == "bf16" else t


def _host(t):
    return t.double().cpu().numpy()


def _rounded(t, like):
    return t.float().to(like.dtype)


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("residual,weight,pad,offset", [(True, True, 0, 0), (False, True, 3, 1), (True, False, 16, 0), (False, False, 0, 5)])
def test_norm(rows, cols, dtype, residual, weight, pad, offset):
    az, torch = _az()
    rng = _rng(rows, cols, 1)
    x, r = _data(rng, rows, cols, dtype), _data(rng, rows, cols, dtype)
    w = torch.from_numpy((1 + 0.3 * rng.standard_normal(cols)).astype(np.float32)) if weight else None
    xd, _ = _strided(x, pad, offset=offset)
    rd = _strided(r, pad + 8, offset=offset)[0] if residual else None
    sd, swhole = _strided(torch.zeros_like(x), pad + 1, fill=7.0, offset=offset)
    yd, ywhole = _strided(torch.zeros_like(x), pad + 2, fill=7.0, offset=offset)
    codes = torch.full((rows + 1, -(-cols // 16) * 16 + 16), 0xAB, dtype=torch.uint8, device="cuda")
    scales = torch.full((rows, -(-cols // 128)), 0xCD, dtype=torch.uint8, device="cuda")
    q = az.CodeMatrix(codes[:rows], scales, cols)
    az.norm_tensors(xd, y=yd, q=q, residual=rd, sum=sd if residual else None, weight=w.cuda() if weight else None, eps=1e-5)
    h = (x.float() + r.float()).to(x.dtype) if residual else x
    if residual:
        assert torch.equal(sd.cpu(), h)
        assert int((swhole != 7.0).sum()) <= rows * cols
    want, _ = O.norm(h.double().numpy(), w.numpy() if weight else None, 1e-5)
    got = _host(yd)
    half = 2.0 ** -8 if dtype == "bf16" else 0.0
    assert np.all(np.abs(got - want) <= (3 * E + half) * (1 + 1e-6) * np.abs(want) + 2.0 ** -149)
    outside = ywhole.clone()
    outside[offset:offset + rows * (cols + pad + 2)].view(rows, -1)[:, :cols] = 7.0
    assert bool((outside == 7.0).all())  # nothing beside the rows is written
    c, s = codes.cpu().numpy(), scales.cpu().numpy()
    assert np.all(c[:rows, cols:] == 0xAB) and np.all(c[rows:] == 0xAB)
    if dtype == "f32":
        wc, ws = C.quantize(got)
        assert np.array_equal(c[:rows, :cols], wc) and np.array_equal(s, ws)
    else:
        step = 2.0 ** (C.spread(s, rows, cols, 1).astype(np.float64) - 127)
        assert np.all(np.abs(C.value(c[:rows, :cols], s) - want) <= np.maximum((2.0 ** -4 + 4 * E) * np.abs(want), 2.0 ** -10 * step))
        wc, ws = C.quantize(want)
        assert np.mean(s != ws) < 1e-3


@pytest.mark.parametrize("cols", [100, 4096, 20000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norm_in_place(cols, dtype):
    az, torch = _az()
    rng = _rng(cols, 2)
    x, r = _data(rng, 5, cols, dtype).cuda(), _data(rng, 5, cols, dtype).cuda()
    s, y = torch.empty_like(x), torch.empty_like(x)
    az.norm_tensors(x, y=y, residual=r, sum=s)
    a, b = x.clone(), r.clone()
    y2 = torch.empty_like(x)
    az.norm_tensors(a, y=y2, residual=b, sum=b)  # the stream, updated in its place
    assert torch.equal(b, s) and torch.equal(y2, y)
    az.norm_tensors(a, y=a, residual=r, sum=s)   # the result in x's place
    assert torch.equal(a, y)
    a = x.clone()
    az.norm_tensors(a, residual=r, sum=a)        # the sum alone
    assert torch.equal(a, s)


@pytest.mark.parametrize("cols", [130, 20000])
def test_norm_special_rows(cols):
    az, torch = _az()
    x = torch.ones((6, cols))
    x[0] = 0.0
    x[1, 3] = float("nan")
    x[2, 3] = float("inf")
    x[3] = 1e30   # squares past fp32
    x[4] = 1e-30  # and below it
    x[5, :] = 3e38
    y, q = torch.empty((6, cols), device="cuda"), az.CodeMatrix.empty(6, cols)
    az.norm_tensors(x.cuda(), y=y, q=q, eps=1e-12)
    y = y.cpu()
    assert bool((y[0] == 0).all()) and bool(torch.isnan(y[1]).all())
    assert bool(torch.isnan(y[2, 3])) and bool((y[2, 4:] == 0).all())
    want = O.norm(x.double().numpy()[3:], None, np.float64(np.float32(1e-12)))[0]
    # (a root of 3e38 has an inverse below 2^-126, with two bits less)
    assert np.all(np.abs(y[3:].double().numpy() - want) <= 8 * E * np.abs(want) + 2.0 ** -149)
    codes = q.codes.cpu()[:, :cols]
    assert bool((codes[1] == 0x7F).all()) and int(codes[2, 3]) == 0x7F and bool((codes[0] == 0).all())


def _grad_case(rows, cols, dtype, weight, dsum, pad=0, offset=0):
    az, torch = _az()
    rng = _rng(rows, cols, 3)
    h, dy, ds = (_data(rng, rows, cols, dtype) for _ in range(3))
    w = torch.from_numpy((1 + 0.3 * rng.standard_normal(cols)).astype(np.float32)) if weight else None
    dev = [_strided(t, pad + i, offset=offset)[0] for i, t in enumerate((h, dy, ds))]
    dx, whole = _strided(torch.zeros_like(h), pad + 5, fill=7.0, offset=offset)
    dw = torch.full((cols,), 0.5, device="cuda")
    az.norm_grad_tensors(dev[1], dev[0], dx, dsum=dev[2] if dsum else None, weight=w.cuda() if weight else None, dw=dw, eps=1e-5)
    want_x, want_w = O.norm_grad(dy.double().numpy(), h.double().numpy(), w.numpy() if weight else None, ds.double().numpy() if dsum else None, 1e-5)
    hh, dd = h.double().numpy(), dy.double().numpy()
    r = O.norm(hh, None, 1e-5)[1]
    g, u = dd * (w.double().numpy() if weight else 1.0), hh * r
    size = r * (np.abs(g) + np.abs(u) * np.mean(np.abs(g * u), axis=1, keepdims=True))
    half = 2.0 ** -8 if dtype == "bf16" else E
    assert np.all(np.abs(_host(dx) - want_x) <= 10 * E * size * (1 + half) + half * (1 + 1e-6) * np.abs(want_x) + E * np.abs(want_x))
    bound_w = (rows + 67) * E * np.sum(np.abs(dd * u), axis=0)
    assert np.all(np.abs(_host(dw) - want_w) <= bound_w)
    assert int((whole != 7.0).sum()) <= rows * cols
    return dev, w, dx, dw, want_w, bound_w, ds


@pytest.mark.parametrize("rows,cols", SHAPES + [(1000, 200), (2500, 64), (600, 1030)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("weight,dsum,pad,offset", [(True, True, 0, 0), (False, False, 3, 1)])
def test_norm_grad(rows, cols, dtype, weight, dsum, pad, offset):
    az, torch = _az()
    dev, w, dx, dw, want_w, bound_w, ds = _grad_case(rows, cols, dtype, weight, dsum, pad, offset)
    again, dw2, wd = dev[1].clone(), dw.clone(), w.cuda() if weight else None
    az.norm_grad_tensors(again, dev[0].contiguous(), again, dsum=dev[2] if dsum else None, weight=wd, dw=dw2, eps=1e-5, accumulate=True)
    assert torch.equal(again, dx)  # in dy's place
    assert np.all(np.abs(_host(dw2) - 2 * want_w) <= 2 * bound_w + 2 * E * np.abs(2 * want_w))
    alone = torch.zeros_like(dw)
    az.norm_grad_tensors(dev[1], dev[0], None, weight=wd, dw=alone, eps=1e-5)
    assert torch.equal(alone, dw)
    only = torch.zeros_like(dx)
    az.norm_grad_tensors(dev[1], dev[0], only, dsum=dev[2] if dsum else None, weight=wd, eps=1e-5)
    assert torch.equal(only, dx)


@pytest.mark.parametrize("rows,cols", SHAPES + [(600, 1030), (400, 8199)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("weight,pad,offset", [(True, 0, 0), (False, 3, 1), (True, 16, 5)])
def test_results_in_their_inputs_place(rows, cols, dtype, weight, pad, offset):
    """y in x's, the sum in x's and in the residual's, dx in dsum's and in dy's, padded rows too: the same bits as elsewhere, and
    nothing between the rows is written."""
    az, torch = _az()
    rng = _rng(rows, cols, 12)
    x, r, d = (_data(rng, rows, cols, dtype) for _ in range(3))
    w = torch.from_numpy((1 + 0.3 * rng.standard_normal(cols)).astype(np.float32)).cuda() if weight else None

    def place(t):
        v, whole = _strided(t, pad, fill=7.0, offset=offset)
        return v, whole

    def beside(v, whole):
        v.fill_(7.0)
        return bool((whole == 7.0).all())

    xd, rd, dd = (place(t)[0] for t in (x, r, d))
    y, y2, s, dx, dx2 = (place(torch.zeros_like(x))[0] for _ in range(5))
    az.norm_tensors(xd, y=y, weight=w)
    az.norm_tensors(xd, y=y2, residual=rd, sum=s, weight=w)
    az.norm_grad_tensors(dd, xd, dx, dsum=rd, weight=w)
    az.norm_grad_tensors(dd, xd, dx2, weight=w)
    a, whole = place(x)
    az.norm_tensors(a, y=a, weight=w)
    assert torch.equal(a, y) and beside(a, whole)
    a, whole = place(x)
    az.norm_tensors(a, y=a, residual=rd, sum=s.zero_(), weight=w)
    assert torch.equal(a, y2) and beside(a, whole)
    for t in (x, r):
        a, whole = place(t)
        out = place(torch.zeros_like(x))[0]
        az.norm_tensors(a if t is x else xd, y=out, residual=rd if t is x else a, sum=a, weight=w)
        assert torch.equal(a, s) and torch.equal(out, y2) and beside(a, whole)
    a, whole = place(r)
    az.norm_grad_tensors(dd, xd, a, dsum=a, weight=w)
    assert torch.equal(a, dx) and beside(a, whole)
    a, whole = place(d)
    az.norm_grad_tensors(a, xd, a, dsum=rd, weight=w)
    assert torch.equal(a, dx) and beside(a, whole)
    a, whole = place(d)
    az.norm_grad_tensors(a, xd, a, weight=w)
    assert torch.equal(a, dx2) and beside(a, whole)


def test_norm_grad_against_differences():
    """Central differences of the kernel's own loss, sum(dy * y) in fp64: with a step t its error is t^2 f''' / 6 and E |y| dy / t."""
    az, torch = _az()
    rows, cols, t = 3, 40, 2.0 ** -8
    rng = _rng(11)
    x, dy = _data(rng, rows, cols, "f32"), _data(rng, rows, cols, "f32")
    w = torch.from_numpy((1 + 0.3 * rng.standard_normal(cols)).astype(np.float32)).cuda()
    dx, dw = torch.empty((rows, cols), device="cuda"), torch.empty((cols,), device="cuda")
    az.norm_grad_tensors(dy.cuda(), x.cuda(), dx, weight=w, dw=dw)

    def loss(xx, ww):
        y = torch.empty((rows, cols), device="cuda")
        az.norm_tensors(xx.cuda(), y=y, weight=ww)
        return float((y.cpu().double() * dy.double()).sum())

    noise = 4 * E * float((dy.double().abs() * 10).sum()) / t
    for i, j in ((0, 0), (1, 7), (2, 39)):
        a, b = x.clone(), x.clone()
        a[i, j] += t
        b[i, j] -= t
        step = float(a[i, j].double() - b[i, j].double())
        assert abs((loss(a, w) - loss(b, w)) / step - float(dx[i, j])) <= noise + 1e-3 * float(dx.abs().max())
        a, b = w.clone(), w.clone()
        a[j] += t
        b[j] -= t
        step = float(a[j].double() - b[j].double())
        assert abs((loss(x, a) - loss(x, b)) / step - float(dw[j])) <= noise + 1e-6 * float(dw.abs().max())


def test_no_rows():
    az, torch = _az()
    none = torch.empty((0, 64), device="cuda")
    az.norm_tensors(none, y=none.clone())
    dw = torch.full((64,), 3.0, device="cuda")
    az.norm_grad_tensors(none, none, none.clone(), dw=dw, accumulate=True)
    assert bool((dw == 3.0).all())
    az.norm_grad_tensors(none, none, none.clone(), dw=dw)
    assert bool((dw == 0.0).all())
