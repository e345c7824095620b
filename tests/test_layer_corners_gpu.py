"""The norm, 4-bit matrices and the drawn entry as a layer uses them: one after the other, forward and back, on streams of their
own, captured and replayed, two at once; and at the corners of what they document: far rows, the largest sizes, equal
arguments.  Each step is compared with its float64 definition on the values that the step before it gave."""

import numpy as np
import pytest

from oracle import codes as C
from oracle import layer as O

from .test_codes_gpu import _az, _data, _host, _rng

pytestmark = pytest.mark.gpu
E = 2.0 ** -24


class _Layer:
    """A stream's sum and norm into e4m3 codes, product with 4-bit weights, adjusted logits, an entry drawn; the gradient of
    the logits through the transposed weights, the norm's and the layer's weights."""

    def __init__(self, m, n, k, seed):
        az, torch = _az()
        rng = _rng(m, n, k, seed)
        self.az, self.m, self.n, self.k = az, m, n, k
        self.x, self.r = _data(rng, m, k, "bf16").cuda(), _data(rng, m, k, "bf16").cuda()
        up = lambda x: torch.from_numpy(np.asarray(x, np.float32)).cuda()  # noqa: E731
        self.g, self.w, self.b = up(1 + 0.2 * rng.standard_normal(k)), up(0.1 * rng.standard_normal((n, k))), up(rng.standard_normal(n))
        self.legal = torch.from_numpy((rng.random((m, n)) < 0.3).astype(np.uint8)).cuda()
        self.legal[0] = 0
        self.u, self.t, self.p = up(rng.random(m)), up(rng.uniform(0.5, 1.5, m)), up(rng.uniform(0.5, 1.0, m))
        self.h, self.q = torch.empty_like(self.x), az.CodeMatrix.empty(m, k)
        self.wq, self.wt = az.Fp4Matrix.empty(n, k), az.Fp4Matrix.empty(k, n)
        self.z, self.l = torch.empty((m, n), device="cuda"), torch.empty((m, n), device="cuda")
        self.out, self.prob = torch.empty((m,), dtype=torch.int32, device="cuda"), torch.empty((m,), device="cuda")
        self.dz = (0.1 * up(rng.standard_normal((m, n)))).bfloat16()
        self.dq, self.dy = az.Fp4Matrix.empty(m, n), torch.empty((m, k), dtype=torch.bfloat16, device="cuda")
        self.ds, self.dx = _data(rng, m, k, "bf16").cuda(), torch.empty_like(self.x)
        self.dg, self.dw = torch.empty((k,), device="cuda"), torch.empty((n, k), device="cuda")
        need = (az.az_codes_nibbles_matmul_workspace(self.q.c, self.wq.c, az.AZ_F32), az.az_nibbles_matmul_workspace(self.dq.c, self.wt.c, az.AZ_BF16),
                az.az_rms_norm_grad_workspace(m, k), az.az_codes_weight_grad_workspace(m, n, k))
        self.ws = torch.empty((max(16, *need),), dtype=torch.uint8, device="cuda")

    def step(self, own=True, stream=None):
        az, kw = self.az, dict(workspace=self.ws if own else None, stream=stream)
        az.norm_tensors(self.x, q=self.q, residual=self.r, sum=self.h, weight=self.g, eps=1e-5, stream=stream)
        az.quantize_tensors(self.w, self.wq, self.wt, stream=stream)
        az.matmul_tensors(self.q, self.wq, self.z, bias=self.b, **kw)
        az.policy_tensors(self.z, self.l, mask=self.legal, probabilities=False, stream=stream)
        az.sample_tensors(self.l, self.u, self.out, prob=self.prob, temperature=self.t, top_p=self.p, stream=stream)
        az.quantize_tensors(self.dz, self.dq, stream=stream)
        az.matmul_tensors(self.dq, self.wt, self.dy, **kw)
        az.norm_grad_tensors(self.dy, self.h, self.dx, dsum=self.ds, weight=self.g, dw=self.dg, eps=1e-5, **kw)
        az.weight_grad_tensors(self.dz, self.q, self.dw, **kw)

    def outputs(self):
        return [t.clone() for t in (self.h, self.q.codes[:, :self.k], self.z, self.l, self.out, self.prob, self.dy, self.dx, self.dg, self.dw)]

    def clear(self):
        for t in (self.h, self.q.codes, self.q.scales, self.z, self.l, self.out, self.prob, self.dy, self.dx, self.dg, self.dw):
            t.fill_(5)


def _same(a, b):
    import torch
    return all(torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8)) for x, y in zip(a, b))


@pytest.mark.parametrize("m,n,k", [(1, 40, 200), (7, 300, 520), (200, 260, 1100)])
def test_a_layer_forward_and_back(m, n, k):
    az, torch = _az()
    L = _Layer(m, n, k, 1)
    L.step()
    assert torch.equal(L.h, (L.x.float() + L.r.float()).bfloat16())
    y = O.norm(_host(L.h), _host(L.g), 1e-5)[0]
    back = torch.empty((m, k), device="cuda")
    az.dequantize_tensors(L.q, back)
    a = _host(back)
    step = 2.0 ** (C.spread(L.q.scales.cpu().numpy(), m, k, 1).astype(np.float64) - 127)
    assert np.all(np.abs(a - y) <= np.maximum((2.0 ** -4 + 4 * E) * np.abs(y), 2.0 ** -10 * step))
    w, wt, dq = (O.value(*O.quantize(v)) for v in (_host(L.w), _host(L.w).T, _host(L.dz)))
    z = a @ w.T + _host(L.b)
    assert np.all(np.abs(_host(L.z) - z) <= (k + 1) * 2.0 ** -23 * (np.abs(a) @ np.abs(w).T + np.abs(_host(L.b))))
    for i in range(m):
        token, prob, near = O.draw(np.where(L.legal[i].cpu().numpy() != 0, _host(L.z)[i], -np.inf), float(L.u[i]), temperature=float(L.t[i]), top_p=float(L.p[i]))
        if near > 1e-9:
            assert int(L.out[i]) == token and abs(float(L.prob[i]) - prob) <= (E + 1e-9) * prob
    assert int(L.out[0]) == -1 and float(L.prob[0]) == 0.0
    dy, size = dq @ wt.T, np.abs(dq) @ np.abs(wt).T
    sums = (n + 1) * 2.0 ** -23 * size
    assert np.all(np.abs(_host(L.dy) - dy) <= 2.0 ** -8 * (np.abs(dy) + sums) + sums)
    dx, dg = O.norm_grad(_host(L.dy), _host(L.h), _host(L.g), _host(L.ds), 1e-5)
    r = O.norm(_host(L.h), None, 1e-5)[1]
    g, unit = _host(L.dy) * _host(L.g), _host(L.h) * r
    bound = r * (np.abs(g) + np.abs(unit) * np.mean(np.abs(g * unit), axis=1, keepdims=True))
    assert np.all(np.abs(_host(L.dx) - dx) <= 10 * E * bound * 1.01 + (2.0 ** -8 * 1.0001 + E) * np.abs(dx))
    assert np.all(np.abs(_host(L.dg) - dg) <= (m + 67) * E * np.sum(np.abs(_host(L.dy) * unit), axis=0))
    dw = _host(L.dz).T @ a
    assert np.all(np.abs(_host(L.dw) - dw) <= (m + 1) * 2.0 ** -23 * (np.abs(_host(L.dz)).T @ np.abs(a)))


@pytest.mark.parametrize("own", [True, False])
def test_on_another_stream_and_captured(own):
    """Workspaces given, and made inside the call on its stream and in the captured graph."""
    import torch
    L = _Layer(90, 300, 700, 2)
    L.step(own)
    torch.cuda.synchronize()
    want = L.outputs()
    L.clear()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    L.step(own, stream=s)
    s.synchronize()
    assert _same(want, L.outputs())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        L.step(own)
    for i in range(4):
        L.x.copy_(_data(_rng(70 + i), 90, 700, "bf16"))
        L.u.fill_(0.2 * i + 0.1)
        L.clear()
        g.replay()
        torch.cuda.synchronize()
        got = L.outputs()
        L.clear()
        L.step(own)  # the program's own eager work between the replays
        torch.cuda.synchronize()
        assert _same(got, L.outputs()), i


def test_two_layers_at_once():
    import torch
    layers = [_Layer(60, 200, 9000, 3), _Layer(40, 500, 300, 4)]
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
        assert _same(w, L.outputs())


def _far_rows(t, ld):
    """t in rows ld elements apart, on memory that is otherwise not written."""
    import torch
    rows, cols = t.shape
    v = torch.empty((rows - 1) * ld + cols, dtype=t.dtype, device="cuda").as_strided((rows, cols), (ld, 1))
    v.copy_(t)
    return v


def test_rows_past_32_bit_offsets():
    az, torch = _az()
    ld = (1 << 31) // 2 + 4099  # three rows of bf16: byte offsets past 2^32, element offsets past 2^31
    for cols in (1000, 1003):
        t = _data(_rng(cols, 5), 3, cols, "bf16").cuda()
        dy = _data(_rng(cols, 6), 3, cols, "bf16").cuda()
        far = _far_rows(t, ld)
        y, y2, q, q2 = torch.empty_like(t), _far_rows(torch.zeros_like(t), ld), az.CodeMatrix.empty(3, cols), az.CodeMatrix.empty(3, cols)
        az.norm_tensors(t, y=y, q=q)
        az.norm_tensors(far, y=y2, q=q2)
        assert torch.equal(y, y2) and torch.equal(q.codes[:, :cols], q2.codes[:, :cols])
        del y2
        dx, dx2, dw, dw2 = torch.empty_like(t), _far_rows(torch.zeros_like(t), ld), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
        az.norm_grad_tensors(dy, t, dx, dw=dw)
        az.norm_grad_tensors(dy, far, dx2, dw=dw2)
        assert torch.equal(dx, dx2) and torch.equal(dw, dw2)
        del dx2
        f, f2, back = az.Fp4Matrix.empty(3, cols), az.Fp4Matrix.empty(3, cols), _far_rows(torch.zeros_like(t), ld)
        az.quantize_tensors(t, f)
        az.quantize_tensors(far, f2)
        assert torch.equal(f.codes[:, :cols // 2], f2.codes[:, :cols // 2])
        az.dequantize_tensors(f, y)
        az.dequantize_tensors(f, back)
        assert torch.equal(y, back)
        del back
        u, out, out2 = torch.full((3,), 0.37, device="cuda"), torch.empty(3, dtype=torch.int32, device="cuda"), torch.empty(3, dtype=torch.int32, device="cuda")
        az.sample_tensors(t, u, out)
        az.sample_tensors(far, u, out2)
        assert torch.equal(out, out2) and int(out.min()) >= 0
        del far
        torch.cuda.empty_cache()


def test_the_longest_rows():
    az, torch = _az()
    v = 1 << 24
    x = torch.randn((2, v), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    y, q = torch.empty_like(x), az.CodeMatrix.empty(2, v)
    az.norm_tensors(x, y=y, q=q)
    want = x.double() / torch.sqrt((x.double() ** 2).mean(dim=1, keepdim=True) + float(np.float32(1e-6)))
    assert bool(((y.double() - want).abs() <= 3.1 * E * want.abs()).all())
    codes = az.CodeMatrix.empty(2, v)
    az.quantize_tensors(y, codes)
    assert torch.equal(codes.codes, q.codes) and torch.equal(codes.scales, q.scales)
    dw = torch.empty((v,), device="cuda")
    az.norm_grad_tensors(x, x, y, dw=dw)
    u = want
    assert bool(((dw.double() - (x.double() * u).sum(dim=0)).abs() <= 8 * E * (x.double() * u).abs().sum(dim=0)).all())
    # drawn: the weights are whole multiples of 2^-38, each off by half of one
    p = torch.softmax(x.double(), dim=1)
    sums = p.cumsum(dim=1)
    u = torch.tensor([0.25, 0.8125], device="cuda")
    for kw in ({}, {"top_k": torch.tensor([v, v - 1], dtype=torch.int32, device="cuda")}):
        out, prob = torch.empty(2, dtype=torch.int32, device="cuda"), torch.empty(2, device="cuda")
        az.sample_tensors(x, u, out, prob=prob, **kw)
        for i in range(2):
            j = int(out[i])
            lo, hi = float(sums[i, j - 1]), float(sums[i, j])
            assert lo - 1e-4 * p[i, j] <= float(u[i]) <= hi + 1e-4 * p[i, j]
            assert abs(float(prob[i]) - float(p[i, j])) <= 1e-6 * float(p[i, j])
    # greedy, and far more ties than fit anywhere
    x.fill_(1.0)
    out = torch.empty(2, dtype=torch.int32, device="cuda")
    az.sample_tensors(x, u, out, temperature=torch.zeros(2, device="cuda"))
    assert out.tolist() == [0, 0]
    az.sample_tensors(x, u, out, top_k=torch.tensor([1 << 23, 1 << 20], dtype=torch.int32, device="cuda"), top_p=torch.tensor([0.5, 1.0], device="cuda"))
    assert out.tolist() == [1 << 20, 13 << 16]


def test_many_rows():
    az, torch = _az()
    rows = 1 << 20
    l = torch.zeros((rows, 5), device="cuda")
    u = (torch.arange(rows, device="cuda") % 1000).float() / 1000 + 0.0005
    out = torch.empty(rows, dtype=torch.int32, device="cuda")
    az.sample_tensors(l, u, out)
    assert torch.equal(out, (u.double() * 5).to(torch.int32))
    x = torch.randn((300001, 24), device="cuda").bfloat16()
    y, dw = torch.empty_like(x), torch.empty(24, device="cuda")
    az.norm_tensors(x, y=y)
    d = x.double()
    unit = d / torch.sqrt((d * d).mean(dim=1, keepdim=True) + 1e-6)
    assert bool(((y.double() - unit).abs() <= (2.0 ** -8 + 1e-6) * unit.abs()).all())
    az.norm_grad_tensors(x, x, None, dw=dw)
    assert bool(((dw.double() - (d * unit).sum(dim=0)).abs() <= (300001 / 16 + 100) * E * (d * unit).abs().sum(dim=0)).all())


def test_one_matrix_as_both_operands():
    az, torch = _az()
    x = _data(_rng(9), 70, 900, "f32")
    f = az.Fp4Matrix.empty(70, 900)
    az.quantize_tensors(x.cuda(), f)
    v, o = O.value(*O.quantize(x.numpy())), torch.empty((70, 70), device="cuda")
    az.matmul_tensors(f, f, o)
    assert np.all(np.abs(_host(o) - v @ v.T) <= 900 * 2.0 ** -23 * (np.abs(v) @ np.abs(v).T))
    assert torch.equal(o, o.t())


def test_no_rows_of_matrices():
    az, torch = _az()
    none, some = az.Fp4Matrix.empty(0, 100), az.Fp4Matrix.empty(3, 100)
    az.matmul_tensors(none, some, torch.empty((0, 3), device="cuda"))
    az.matmul_tensors(some, none, torch.empty((3, 0), device="cuda"))
    az.matmul_tensors(az.CodeMatrix.empty(0, 100), some, torch.empty((0, 3), device="cuda"))
    az.quantize_tensors(torch.empty((0, 100), device="cuda"), none)
    az.dequantize_tensors(none, torch.empty((0, 100), device="cuda"))
    az.sample_tensors(torch.empty((0, 7), device="cuda"), torch.empty(0, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"))
