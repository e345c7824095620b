"""The norm, 4-bit matrices and the drawn entry refuse bad arguments before they touch a device, and their float64
definitions (oracle/layer.py) agree with facts that they do not compute."""

import ctypes

import numpy as np
import pytest

import paper_2609_37447_amd as az
from oracle import layer as O

from .test_operators_cpu import E, U, M, P


def F(rows=4, cols=40, ld=32, ld_scales=4, codes=P, scales=P):
    return az.az_fp4_matrix(codes, scales, rows, cols, ld, ld_scales)


BAD = [(F(rows=-1), E), (F(cols=0), E), (F(ld=24), E), (F(ld=16), E), (F(ld_scales=1), E), (F(ld_scales=6), E), (F(codes=None), E),
       (F(scales=None), E), (F(codes=P + 8), E), (F(scales=P + 2), E), (F(rows=2 ** 31), U), (F(cols=2 ** 30 + 1, ld=2 ** 30, ld_scales=2 ** 26), U),
       (F(rows=2 ** 24, cols=128 * 128 + 1, ld=2 ** 14, ld_scales=1024), U)]


@pytest.mark.parametrize("m,status", BAD)
def test_bad_matrices_are_refused(m, status):
    L, good, codes = az.lib(), F(), M()
    far = 1 << 40
    assert L.az_nibbles_quantize(P, az.AZ_F32, far, m, None, None) == status
    assert L.az_nibbles_dequantize(m, P, az.AZ_F32, far, None) == status
    assert L.az_nibbles_matmul(m, good, None, P, az.AZ_F32, far, P, far, None) == status
    assert L.az_nibbles_matmul(good, m, None, P, az.AZ_F32, far, P, far, None) == status
    assert L.az_codes_nibbles_matmul(codes, m, None, P, az.AZ_F32, far, P, far, None) == status
    assert b"az_codes_nibbles_matmul" in L.az_last_error()


def test_bad_calls_on_matrices_are_refused():
    L, m = az.lib(), F()
    q = L.az_nibbles_quantize
    assert q(None, az.AZ_F32, 40, m, None, None) == E and q(P, az.AZ_INT8, 40, m, None, None) == E and q(P, az.AZ_F32, 39, m, None, None) == E
    assert q(P + 2, az.AZ_F32, 40, m, None, None) == E and q(P + 1, az.AZ_BF16, 40, m, None, None) == E and q(P, az.AZ_F32, 40, None, None, None) == E
    assert q(P, az.AZ_F32, 40, m, F(40, 5, 16), None) == E and q(P, az.AZ_F32, 40, m, F(39, 4, 16), None) == E
    assert q(P, az.AZ_F32, 40, m, F(40, 4, 8), None) == E
    assert q(None, az.AZ_F32, 40, F(rows=0, codes=None, scales=None), None, None) == az.AZ_OK
    d = L.az_nibbles_dequantize
    assert d(m, None, az.AZ_F32, 40, None) == E and d(m, P, 7, 40, None) == E and d(m, P, az.AZ_F32, 39, None) == E and d(None, P, az.AZ_F32, 40, None) == E
    for mm, a in ((L.az_nibbles_matmul, F), (L.az_codes_nibbles_matmul, M)):
        assert mm(a(cols=39), m, None, P, az.AZ_F32, 4, P, 1 << 40, None) == E
        assert mm(a(), m, None, P, az.AZ_INT8, 4, P, 1 << 40, None) == E and mm(a(), m, None, P, az.AZ_F32, 3, P, 1 << 40, None) == E
        assert mm(a(), m, None, None, az.AZ_F32, 4, P, 1 << 40, None) == E and mm(a(), m, P + 1, P, az.AZ_F32, 4, P, 1 << 40, None) == E
        assert mm(a(), m, None, P + 2, az.AZ_F32, 4, P, 1 << 40, None) == E and mm(a(), m, None, P, az.AZ_F32, 4, P + 8, 1 << 40, None) == E
        assert mm(None, m, None, P, az.AZ_F32, 4, P, 1 << 40, None) == E and mm(a(), None, None, P, az.AZ_F32, 4, P, 1 << 40, None) == E
        assert mm(a(rows=0), m, None, None, az.AZ_F32, 4, P, 1 << 40, None) == az.AZ_OK
        assert mm(a(), F(rows=0), None, None, az.AZ_F32, 4, P, 1 << 40, None) == az.AZ_OK
        assert mm(a(ld=1 << 27), m, None, P, az.AZ_F32, 4, P, 1 << 40, None) == U and mm(a(), F(ld=1 << 27), None, P, az.AZ_F32, 4, P, 1 << 40, None) == U
        assert mm(a(), F(ld_scales=1 << 26), None, P, az.AZ_F32, 4, P, 1 << 40, None) == U
        assert mm(a(rows=1, cols=16, ld=16), F(rows=2 ** 31 - 1, cols=16, ld=16), None, P, az.AZ_F32, 1 << 40, P, 1 << 40, None) == U
    assert L.az_nibbles_matmul(F(ld_scales=1 << 26), m, None, P, az.AZ_F32, 4, P, 1 << 40, None) == U


def test_workspaces_of_products():
    L = az.lib()
    a, c, b = F(333, 10240, 5120, 320), M(333, 10240, 10240), F(1880, 10240, 5120, 320)
    for mm, size, x in ((L.az_nibbles_matmul, az.az_nibbles_matmul_workspace, a), (L.az_codes_nibbles_matmul, az.az_codes_nibbles_matmul_workspace, c)):
        for dtype in (az.AZ_F32, az.AZ_BF16):
            need = size(x, b, dtype)
            assert need > 0 and need % (333 * 1880 * 4) == 0
            assert mm(x, b, None, P, dtype, 1880, P, need - 1, None) == E and mm(x, b, None, P, dtype, 1880, None, need, None) == E
            assert b"workspace" in L.az_last_error()
    top = 2 ** 63 - 1
    for bad in (F(rows=top, cols=10240), F(rows=333, cols=top), F(rows=0), F(rows=-1)):
        assert az.az_nibbles_matmul_workspace(bad, b, az.AZ_F32) == 0 and az.az_nibbles_matmul_workspace(a, bad, az.AZ_F32) == 0
        assert az.az_codes_nibbles_matmul_workspace(c, bad, az.AZ_F32) == 0
    assert L.az_nibbles_matmul_workspace(None, b, 0) == 0


def norm(**kw):
    v = dict(rows=4, cols=40, x=P, dtype=az.AZ_F32, eps=1e-6, ld_x=40, residual=None, ld_residual=0, weight=None, sum=None, ld_sum=0, y=P, ld_y=40, q=None)
    v.update(kw)
    return az.az_norm(*v.values())


def test_bad_norms_are_refused():
    L = az.lib()
    st = lambda **kw: L.az_rms_norm(norm(**kw), None)  # noqa: E731
    q = lambda *a, **kw: ctypes.addressof(keep.append(M(*a, **kw)) or keep[-1])  # noqa: E731
    keep = []
    assert L.az_rms_norm(None, None) == E
    assert st(rows=-1) == E and st(cols=0) == E and st(dtype=az.AZ_INT8) == E and st(x=None) == E and st(ld_x=39) == E and st(x=P + 2) == E
    assert st(rows=2 ** 31) == U and st(cols=2 ** 24 + 1, ld_x=1 << 30, ld_y=1 << 30) == U
    for eps in (0.0, -1e-6, float("nan"), float("inf"), 1e-45, 1e-39):
        assert st(eps=eps) == E
    assert st(y=None) == E and st(ld_y=39) == E and st(y=P + 1) == E
    assert st(residual=P, ld_residual=39) == E and st(residual=P + 2, ld_residual=40) == E and st(sum=P, ld_sum=39) == E and st(weight=P + 2) == E
    assert st(q=q(4, 41, 48)) == E and st(q=q(5, 40, 48)) == E and st(q=q(4, 40, 48, 128)) == E and st(q=q(4, 40, 40)) == E and st(q=q(codes=None)) == E
    assert st(rows=0, x=None, y=None) == az.AZ_OK
    assert b"az_rms_norm" in L.az_last_error()


def test_bad_norm_gradients_are_refused():
    L = az.lib()

    def st(ws=P, size=1 << 40, **kw):
        v = dict(rows=4, cols=40, dy=P, dtype=az.AZ_F32, eps=1e-6, ld_dy=40, h=P, ld_h=40, weight=None, dsum=None, ld_dsum=0, dx=P, ld_dx=40,
                 dweight=P, accumulate=0)
        v.update(kw)
        return L.az_rms_norm_grad(az.az_norm_grad(*v.values()), ws, size, None)

    need = az.az_rms_norm_grad_workspace(4, 40)
    assert need > 0 and need % 16 == 0
    assert L.az_rms_norm_grad(None, P, 1 << 40, None) == E
    assert st(rows=-1) == E and st(cols=0) == E and st(dtype=7) == E and st(eps=0.0) == E and st(rows=2 ** 31) == U and st(cols=2 ** 24 + 1) == U
    assert st(dy=None) == E and st(h=None) == E and st(ld_dy=39) == E and st(ld_h=39) == E and st(dsum=P, ld_dsum=39) == E and st(ld_dx=39) == E
    assert st(dx=None, dweight=None) == E and st(weight=P + 1) == E and st(dweight=P + 2) == E and st(dx=P + 2) == E
    assert st(size=need - 1) == E and st(ws=None) == E and st(ws=P + 4) == E
    assert b"workspace" in L.az_last_error()
    assert st(rows=0, dy=None, h=None, dx=None, dweight=None, ws=None, size=0) == az.AZ_OK
    top = 2 ** 63 - 1
    assert az.az_rms_norm_grad_workspace(0, 40) == az.az_rms_norm_grad_workspace(4, 0) == az.az_rms_norm_grad_workspace(-1, 40) == 0
    assert az.az_rms_norm_grad_workspace(top, 40) == az.az_rms_norm_grad_workspace(4, top) == 0
    for rows, cols in ((1, 1), (16384, 4096), (2 ** 31 - 1, 24), (7, 2 ** 24)):
        assert 4 * cols <= az.az_rms_norm_grad_workspace(rows, cols) <= 4 * cols * (min(rows, 16384) + 4)


def test_bad_draws_are_refused():
    L = az.lib()

    def st(out=P, prob=None, **kw):
        v = dict(logits=P, dtype=az.AZ_F32, rows=2, vocab=100, ld=100, u=P, temperature=None, top_k=None, top_p=None, min_p=None)
        v.update(kw)
        return L.az_logits_sample(az.az_sampling(*v.values()), out, prob, None)

    assert L.az_logits_sample(None, P, None, None) == E
    assert st(rows=-1) == E and st(vocab=0) == E and st(rows=(1 << 20) + 1) == U and st(vocab=(1 << 24) + 1, ld=1 << 30) == U
    assert st(logits=None) == E and st(dtype=az.AZ_INT8) == E and st(ld=99) == E and st(logits=P + 2) == E
    assert st(u=None) == E and st(out=None) == E
    for name in ("u", "temperature", "top_k", "top_p", "min_p"):
        assert st(**{name: P + 2}) == E
    assert st(out=P + 1) == E and st(prob=P + 2) == E
    assert st(rows=0, logits=None, u=None, out=None) == az.AZ_OK
    assert b"az_logits_sample" in L.az_last_error()


def test_struct_layouts():
    assert ctypes.sizeof(az.az_fp4_matrix) == 48 and ctypes.sizeof(az.az_norm) == 104
    assert ctypes.sizeof(az.az_norm_grad) == 112 and ctypes.sizeof(az.az_sampling) == 72


# --------------------------------------------------------------------------- #
# The definitions
# --------------------------------------------------------------------------- #
def test_definition_of_codes():
    assert O.scale_exponent(0.0) == 0 and O.scale_exponent(6.0) == 0 and O.scale_exponent(6.1) == 1 and O.scale_exponent(3.0) == -1
    assert O.scale_exponent(3.4e38) == 125 and O.scale_exponent(1e-40) == -125
    assert O.nearest(np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])).tolist() == [0, 2, 2, 4, 4, 6, 6]  # ties to the even code
    assert O.nearest(np.array([0.2500001, -0.7499999, 4.999, -5.001, -0.0])).tolist() == [1, 9, 6, 15, 8]
    rng = np.random.Generator(np.random.PCG64(1))
    x = rng.standard_normal((30, 70)) * 2.0 ** rng.integers(-20, 20, (30, 1))
    c, s = O.quantize(x)
    v = O.value(c, s)
    for i in range(30):  # every value is the nearest of its block's fifteen
        for j in range(70):
            assert np.abs(v[i, j] - x[i, j]) <= np.abs(O.TABLE * 2.0 ** (float(s[i, j // 32]) - 127) - x[i, j]).min() * (1 + 1e-12)
    assert np.array_equal(O.value(*O.quantize(v)), v)  # quantising stored values changes nothing
    p = O.packed(c[:, :69])
    assert p.shape == (30, 35) and np.array_equal(p[:, 3] & 15, c[:, 6]) and np.array_equal(p[:, 3] >> 4, c[:, 7]) and np.all(p[:, 34] >> 4 == 0)


def test_definition_of_the_norm_and_its_gradients():
    """Unit root-mean-square without eps; gradients by central differences of sum(dy * y): with a step t the error is
    t^2 f''' / 6, beside 2^-52 f / t."""
    rng = np.random.Generator(np.random.PCG64(2))
    h, dy, w, ds = rng.standard_normal((3, 17)), rng.standard_normal((3, 17)), rng.standard_normal(17), rng.standard_normal((3, 17))
    assert np.allclose(np.mean(O.norm(h, None, 1e-300)[0] ** 2, axis=1), 1.0, rtol=1e-14)
    dx, dw = O.norm_grad(dy, h, w, ds, 1e-3)
    loss = lambda h, w: np.sum(dy * O.norm(h, w, 1e-3)[0]) + np.sum(ds * h)  # noqa: E731
    t = 1e-5
    for i, j in ((0, 0), (1, 5), (2, 16)):
        d = np.zeros_like(h)
        d[i, j] = t
        assert abs((loss(h + d, w) - loss(h - d, w)) / (2 * t) - dx[i, j]) < 1e-8
        assert abs((loss(h, w + d[i]) - loss(h, w - d[i])) / (2 * t) - dw[j]) < 1e-8


def test_definition_of_the_draw():
    l = np.log(np.array([0.1, 0.4, 0.05, 0.4, 0.05]))
    at, w, _ = O.kept(l)
    assert at.tolist() == [0, 1, 2, 3, 4] and np.allclose(w / w.sum(), np.exp(l))
    assert O.kept(l, top_k=1)[0].tolist() == [1] and O.kept(l, top_k=2)[0].tolist() == [1, 3] and O.kept(l, top_k=4)[0].tolist() == [0, 1, 2, 3]
    assert O.kept(l, top_p=0.39)[0].tolist() == [1] and O.kept(l, top_p=0.41)[0].tolist() == [1, 3] and O.kept(l, top_p=0.0)[0].tolist() == [1]
    assert O.kept(l, top_k=3, top_p=0.85)[0].tolist() == [1, 3]   # of the 0.9 that are left
    assert O.kept(l, min_p=0.2)[0].tolist() == [0, 1, 3] and O.kept(l, min_p=3.0)[0].tolist() == [1, 3]
    assert O.kept(l, temperature=0.0)[0].tolist() == [1]
    assert O.kept(l, temperature=0.5)[1][1] / O.kept(l, temperature=0.5)[1][0] == pytest.approx(16.0)
    assert [O.draw(l, u)[0] for u in (0.0, 0.0999, 0.1001, 0.52, 0.56, 0.96)] == [0, 0, 1, 2, 3, 4]
    assert O.draw(np.full(3, -np.inf), 0.5)[:2] == (-1, 0.0) and O.draw(np.array([0.0, np.nan]), 0.5)[0] == -1
    assert O.draw(np.array([0.0, np.inf]), 0.5)[0] == -1 and O.draw(np.array([-np.inf, 2.0]), 0.99)[:2] == (1, 1.0)
