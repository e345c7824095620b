"""The stand-alone operators refuse bad arguments before they touch a device, and their
float64 definitions (oracle/codes.py) agree with facts that they do not compute."""

import ctypes

import numpy as np
import pytest

import paper_2609_37447_amd as az
from oracle import codes as O

E, U = az.AZ_ERR_INVALID_ARG, az.AZ_ERR_UNSUPPORTED
P = 4096  # an aligned address that no call below gets to use


def M(rows=4, cols=40, ld=48, scale_rows=1, codes=P, scales=P):
    return az.az_code_matrix(codes, scales, rows, cols, ld, scale_rows)


BAD = [(M(rows=-1), E), (M(cols=0), E), (M(ld=40), E), (M(ld=32), E), (M(scale_rows=2), E), (M(scale_rows=0), E), (M(codes=None), E),
       (M(scales=None), E), (M(codes=P + 8), E), (M(rows=2 ** 31), U), (M(cols=2 ** 30 + 1, ld=2 ** 30 + 16), U),
       (M(rows=2 ** 24, cols=128 * 128 + 1, ld=128 * 129), U)]


@pytest.mark.parametrize("m,status", BAD)
def test_bad_matrices_are_refused(m, status):
    L = az.lib()
    good = M()
    assert L.az_codes_quantize(P, az.AZ_F32, 1 << 40, m, None, None) == status
    assert L.az_codes_dequantize(m, P, az.AZ_F32, 1 << 40, None) == status
    assert L.az_codes_matmul(m, good, None, P, az.AZ_F32, 1 << 40, P, 1 << 40, None) == status
    assert L.az_codes_matmul(good, m, None, P, az.AZ_F32, 1 << 40, P, 1 << 40, None) == status
    if m.scale_rows == 1:
        assert L.az_codes_weight_grad(P, 1 << 40, 4, m, P, az.AZ_F32, 1 << 40, None, 0, P, 1 << 40, None) == status
    assert b"az_codes" in L.az_last_error()


def test_bad_calls_are_refused():
    L = az.lib()
    m = M()
    q = L.az_codes_quantize
    assert q(None, az.AZ_F32, 40, m, None, None) == E
    assert q(P, az.AZ_INT8, 40, m, None, None) == E
    assert q(P, az.AZ_F32, 39, m, None, None) == E
    assert q(P + 2, az.AZ_F32, 40, m, None, None) == E
    assert q(P + 1, az.AZ_BF16, 40, m, None, None) == E
    assert q(P, az.AZ_F32, 40, None, None, None) == E
    t = M(scale_rows=128)
    assert q(P, az.AZ_F32, 40, m, M(40, 4, 16, 128), None) == E     # rows with scales of their own have no transposed form
    assert q(P, az.AZ_F32, 40, t, M(40, 4, 16, 1), None) == E
    assert q(P, az.AZ_F32, 40, t, M(40, 5, 16, 128), None) == E
    assert q(P, az.AZ_F32, 40, t, M(40, 4, 8, 128), None) == E
    assert q(None, az.AZ_F32, 40, M(rows=0, codes=None, scales=None), None, None) == az.AZ_OK
    d = L.az_codes_dequantize
    assert d(m, None, az.AZ_F32, 40, None) == E and d(m, P, 7, 40, None) == E and d(m, P, az.AZ_F32, 39, None) == E
    assert d(None, P, az.AZ_F32, 40, None) == E
    mm = L.az_codes_matmul
    assert mm(m, M(cols=41), None, P, az.AZ_F32, 4, P, 1 << 40, None) == E
    assert mm(m, m, None, P, az.AZ_INT8, 4, P, 1 << 40, None) == E
    assert mm(m, m, None, P, az.AZ_F32, 3, P, 1 << 40, None) == E
    assert mm(m, m, None, None, az.AZ_F32, 4, P, 1 << 40, None) == E
    assert mm(m, m, P + 1, P, az.AZ_F32, 4, P, 1 << 40, None) == E
    assert mm(m, m, None, P + 2, az.AZ_F32, 4, P, 1 << 40, None) == E
    assert mm(M(rows=0), m, None, None, az.AZ_F32, 4, P, 1 << 40, None) == az.AZ_OK
    assert mm(m, M(rows=0), None, None, az.AZ_F32, 4, P, 1 << 40, None) == az.AZ_OK
    g = L.az_codes_weight_grad
    need = az.az_codes_weight_grad_workspace(4, 8, 40)
    ok = (P, 8, 8, m, P, az.AZ_F32, 40, None, 0, P, need, None)

    def grad(**kw):
        names = ("dy", "ld_dy", "n", "x", "dw", "dtype", "ld_dw", "db", "add", "ws", "size", "stream")
        return g(*[kw.get(k, v) for k, v in zip(names, ok)])

    assert grad(x=M(scale_rows=128)) == E and grad(n=-1) == E and grad(dy=None) == E and grad(dw=None) == E
    assert grad(ld_dy=7) == E and grad(ld_dw=39) == E and grad(dtype=az.AZ_INT8) == E and grad(db=P + 2) == E
    assert grad(dy=P + 1) == E and grad(dw=P + 2) == E and grad(ws=P + 8) == E and grad(x=None) == E
    assert grad(n=0) == az.AZ_OK


def test_workspaces_are_demanded():
    L = az.lib()
    rows, n, cols = 1 << 16, 64, 128  # few outputs of many rows: the sum is split
    need = az.az_codes_weight_grad_workspace(rows, n, cols)
    if need:
        x = M(rows=rows, cols=cols, ld=cols)
        assert L.az_codes_weight_grad(P, n, n, x, P, az.AZ_F32, cols, None, 0, P, need - 1, None) == E
        assert L.az_codes_weight_grad(P, n, n, x, P, az.AZ_F32, cols, None, 0, None, need, None) == E
    a, b = M(rows=64, cols=1 << 14, ld=1 << 14), M(rows=256, cols=1 << 14, ld=1 << 14)
    need = az.az_codes_matmul_workspace(a, b, az.AZ_BF16)
    if need:
        assert L.az_codes_matmul(a, b, None, P, az.AZ_BF16, 256, P, need - 1, None) == E
        assert L.az_codes_matmul(a, b, None, P, az.AZ_BF16, 256, None, need, None) == E
    assert L.az_codes_matmul(a, b, None, P, az.AZ_BF16, 256, P + 8, 1 << 40, None) == E
    assert az.az_codes_matmul_workspace(M(rows=0), b, az.AZ_BF16) == 0
    need = az.az_logits_policy_workspace(1, 1 << 17)
    if need:
        l = logits(rows=1, vocab=1 << 17, ld=1 << 17)
        assert L.az_logits_policy(l, 1, P, 1 << 17, P, need - 1, None) == E
        assert L.az_logits_policy(l, 1, P, 1 << 17, None, need, None) == E
    assert az.az_codes_weight_grad_workspace(0, 64, 128) == 0
    assert az.az_codes_weight_grad_workspace(-1, -1, -1) == 0
    assert az.az_logits_policy_workspace(0, 100) == 0 and az.az_logits_policy_workspace(-1, -1) == 0


def logits(**kw):
    v = dict(logits=P, dtype=az.AZ_F32, rows=2, vocab=100, ld=100, mask=None, mask_kind=0, ld_mask=0, bias=None, ld_bias=0,
             history=None, ld_history=0, max_history=0, lengths=None, penalties=None)
    v.update(kw)
    return az.az_logits(*v.values())


def test_bad_logits_are_refused():
    L = az.lib()

    def st(out=P, ld_out=100, ws=P, size=1 << 40, **kw):
        return L.az_logits_policy(logits(**kw), 1, out, ld_out, ws, size, None)

    assert L.az_logits_policy(None, 1, P, 100, P, 1 << 40, None) == E
    assert st(logits=None) == E and st(out=None) == E and st(rows=-1) == E and st(vocab=0) == E
    assert st(rows=(1 << 20) + 1) == U and st(vocab=(1 << 24) + 1, ld=1 << 25, ld_out=1 << 25) == U
    assert st(ld=99) == E and st(ld_out=99) == E and st(dtype=az.AZ_INT8) == E and st(logits=P + 2) == E and st(out=P + 2) == E
    assert st(mask_kind=3) == E and st(mask_kind=-1) == E
    assert st(mask_kind=1) == E and st(mask=P, mask_kind=1, ld_mask=99) == E
    assert st(mask=P, mask_kind=2, ld_mask=3) == E and st(mask=P + 1, mask_kind=2, ld_mask=4) == E
    assert st(bias=P, ld_bias=99) == E and st(bias=P + 1) == E
    assert st(max_history=-1) == E and st(history=P, ld_history=4, max_history=5, penalties=P) == E
    assert st(history=P, ld_history=5, max_history=5) == E and st(history=P + 2, ld_history=5, max_history=5, penalties=P) == E
    assert st(ws=P + 4) == E
    assert st(rows=0, logits=None, out=None) == az.AZ_OK
    assert b"az_logits_policy" in L.az_last_error()


def test_streams_and_operands_of_other_devices_are_refused():
    import torch
    from types import SimpleNamespace as N
    from paper_2609_37447_amd import _binding as B
    d0, d1 = torch.device("cuda", 0), torch.device("cuda", 1)
    assert B._on(d0, N(device=d0, cuda_stream=7), None, N(device=d0)) == 7
    with pytest.raises(ValueError, match="stream"):
        B._on(d0, N(device=d1, cuda_stream=7))
    with pytest.raises(ValueError, match="operands"):
        B._on(d0, N(device=d0, cuda_stream=7), N(device=d1))


def test_struct_layouts():
    assert ctypes.sizeof(az.az_code_matrix) == 48
    assert ctypes.sizeof(az.az_logits) == 112


# --------------------------------------------------------------------------- #
# The definitions
# --------------------------------------------------------------------------- #
def test_definition_scale_boundaries():
    assert O.scale_exponent(0.0) == 0 and O.scale_exponent(448.0) == 0 and O.scale_exponent(448.1) == 1
    assert O.scale_exponent(224.0) == -1 and O.scale_exponent(1.0) == -8 and O.scale_exponent(3.4e38) == 119
    assert O.scale_exponent(1e-40) == -117


def test_definition_round_trip_and_rounding():
    import torch
    rng = np.random.Generator(np.random.PCG64(1))
    for sr in (1, 128):
        x = rng.standard_normal((200, 300)) * 2.0 ** rng.integers(-20, 20, (200, 1))
        c, s = O.quantize(x, sr)
        v = O.value(c, s, sr)
        step = 2.0 ** (O.spread(s, 200, 300, sr).astype(float) - 127)
        assert np.all(np.abs(v - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * step))  # half a step, or half a sub-normal one
        c2, s2 = O.quantize(v, sr)
        assert np.array_equal(O.value(c2, s2, sr), v)           # quantising stored values changes nothing
        want = torch.from_numpy(x / step).float().to(torch.float8_e4m3fn).double().numpy() * step
        # torch's cast of the fp32 quotient (exact up to the fp32 rounding of x itself)
        assert np.mean(v != want) < 1e-5


def test_definition_policy_facts():
    rng = np.random.Generator(np.random.PCG64(2))
    l = rng.standard_normal((3, 50))
    ok = rng.random((3, 50)) < 0.4
    ok[1] = False
    p = O.policy(l, ok)
    assert np.allclose(p.sum(1), [1, 0, 1]) and np.all(p[~ok] == 0)
    assert np.allclose(p, O.policy(l + 3.0, ok))                # a shift changes nothing
    h, pen = [[4, 4, 7], [], [0]], [[2.0, 0.5, 0.25]] * 3
    a = O.adjusted_logits(l, history=h, penalties=pen)
    d = a - l
    assert np.count_nonzero(d) == 3
    assert np.isclose(a[0, 4], (l[0, 4] / 2 if l[0, 4] > 0 else l[0, 4] * 2) - 1.25)
    assert np.isclose(a[0, 7], (l[0, 7] / 2 if l[0, 7] > 0 else l[0, 7] * 2) - 0.75)
