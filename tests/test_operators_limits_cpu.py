"""Refusals of the stand-alone operators at the ends of their ranges and of workspaces that are too small, before
they touch a device."""

import paper_2609_37447_amd as az

from .test_operators_cpu import E, U, M, P


def test_a_workspace_a_byte_too_small_is_refused():
    L = az.lib()
    a, b = M(rows=333, cols=10240, ld=10240), M(rows=1880, cols=10240, ld=10240)
    for dtype in (az.AZ_F32, az.AZ_BF16):
        need = az.az_codes_matmul_workspace(a, b, dtype)
        assert need > 0 and need % (333 * 1880 * 4) == 0  # fp32 sums over parts
        assert L.az_codes_matmul(a, b, None, P, dtype, 1880, P, need - 1, None) == E
        assert L.az_codes_matmul(a, b, None, P, dtype, 1880, None, need, None) == E
        assert L.az_codes_matmul(a, b, None, P, dtype, 1880, P + 4, need, None) == E
        assert b"workspace" in L.az_last_error()
    need = az.az_codes_weight_grad_workspace(1 << 16, 64, 128)
    assert need > 0
    x = M(rows=1 << 16, cols=128, ld=128)
    assert L.az_codes_weight_grad(P, 64, 64, x, P, az.AZ_F32, 128, None, 0, P, need - 1, None) == E
    need = az.az_logits_policy_workspace(1, 1 << 17)
    assert need > 0
    l = az.az_logits(P, az.AZ_F32, 1, 1 << 17, 1 << 17)
    assert L.az_logits_policy(l, 1, P, 1 << 17, P, need - 1, None) == E
    assert L.az_logits_policy(l, 1, P, 1 << 17, None, need, None) == E


def test_more_tiles_than_a_launch_has_are_refused():
    # the largest sizes that matrices may have: 2^24 tiles of 256 threads, one launch's limit and one more
    L, top = az.lib(), 2 ** 31 - 1
    assert L.az_codes_quantize(P, az.AZ_F32, 1, M(rows=top, cols=1, ld=16, scale_rows=128), None, None) == U
    for dtype in (az.AZ_F32, az.AZ_BF16):
        assert L.az_codes_matmul(M(rows=1, cols=16, ld=16), M(rows=top, cols=16, ld=16), None, P, dtype, top, P, 1 << 40, None) == U
    assert az.az_codes_weight_grad_workspace(1, top, 16) == 0
    assert L.az_codes_weight_grad(P, 1 << 31, top, M(rows=1, cols=16, ld=16), P, az.AZ_F32, 16, P, 0, None, 0, None) == U
    assert b"launch" in L.az_last_error()


def test_no_rows_have_a_transposed_form():
    L, none = az.lib(), M(rows=0, scale_rows=128, codes=None, scales=None)
    q = L.az_codes_quantize
    assert q(None, az.AZ_F32, 40, none, M(rows=40, cols=0, ld=0, scale_rows=128, codes=None, scales=None), None) == az.AZ_OK
    assert q(None, az.AZ_F32, 40, none, M(rows=40, cols=5, ld=16, scale_rows=128), None) == az.AZ_OK  # (it has no shape to hold it against)
    assert q(None, az.AZ_F32, 40, none, M(rows=40, cols=0, ld=0, scale_rows=1), None) == E


def test_sizes_that_are_refused_have_no_workspace():
    L, top = az.lib(), 2 ** 63 - 1
    assert az.az_logits_policy_workspace(1, 2 ** 31 - 1) == 0 and az.az_logits_policy_workspace(2 ** 31 - 1, 1 << 24) == 0
    assert az.az_logits_policy_workspace(1 << 20, 1 << 24) > 0
    assert az.az_codes_weight_grad_workspace(top, 64, 128) == 0 and az.az_codes_weight_grad_workspace(1 << 16, 64, top) == 0
    assert az.az_codes_weight_grad_workspace(2 ** 31 - 1, 64, 128) > 0
    good = M(rows=333, cols=10240, ld=10240)
    for bad in (M(rows=top, cols=10240, ld=10240), M(rows=333, cols=top, ld=10240), M(rows=2 ** 31, cols=1 << 20, ld=1 << 20)):
        assert az.az_codes_matmul_workspace(bad, good, az.AZ_BF16) == 0 and az.az_codes_matmul_workspace(good, bad, az.AZ_BF16) == 0
    assert L.az_logits_policy(az.az_logits(P, az.AZ_F32, 1, 2 ** 31 - 1, 2 ** 31), 1, P, 2 ** 31, None, 0, None) == U
