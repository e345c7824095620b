"""Refusals of the stand-alone operators at the ends of their ranges and of workspaces that are too small, before
they touch a device."""

import paper_2609_37447_amd as az

from .test_operators_cpu import E, M, P


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
