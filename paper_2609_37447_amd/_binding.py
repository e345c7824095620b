"""ctypes binding of the C ABI in include/az.h (argument marshalling only).

Every computation runs in the HIP library; this module only converts Python
arguments to the C types and raises on a non-zero status.  It fails loudly if
the library has not been built.
"""

from __future__ import annotations

import ctypes
import os
from sys import modules as _modules  # (of calls on tensors, whose module is there: an import statement takes five times as long)

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libaz_mi355x.so")

AZ_ABI_VERSION = 2
AZ_POLICY_PLANES, AZ_POLICY_FROMTO = 0, 1
AZ_VALUE_TANH, AZ_VALUE_WDL = 0, 1
AZ_F32, AZ_BF16, AZ_INT8, AZ_FP8_E4M3 = 0, 1, 2, 3
DTYPES = {"f32": AZ_F32, "bf16": AZ_BF16, "int8": AZ_INT8, "fp8": AZ_FP8_E4M3}
AZ_OK, AZ_ERR_INVALID_ARG, AZ_ERR_UNSUPPORTED, AZ_ERR_NOMEM, AZ_ERR_DEVICE = 0, -1, -2, -3, -4

# Every symbol include/az.h declares.
EXPORTS = ("az_weight_count", "az_net_load", "az_eval_batch", "az_eval_batch_wdl", "az_net_moves",
           "az_net_set_tiling",
           "az_net_tiling_for", "az_net_device_bytes", "az_net_free", "az_compare_outputs",
           "az_pipeline_create", "az_pipeline_slot", "az_pipeline_submit", "az_pipeline_query",
           "az_pipeline_wait", "az_pipeline_drive", "az_pipeline_free", "az_debug_fail_allocation",
           "az_debug_live_allocations", "az_eval_batch_compact_noalloc",
           "az_codes_quantize", "az_codes_dequantize", "az_codes_matmul", "az_codes_matmul_workspace",
           "az_codes_weight_grad",           "az_codes_weight_grad_workspace", "az_logits_policy", "az_logits_policy_workspace",
           "az_rms_norm", "az_rms_norm_grad", "az_rms_norm_grad_workspace", "az_nibbles_quantize", "az_nibbles_dequantize",
           "az_nibbles_matmul", "az_nibbles_matmul_workspace", "az_codes_nibbles_matmul", "az_codes_nibbles_matmul_workspace",
           "az_logits_sample",
           "az_status_string", "az_last_error")


class az_layer_spec(ctypes.Structure):
    _fields_ = [("abi_version", ctypes.c_int32), ("in_planes", ctypes.c_int32),
                ("blocks", ctypes.c_int32), ("filters", ctypes.c_int32),
                ("policy_planes", ctypes.c_int32), ("value_hidden", ctypes.c_int32),
                ("value_conv_relu", ctypes.c_int32), ("act_cap", ctypes.c_float),
                ("max_batch", ctypes.c_int32),
                # abi_version 2
                ("pool_every", ctypes.c_int32), ("policy_head", ctypes.c_int32),
                ("token_dim", ctypes.c_int32), ("value_head", ctypes.c_int32),
                ("value_channels", ctypes.c_int32)]


class az_layer_spec_v1(ctypes.Structure):
    """The version-1 layout (the first nine fields), as older callers pass it."""
    _fields_ = az_layer_spec._fields_[:9]


AZ_CODE_BLOCK = 128
AZ_MASK_NONE, AZ_MASK_BYTES, AZ_MASK_BITS = 0, 1, 2


class az_code_matrix(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("rows", ctypes.c_int64),
                ("cols", ctypes.c_int64), ("ld", ctypes.c_int64), ("scale_rows", ctypes.c_int32)]


class az_logits(ctypes.Structure):
    _fields_ = [("logits", ctypes.c_void_p), ("dtype", ctypes.c_int32), ("rows", ctypes.c_int32),
                ("vocab", ctypes.c_int32), ("ld", ctypes.c_int64), ("mask", ctypes.c_void_p),
                ("mask_kind", ctypes.c_int32), ("ld_mask", ctypes.c_int64), ("bias", ctypes.c_void_p),
                ("ld_bias", ctypes.c_int64), ("history", ctypes.c_void_p), ("ld_history", ctypes.c_int64),
                ("max_history", ctypes.c_int32), ("lengths", ctypes.c_void_p), ("penalties", ctypes.c_void_p)]


AZ_FP4_BLOCK = 32


class az_fp4_matrix(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("rows", ctypes.c_int64),
                ("cols", ctypes.c_int64), ("ld", ctypes.c_int64), ("ld_scales", ctypes.c_int64)]


class az_norm(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("x", ctypes.c_void_p), ("dtype", ctypes.c_int32),
                ("eps", ctypes.c_float), ("ld_x", ctypes.c_int64), ("residual", ctypes.c_void_p),
                ("ld_residual", ctypes.c_int64), ("weight", ctypes.c_void_p), ("sum", ctypes.c_void_p),
                ("ld_sum", ctypes.c_int64), ("y", ctypes.c_void_p), ("ld_y", ctypes.c_int64),
                ("q", ctypes.c_void_p)]  # address of an az_code_matrix


class az_norm_grad(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int64), ("cols", ctypes.c_int64), ("dy", ctypes.c_void_p), ("dtype", ctypes.c_int32),
                ("eps", ctypes.c_float), ("ld_dy", ctypes.c_int64), ("h", ctypes.c_void_p), ("ld_h", ctypes.c_int64),
                ("weight", ctypes.c_void_p), ("dsum", ctypes.c_void_p), ("ld_dsum", ctypes.c_int64),
                ("dx", ctypes.c_void_p), ("ld_dx", ctypes.c_int64), ("dweight", ctypes.c_void_p),
                ("accumulate", ctypes.c_int32)]


class az_sampling(ctypes.Structure):
    _fields_ = [("logits", ctypes.c_void_p), ("dtype", ctypes.c_int32), ("rows", ctypes.c_int32),
                ("vocab", ctypes.c_int32), ("ld", ctypes.c_int64), ("u", ctypes.c_void_p),
                ("temperature", ctypes.c_void_p), ("top_k", ctypes.c_void_p), ("top_p", ctypes.c_void_p),
                ("min_p", ctypes.c_void_p)]


class AzError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str):
        super().__init__(f"{where}: status {status} ({detail})")
        self.status = status


_lib = None


def lib():
    """The loaded library (CDLL); raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError(f"{LIB_PATH} is missing: build it with "
                              "`python -m paper_2609_37447_amd.build`")
        # torch ships its own HIP runtime under the same soname as ROCm's
        # (libamdhip64.so.7).  Loading torch first makes this library bind to
        # that one copy; loaded the other way round, torch would bring up a
        # second runtime beside it and find no GPU.
        import torch  # noqa: F401
        L = ctypes.CDLL(LIB_PATH)
        P, I32, SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
        FP = ctypes.POINTER(ctypes.c_float)
        L.az_weight_count.argtypes, L.az_weight_count.restype = [ctypes.POINTER(az_layer_spec)], SZ
        L.az_net_load.argtypes = [ctypes.POINTER(az_layer_spec), FP, SZ, I32, FP, SZ, FP, SZ,
                                  ctypes.POINTER(P)]
        L.az_net_load.restype = ctypes.c_int
        L.az_eval_batch.argtypes = [P, P, P, I32, P, P, P]
        L.az_eval_batch.restype = ctypes.c_int
        L.az_eval_batch_wdl.argtypes = [P, P, P, I32, P, P, P, P]
        L.az_eval_batch_wdl.restype = ctypes.c_int
        L.az_net_moves.argtypes, L.az_net_moves.restype = [P], ctypes.c_int
        L.az_net_set_tiling.argtypes, L.az_net_set_tiling.restype = [P, I32], ctypes.c_int
        L.az_net_tiling_for.argtypes, L.az_net_tiling_for.restype = [P, I32], ctypes.c_int
        L.az_net_device_bytes.argtypes, L.az_net_device_bytes.restype = [P], SZ
        L.az_net_free.argtypes, L.az_net_free.restype = [P], None
        L.az_compare_outputs.argtypes = [P, P, P, P, P, I32, I32, P, P]
        L.az_compare_outputs.restype = ctypes.c_int
        L.az_pipeline_create.argtypes = [P, I32, I32, I32, I32, ctypes.POINTER(P)]
        L.az_pipeline_create.restype = ctypes.c_int
        L.az_pipeline_slot.argtypes = [P, I32, ctypes.POINTER(P), ctypes.POINTER(P), ctypes.POINTER(P),
                                       ctypes.POINTER(P), ctypes.POINTER(P)]
        L.az_pipeline_slot.restype = ctypes.c_int
        L.az_pipeline_submit.argtypes, L.az_pipeline_submit.restype = [P, I32, I32], ctypes.c_int
        L.az_pipeline_query.argtypes, L.az_pipeline_query.restype = [P, I32], ctypes.c_int
        L.az_pipeline_wait.argtypes, L.az_pipeline_wait.restype = [P, I32], ctypes.c_int
        L.az_pipeline_free.argtypes, L.az_pipeline_free.restype = [P], None
        L.az_pipeline_drive.argtypes = [P, I32, I32, I32, I32, I32, ctypes.POINTER(ctypes.c_double)]
        L.az_pipeline_drive.restype = ctypes.c_int
        L.az_eval_batch_compact_noalloc.argtypes = [P, P, P, I32, I32, P, P, P, P]
        L.az_eval_batch_compact_noalloc.restype = ctypes.c_int
        M, I64 = ctypes.POINTER(az_code_matrix), ctypes.c_int64
        L.az_codes_quantize.argtypes = [P, I32, I64, M, M, P]
        L.az_codes_dequantize.argtypes = [M, P, I32, I64, P]
        L.az_codes_matmul.argtypes = [M, M, P, P, I32, I64, P, SZ, P]
        L.az_codes_matmul_workspace.argtypes, L.az_codes_matmul_workspace.restype = [M, M, I32], SZ
        L.az_codes_weight_grad.argtypes = [P, I64, I32, M, P, I32, I64, P, I32, P, SZ, P]
        L.az_logits_policy.argtypes = [ctypes.POINTER(az_logits), I32, P, I64, P, SZ, P]
        for f in (L.az_codes_quantize, L.az_codes_dequantize, L.az_codes_matmul, L.az_codes_weight_grad,
                  L.az_logits_policy):
            f.restype = ctypes.c_int
        L.az_codes_weight_grad_workspace.argtypes, L.az_codes_weight_grad_workspace.restype = [I64, I32, I64], SZ
        L.az_logits_policy_workspace.argtypes, L.az_logits_policy_workspace.restype = [I32, I32], SZ
        N4 = ctypes.POINTER(az_fp4_matrix)
        L.az_rms_norm.argtypes = [ctypes.POINTER(az_norm), P]
        L.az_rms_norm_grad.argtypes = [ctypes.POINTER(az_norm_grad), P, SZ, P]
        L.az_nibbles_quantize.argtypes = [P, I32, I64, N4, N4, P]
        L.az_nibbles_dequantize.argtypes = [N4, P, I32, I64, P]
        L.az_nibbles_matmul.argtypes = [N4, N4, P, P, I32, I64, P, SZ, P]
        L.az_codes_nibbles_matmul.argtypes = [M, N4, P, P, I32, I64, P, SZ, P]
        L.az_logits_sample.argtypes = [ctypes.POINTER(az_sampling), P, P, P]
        for f in (L.az_rms_norm, L.az_rms_norm_grad, L.az_nibbles_quantize, L.az_nibbles_dequantize, L.az_nibbles_matmul,
                  L.az_codes_nibbles_matmul, L.az_logits_sample):
            f.restype = ctypes.c_int
        L.az_rms_norm_grad_workspace.argtypes, L.az_rms_norm_grad_workspace.restype = [I64, I64], SZ
        L.az_nibbles_matmul_workspace.argtypes, L.az_nibbles_matmul_workspace.restype = [N4, N4, I32], SZ
        L.az_codes_nibbles_matmul_workspace.argtypes, L.az_codes_nibbles_matmul_workspace.restype = [M, N4, I32], SZ
        L.az_debug_fail_allocation.argtypes, L.az_debug_fail_allocation.restype = [I32], None
        L.az_debug_live_allocations.argtypes, L.az_debug_live_allocations.restype = [], ctypes.c_int64
        L.az_status_string.argtypes, L.az_status_string.restype = [ctypes.c_int], ctypes.c_char_p
        L.az_last_error.argtypes, L.az_last_error.restype = [], ctypes.c_char_p
        _lib = L
    return _lib


def make_spec(in_planes, blocks, filters, policy_planes, value_hidden, value_conv_relu=0,
              act_cap=0.0, max_batch=1, abi_version=AZ_ABI_VERSION, pool_every=0,
              policy_head=AZ_POLICY_PLANES, token_dim=0, value_head=AZ_VALUE_TANH,
              value_channels=1) -> az_layer_spec:
    return az_layer_spec(abi_version, in_planes, blocks, filters, policy_planes, value_hidden,
                         value_conv_relu, act_cap, max_batch, pool_every, policy_head, token_dim,
                         value_head, value_channels)


def spec_from_shape(shape, max_batch: int) -> az_layer_spec:
    """az_layer_spec from any object with the NetShape attribute names."""
    fromto = getattr(shape, "policy_head", "planes") == "fromto"
    wdl = getattr(shape, "value_head", "tanh") == "wdl"
    return make_spec(shape.in_planes, shape.blocks, shape.filters, shape.policy_planes,
                     shape.value_hidden, shape.value_conv_relu, shape.act_cap, max_batch,
                     pool_every=getattr(shape, "pool_every", 0),
                     policy_head=AZ_POLICY_FROMTO if fromto else AZ_POLICY_PLANES,
                     token_dim=shape.token_dim if fromto else 0,
                     value_head=AZ_VALUE_WDL if wdl else AZ_VALUE_TANH,
                     value_channels=getattr(shape, "value_channels", 1))


def _check(status: int, where: str) -> int:
    if status < 0:
        detail = lib().az_last_error().decode(errors="replace")
        raise AzError(status, where, detail or az_status_string(status))
    return status


def _fptr(a):
    if a is None:
        return None, 0
    a = np.ascontiguousarray(a, dtype=np.float32)
    return a, a.size


def az_weight_count(spec: az_layer_spec) -> int:
    return int(lib().az_weight_count(ctypes.byref(spec)))


def az_net_load(spec: az_layer_spec, weights, dtype, w_scales=None, act_scales=None,
                raise_on_error: bool = True):
    """Returns the handle (int), or (status) when raise_on_error is False and it fails."""
    dt = DTYPES[dtype] if isinstance(dtype, str) else int(dtype)
    w, nw = _fptr(weights)
    ws, nws = _fptr(w_scales)
    acs, nacs = _fptr(act_scales)
    FP = ctypes.POINTER(ctypes.c_float)
    cast = lambda a: a.ctypes.data_as(FP) if a is not None else None  # noqa: E731
    out = ctypes.c_void_p()
    st = lib().az_net_load(ctypes.byref(spec), cast(w), nw, dt, cast(ws), nws, cast(acs), nacs,
                           ctypes.byref(out))
    if not raise_on_error:
        return (st, out.value) if st == AZ_OK else (st, None)
    _check(st, "az_net_load")
    return out.value


def az_eval_batch(net, planes_ptr: int, legal_ptr: int, B: int, policy_ptr: int, value_ptr: int,
                  stream: int = 0, raise_on_error: bool = True) -> int:
    st = lib().az_eval_batch(net, planes_ptr, legal_ptr, int(B), policy_ptr, value_ptr, stream)
    return _check(st, "az_eval_batch") if raise_on_error else st


def az_eval_batch_wdl(net, planes_ptr: int, legal_ptr: int, B: int, policy_ptr: int, value_ptr: int,
                      wdl_ptr, stream: int = 0, raise_on_error: bool = True) -> int:
    st = lib().az_eval_batch_wdl(net, planes_ptr, legal_ptr, int(B), policy_ptr, value_ptr, wdl_ptr, stream)
    return _check(st, "az_eval_batch_wdl") if raise_on_error else st


def az_net_moves(net) -> int:
    return _check(lib().az_net_moves(net), "az_net_moves")


def az_net_set_tiling(net, tiling: int, raise_on_error: bool = True) -> int:
    st = lib().az_net_set_tiling(net, int(tiling))
    return _check(st, "az_net_set_tiling") if raise_on_error else st


def az_net_tiling_for(net, B: int) -> int:
    return _check(lib().az_net_tiling_for(net, int(B)), "az_net_tiling_for")


def az_net_device_bytes(net) -> int:
    return int(lib().az_net_device_bytes(net))


def az_net_free(net) -> None:
    lib().az_net_free(net)


def az_debug_fail_allocation(n: int) -> None:
    lib().az_debug_fail_allocation(int(n))


def az_debug_live_allocations() -> int:
    return int(lib().az_debug_live_allocations())


def az_status_string(status: int) -> str:
    return lib().az_status_string(int(status)).decode()


def az_last_error() -> str:
    return lib().az_last_error().decode(errors="replace")


# --------------------------------------------------------------------------- #
# torch convenience: device tensors and streams (PyTorch provides memory and
# streams only)
# --------------------------------------------------------------------------- #
def eval_tensors(net, planes, legal, policy, value, stream=None, wdl=None) -> int:
    """az_eval_batch (az_eval_batch_wdl when wdl is given) on torch CUDA tensors;
    stream defaults to torch's current one."""
    import torch
    B = planes.shape[0]
    named = [("planes", planes), ("legal", legal), ("policy", policy), ("value", value)]
    if wdl is not None:
        named.append(("wdl", wdl))
    for name, t in named:
        if not t.is_cuda or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous device tensor")
    if planes.dtype != torch.float32 or legal.dtype != torch.uint8:
        raise ValueError("planes must be float32 and legal uint8")
    if policy.dtype != torch.float32 or value.dtype != torch.float32:
        raise ValueError("policy and value must be float32")
    if legal.shape[0] != B or policy.shape[0] != B or value.shape[0] != B:
        raise ValueError("batch sizes differ")
    s = torch.cuda.current_stream() if stream is None else stream
    if wdl is not None:
        if wdl.dtype != torch.float32 or tuple(wdl.shape) != (B, 3):
            raise ValueError("wdl must be float32 [B, 3]")
        return az_eval_batch_wdl(net, planes.data_ptr(), legal.data_ptr(), B, policy.data_ptr(),
                                 value.data_ptr(), wdl.data_ptr(), s.cuda_stream)
    return az_eval_batch(net, planes.data_ptr(), legal.data_ptr(), B, policy.data_ptr(),
                         value.data_ptr(), s.cuda_stream)


def az_compare_outputs(policy_ref, value_ref, policy_test, value_test, legal, B: int, n_moves: int,
                       row_metrics, stream) -> int:
    """Device pointers (ints); per-row {top-1 equal, KL(ref || test), |dV|} into row_metrics."""
    return _check(lib().az_compare_outputs(policy_ref, value_ref, policy_test, value_test, legal, B,
                                           n_moves, row_metrics, stream), "az_compare_outputs")


def validate(net_test, net_ref, planes, legal, min_top1: float = 0.8, max_kl: float = 0.1,
             max_dv: float = 0.25, stream=None) -> dict:
    """Deployment validation of a loaded network against a reference network on the
    same positions (torch device tensors planes [B][C][8][8] f32 and legal [B][P*64]
    u8): both are evaluated, the library compares them row by row, and the rows are
    summarised as the mean top-1 legal-move agreement (over rows with a legal move),
    the mean legal-policy KL(ref || test) and the largest value error.  The default
    bounds separate a faithful quantised network from a broken engine (the paper's
    faulty refit showed KL near 1); callers set their own."""
    import torch
    B, NM = legal.shape
    dev = planes.device
    out = {}
    for key, net in (("test", net_test), ("ref", net_ref)):
        pol = torch.empty((B, NM), device=dev)
        val = torch.empty((B,), device=dev)
        eval_tensors(net, planes, legal, pol, val, stream)
        out[key] = (pol, val)
    rows = torch.empty((B, 3), device=dev)
    s = torch.cuda.current_stream() if stream is None else stream
    az_compare_outputs(out["ref"][0].data_ptr(), out["ref"][1].data_ptr(), out["test"][0].data_ptr(),
                       out["test"][1].data_ptr(), legal.data_ptr(), B, NM, rows.data_ptr(), s.cuda_stream)
    s.synchronize()
    r = rows.cpu().numpy().astype(np.float64)
    has = (legal != 0).any(dim=1).cpu().numpy().astype(bool)
    top1 = float(r[has, 0].mean()) if has.any() else 1.0
    kl = float(r[:, 1].mean())
    dv = float(r[:, 2].max())
    return {"top1": top1, "kl": kl, "dv_max": dv, "rows": r,
            "passed": top1 >= min_top1 and kl <= max_kl and dv <= max_dv}


# --------------------------------------------------------------------------- #
# Coded matrices and the policy from logits, on torch device tensors
# --------------------------------------------------------------------------- #
def az_codes_quantize(x, dtype: int, ldx: int, q: az_code_matrix, qt=None, stream: int = 0,
                      raise_on_error: bool = True) -> int:
    st = lib().az_codes_quantize(x, dtype, ldx, q, qt, stream)
    return _check(st, "az_codes_quantize") if raise_on_error else st


def az_codes_dequantize(q: az_code_matrix, x, dtype: int, ldx: int, stream: int = 0, raise_on_error: bool = True) -> int:
    st = lib().az_codes_dequantize(q, x, dtype, ldx, stream)
    return _check(st, "az_codes_dequantize") if raise_on_error else st


def az_codes_matmul_workspace(a: az_code_matrix, b: az_code_matrix, dtype: int) -> int:
    return int(lib().az_codes_matmul_workspace(a, b, dtype))


def az_codes_matmul(a: az_code_matrix, b: az_code_matrix, bias, out, dtype: int, ld_out: int, workspace=None,
                    workspace_bytes: int = 0, stream: int = 0, raise_on_error: bool = True) -> int:
    st = lib().az_codes_matmul(a, b, bias, out, dtype, ld_out, workspace, workspace_bytes, stream)
    return _check(st, "az_codes_matmul") if raise_on_error else st


def az_codes_weight_grad_workspace(rows: int, n: int, cols: int) -> int:
    return int(lib().az_codes_weight_grad_workspace(rows, n, cols))


def az_codes_weight_grad(dy, ld_dy: int, n: int, x: az_code_matrix, dw, dtype: int, ld_dw: int, db=None,
                         accumulate: bool = False, workspace=None, workspace_bytes: int = 0, stream: int = 0,
                         raise_on_error: bool = True) -> int:
    st = lib().az_codes_weight_grad(dy, ld_dy, n, x, dw, dtype, ld_dw, db, int(accumulate), workspace,
                                    workspace_bytes, stream)
    return _check(st, "az_codes_weight_grad") if raise_on_error else st


def az_logits_policy_workspace(rows: int, vocab: int) -> int:
    return int(lib().az_logits_policy_workspace(rows, vocab))


def az_logits_policy(logits: az_logits, probabilities: bool, out, ld_out: int, workspace=None, workspace_bytes: int = 0,
                     stream: int = 0, raise_on_error: bool = True) -> int:
    st = lib().az_logits_policy(logits, int(probabilities), out, ld_out, workspace, workspace_bytes, stream)
    return _check(st, "az_logits_policy") if raise_on_error else st


def az_rms_norm(norm: az_norm, stream: int = 0, raise_on_error: bool = True) -> int:
    st = lib().az_rms_norm(norm, stream)
    return _check(st, "az_rms_norm") if raise_on_error else st


def az_rms_norm_grad_workspace(rows: int, cols: int) -> int:
    return int(lib().az_rms_norm_grad_workspace(rows, cols))


def az_rms_norm_grad(grad: az_norm_grad, workspace=None, workspace_bytes: int = 0, stream: int = 0,
                     raise_on_error: bool = True) -> int:
    st = lib().az_rms_norm_grad(grad, workspace, workspace_bytes, stream)
    return _check(st, "az_rms_norm_grad") if raise_on_error else st


def az_nibbles_quantize(x, dtype: int, ldx: int, q: az_fp4_matrix, qt=None, stream: int = 0,
                        raise_on_error: bool = True) -> int:
    st = lib().az_nibbles_quantize(x, dtype, ldx, q, qt, stream)
    return _check(st, "az_nibbles_quantize") if raise_on_error else st


def az_nibbles_dequantize(q: az_fp4_matrix, x, dtype: int, ldx: int, stream: int = 0, raise_on_error: bool = True) -> int:
    st = lib().az_nibbles_dequantize(q, x, dtype, ldx, stream)
    return _check(st, "az_nibbles_dequantize") if raise_on_error else st


def az_nibbles_matmul_workspace(a: az_fp4_matrix, b: az_fp4_matrix, dtype: int) -> int:
    return int(lib().az_nibbles_matmul_workspace(a, b, dtype))


def az_nibbles_matmul(a: az_fp4_matrix, b: az_fp4_matrix, bias, out, dtype: int, ld_out: int, workspace=None,
                      workspace_bytes: int = 0, stream: int = 0, raise_on_error: bool = True) -> int:
    st = lib().az_nibbles_matmul(a, b, bias, out, dtype, ld_out, workspace, workspace_bytes, stream)
    return _check(st, "az_nibbles_matmul") if raise_on_error else st


def az_codes_nibbles_matmul_workspace(a: az_code_matrix, b: az_fp4_matrix, dtype: int) -> int:
    return int(lib().az_codes_nibbles_matmul_workspace(a, b, dtype))


def az_codes_nibbles_matmul(a: az_code_matrix, b: az_fp4_matrix, bias, out, dtype: int, ld_out: int, workspace=None,
                            workspace_bytes: int = 0, stream: int = 0, raise_on_error: bool = True) -> int:
    st = lib().az_codes_nibbles_matmul(a, b, bias, out, dtype, ld_out, workspace, workspace_bytes, stream)
    return _check(st, "az_codes_nibbles_matmul") if raise_on_error else st


def az_logits_sample(sampling: az_sampling, out, prob=None, stream: int = 0, raise_on_error: bool = True) -> int:
    st = lib().az_logits_sample(sampling, out, prob, stream)
    return _check(st, "az_logits_sample") if raise_on_error else st


def _rows_of(name, t, dtypes):
    """(rows, columns, elements from row to row) of a two-dimensional device tensor."""
    if not t.is_cuda or t.dtype not in dtypes or t.dim() != 2:
        raise ValueError(f"{name} must be a two-dimensional device tensor of {' or '.join(map(str, dtypes))}")
    rows, cols = t.shape
    step, inner = t.stride()
    if cols > 1 and inner != 1 or rows > 1 and step < cols:
        raise ValueError(f"{name} must hold its rows one behind the other, each without gaps")
    return rows, cols, step if rows > 1 else max(step, cols)


def _vector_of(name, t, dtype, n):
    if not t.is_cuda or t.dtype != dtype or t.dim() != 1 or t.shape[0] != n or n > 1 and t.stride(0) != 1:
        raise ValueError(f"{name} must be a contiguous device tensor of {dtype} [{n}]")


class CodeMatrix:
    """A matrix of e4m3 codes with a power-of-two scale for each block of 128 columns of a
    row (scale_rows 1) or of 128 x 128 entries (scale_rows 128), on torch device tensors:
    codes uint8 [rows][columns or more], rows a multiple of 16 bytes apart, and scales uint8
    [ceil(rows / scale_rows)][ceil(cols / 128)].  Keeps its tensors alive."""

    __slots__ = ("codes", "scales", "rows", "cols", "scale_rows", "device", "c")

    def __init__(self, codes, scales, cols=None, scale_rows: int = 1):
        torch = _modules["torch"]
        rows, width, ld = _rows_of("codes", codes, (torch.uint8,))
        cols = width if cols is None else int(cols)
        if not 0 < cols <= width:
            raise ValueError(f"cols {cols} is not in 1..{width}")
        if scale_rows not in (1, AZ_CODE_BLOCK):
            raise ValueError("scale_rows is 1 or 128")
        if rows <= 1:
            ld = -(-ld // 16) * 16
        if rows and width < -(-cols // 16) * 16 and codes.untyped_storage().nbytes() - codes.storage_offset() < (rows - 1) * ld + -(-cols // 16) * 16:
            raise ValueError("codes must hold whole chunks of 16 bytes in every row")
        want = (-(-rows // scale_rows), -(-cols // AZ_CODE_BLOCK))
        if not scales.is_cuda or scales.dtype != torch.uint8 or tuple(scales.shape) != want or not scales.is_contiguous():
            raise ValueError(f"scales must be a contiguous uint8 device tensor {list(want)}")
        if scales.device != codes.device:
            raise ValueError("codes and scales are on different devices")
        self.codes, self.scales, self.rows, self.cols = codes, scales, rows, cols
        self.scale_rows, self.device = scale_rows, codes.device
        self.c = az_code_matrix(codes.data_ptr(), scales.data_ptr(), rows, cols, ld, scale_rows)

    @classmethod
    def empty(cls, rows: int, cols: int, scale_rows: int = 1, device="cuda"):
        """A matrix of these sizes on memory of its own, codes and scales not yet written."""
        import torch
        codes = torch.empty((rows, -(-cols // 16) * 16), dtype=torch.uint8, device=device)
        scales = torch.empty((-(-rows // scale_rows), -(-cols // AZ_CODE_BLOCK)), dtype=torch.uint8, device=device)
        return cls(codes, scales, cols, scale_rows)


class Fp4Matrix:
    """A matrix of 4-bit e2m1 codes, two to a byte, with a power-of-two scale for each block of 32 columns of a row, on
    torch device tensors: codes uint8 [rows][bytes], rows a multiple of 16 bytes apart and cols / 2 or
    more of them, and scales uint8 [rows][ceil(cols / 32) or more], rows a multiple of 4 bytes apart.
    Keeps its tensors alive."""

    __slots__ = ("codes", "scales", "rows", "cols", "device", "c")

    def __init__(self, codes, scales, cols=None):
        torch = _modules["torch"]
        rows, width, ld = _rows_of("codes", codes, (torch.uint8,))
        srows, swidth, lds = _rows_of("scales", scales, (torch.uint8,))
        cols = 2 * width if cols is None else int(cols)
        if not 0 < cols <= 2 * width:
            raise ValueError(f"cols {cols} is not in 1..{2 * width}")
        blocks = -(-cols // AZ_FP4_BLOCK)
        if srows != rows or swidth < blocks:
            raise ValueError(f"scales {[srows, swidth]} are not [{rows}, {blocks} or more]")
        if rows <= 1:
            ld, lds = -(-ld // 16) * 16, -(-lds // 4) * 4
        if rows and width < 16 * blocks and codes.untyped_storage().nbytes() - codes.storage_offset() < (rows - 1) * ld + 16 * blocks:
            raise ValueError("codes must hold whole chunks of 16 bytes in every row")
        if rows and swidth % 4 and scales.untyped_storage().nbytes() - scales.storage_offset() < (rows - 1) * lds + -(-blocks // 4) * 4:
            raise ValueError("scales must hold whole words of 4 bytes in every row")
        if scales.device != codes.device:
            raise ValueError("codes and scales are on different devices")
        self.codes, self.scales, self.rows, self.cols, self.device = codes, scales, rows, cols, codes.device
        self.c = az_fp4_matrix(codes.data_ptr(), scales.data_ptr(), rows, cols, ld, lds)

    @classmethod
    def empty(cls, rows: int, cols: int, device="cuda"):
        """A matrix of these sizes on memory of its own, codes and scales not yet written."""
        import torch
        codes = torch.empty((rows, -(-cols // 32) * 16), dtype=torch.uint8, device=device)
        scales = torch.empty((rows, -(-cols // (4 * AZ_FP4_BLOCK)) * 4), dtype=torch.uint8, device=device)
        return cls(codes, scales, cols)


def _on(device, stream, *others):
    """The call's stream as the library takes it (torch's current one by default), for operands that are all
    on `device`."""
    torch = _modules["torch"]
    for t in others:
        if t is not None and t.device != device:
            raise ValueError("the operands are on different devices")
    if stream is not None and stream.device != device:
        raise ValueError("the stream is another device's")
    return torch._C._cuda_getCurrentRawStream(device.index) if stream is None else stream.cuda_stream


def _call(device, fn, *args) -> int:
    """fn(*args) with `device` as the current one."""
    torch = _modules["torch"]
    if device.index == torch._C._cuda_getDevice():  # (tensors are on the device: CUDA has been initialised)
        return fn(*args)
    with torch.cuda.device(device):
        return fn(*args)


def _workspace(given, need, device, stream):
    """(pointer, bytes) of a call's workspace; made for the call on its stream where none is given."""
    if given is not None:
        if not given.is_cuda or not given.is_contiguous() or given.device != device:
            raise ValueError("workspace must be a contiguous tensor on the operands' device")
        return given.data_ptr(), given.numel() * given.element_size(), given
    if need == 0:
        return None, 0, None
    torch = _modules["torch"]
    if stream is None:
        t = torch.empty((need,), dtype=torch.uint8, device=device)
    else:
        with torch.cuda.stream(stream):
            t = torch.empty((need,), dtype=torch.uint8, device=device)
    return t.data_ptr(), need, t


def _float_type(t) -> int:
    torch = _modules["torch"]
    return AZ_BF16 if t.dtype == torch.bfloat16 else AZ_F32


def quantize_tensors(x, q, transposed=None, stream=None) -> int:
    """az_codes_quantize of x (float32 or bfloat16 [rows][cols]) into the CodeMatrix q and, for matrices with
    scale_rows 128, its transposed copy, or az_nibbles_quantize into the Fp4Matrix q and the transposed
    one; stream defaults to torch's current one."""
    torch = _modules["torch"]
    rows, cols, ld = _rows_of("x", x, (torch.float32, torch.bfloat16))
    if (rows, cols) != (q.rows, q.cols):
        raise ValueError(f"x is {[rows, cols]}, the coded matrix {[q.rows, q.cols]}")
    if transposed is not None and type(transposed) is not type(q):
        raise ValueError("the transposed matrix is of another kind")
    s = _on(x.device, stream, q, transposed)
    return _call(x.device, az_nibbles_quantize if type(q) is Fp4Matrix else az_codes_quantize, x.data_ptr(), _float_type(x), ld, q.c,
                 transposed.c if transposed is not None else None, s)


def dequantize_tensors(q, x, stream=None) -> int:
    """az_codes_dequantize (az_nibbles_dequantize) of the CodeMatrix (Fp4Matrix) q into x (float32 or bfloat16
    [rows][cols])."""
    torch = _modules["torch"]
    rows, cols, ld = _rows_of("x", x, (torch.float32, torch.bfloat16))
    if (rows, cols) != (q.rows, q.cols):
        raise ValueError(f"x is {[rows, cols]}, the coded matrix {[q.rows, q.cols]}")
    s = _on(x.device, stream, q)
    return _call(x.device, az_nibbles_dequantize if type(q) is Fp4Matrix else az_codes_dequantize, q.c, x.data_ptr(), _float_type(x), ld, s)


def matmul_tensors(a, b, out, bias=None, workspace=None, stream=None) -> int:
    """out [a.rows][b.rows] (bfloat16 or float32) = a b^T + bias (float32 [b.rows]): az_codes_matmul of two CodeMatrix,
    az_nibbles_matmul of two Fp4Matrix, az_codes_nibbles_matmul of a CodeMatrix and an Fp4Matrix b.
    A workspace is made for the call (torch's allocator, on the call's stream) unless a tensor is
    given."""
    torch = _modules["torch"]
    m, n, ld = _rows_of("out", out, (torch.float32, torch.bfloat16))
    if (m, n) != (a.rows, b.rows):
        raise ValueError(f"out is {[m, n]}, the product {[a.rows, b.rows]}")
    if bias is not None:
        _vector_of("bias", bias, torch.float32, n)
    if type(b) is not Fp4Matrix:
        if type(a) is Fp4Matrix:
            raise ValueError("a 4-bit matrix is multiplied by a 4-bit one")
        size_of, multiply = az_codes_matmul_workspace, az_codes_matmul
    elif type(a) is Fp4Matrix:
        size_of, multiply = az_nibbles_matmul_workspace, az_nibbles_matmul
    else:
        size_of, multiply = az_codes_nibbles_matmul_workspace, az_codes_nibbles_matmul
    s, dt = _on(out.device, stream, a, b, bias), _float_type(out)
    ws, size, keep = _workspace(workspace, size_of(a.c, b.c, dt), out.device, stream)
    return _call(out.device, multiply, a.c, b.c, bias.data_ptr() if bias is not None else None, out.data_ptr(), dt,
                 ld, ws, size, s)


def weight_grad_tensors(dy, x: CodeMatrix, dw, db=None, accumulate: bool = False, workspace=None, stream=None) -> int:
    """az_codes_weight_grad: dw [n][x.cols] (float32 or bfloat16) and db (float32 [n]) from dy
    (bfloat16 [x.rows][n]) and the layer's saved input x.  A workspace is made for the call
    (torch's allocator, on the call's stream) unless a tensor is given."""
    torch = _modules["torch"]
    m, n, ldy = _rows_of("dy", dy, (torch.bfloat16,))
    if m != x.rows:
        raise ValueError(f"dy has {m} rows, x {x.rows}")
    wn, wk, ldw = _rows_of("dw", dw, (torch.float32, torch.bfloat16))
    if (wn, wk) != (n, x.cols):
        raise ValueError(f"dw is {[wn, wk]}, the gradient {[n, x.cols]}")
    if db is not None:
        _vector_of("db", db, torch.float32, n)
    s = _on(dw.device, stream, dy, x, db)
    ws, size, keep = _workspace(workspace, az_codes_weight_grad_workspace(m, n, x.cols), dw.device, stream)
    return _call(dw.device, az_codes_weight_grad, dy.data_ptr(), ldy, n, x.c, dw.data_ptr(), _float_type(dw), ldw,
                 db.data_ptr() if db is not None else None, accumulate, ws, size, s)


def policy_tensors(logits, out, mask=None, bias=None, history=None, lengths=None, penalties=None,
                   probabilities: bool = True, workspace=None, stream=None) -> int:
    """az_logits_policy of logits (float32 or bfloat16 [rows][vocab]) into out (float32): the policy over
    what the mask allows, or the adjusted logits.  mask: uint8 or bool [rows][vocab] (nonzero =
    allowed) or int32 [rows][ceil(vocab / 32)] of bits; bias: float32 [vocab], [1][vocab] or
    [rows][vocab]; history: int32 [rows][entries] with lengths int32 [rows] (default: all) and penalties
    float32 [rows][3] (repetition, frequency, presence)."""
    torch = _modules["torch"]
    b, v, ld = _rows_of("logits", logits, (torch.float32, torch.bfloat16))
    ob, ov, ldo = _rows_of("out", out, (torch.float32,))
    if (ob, ov) != (b, v):
        raise ValueError(f"out is {[ob, ov]}, the logits {[b, v]}")
    kind, ldm = AZ_MASK_NONE, 0
    if mask is not None:
        mb, mv, ldm = _rows_of("mask", mask, (torch.uint8, torch.bool, torch.int32))
        kind = AZ_MASK_BITS if mask.dtype == torch.int32 else AZ_MASK_BYTES
        if (mb, mv) != (b, -(-v // 32) if kind == AZ_MASK_BITS else v):
            raise ValueError(f"mask {[mb, mv]} does not fit logits {[b, v]}")
    ldb = 0
    if bias is not None:
        if bias.dim() == 1:
            bias = bias.unsqueeze(0)
        bb, bv, ldb = _rows_of("bias", bias, (torch.float32,))
        if bv != v or bb not in (1, b):
            raise ValueError(f"bias {[bb, bv]} does not fit logits {[b, v]}")
        ldb = ldb if bb == b and b > 1 else 0
    t, ldh = 0, 0
    if history is not None:
        hb, t, ldh = _rows_of("history", history, (torch.int32,))
        if hb != b:
            raise ValueError(f"history has {hb} rows, the logits {b}")
        if penalties is None:
            raise ValueError("a history needs penalties")
        if not penalties.is_cuda or penalties.dtype != torch.float32 or tuple(penalties.shape) != (b, 3) or not penalties.is_contiguous():
            raise ValueError(f"penalties must be a contiguous float32 device tensor [{b}, 3]")
        if lengths is not None:
            _vector_of("lengths", lengths, torch.int32, b)
    elif lengths is not None or penalties is not None:
        raise ValueError("lengths and penalties come with a history")
    s = _on(logits.device, stream, out, mask, bias, history, lengths, penalties)
    need = az_logits_policy_workspace(b, v) if probabilities else 0
    ws, size, keep = _workspace(workspace, need, logits.device, stream)
    p = lambda x: x.data_ptr() if x is not None else None  # noqa: E731
    rows = az_logits(p(logits), _float_type(logits), b, v, ld, p(mask), kind, ldm, p(bias), ldb, p(history), ldh, t,
                     p(lengths), p(penalties))
    return _call(logits.device, az_logits_policy, rows, probabilities, out.data_ptr(), ldo, ws, size, s)


def _like(name, t, like, rows, cols, ld):
    """(pointer, elements from row to row) of an optional matrix of the type and sizes of another, whose rows are ld apart."""
    if t is None:
        return None, 0
    if t.dtype != like.dtype or t.shape != like.shape or t.stride() != like.stride() or not t.is_cuda:
        r, c, ld = _rows_of(name, t, (like.dtype,))
        if (r, c) != (rows, cols):
            raise ValueError(f"{name} is {[r, c]}, not {[rows, cols]}")
    return t.data_ptr(), ld


def norm_tensors(x, y=None, q: CodeMatrix = None, residual=None, sum=None, weight=None, eps: float = 1e-6, stream=None) -> int:
    """az_rms_norm of x (float32 or bfloat16 [rows][cols]) plus residual, with weight (float32 [cols]), into y and the
    coded matrix q; sum receives x + residual (it may be either's own tensor).  residual, sum and y are like x."""
    torch = _modules["torch"]
    rows, cols, ld = _rows_of("x", x, (torch.float32, torch.bfloat16))
    pr, ldr = _like("residual", residual, x, rows, cols, ld)
    ps, lds = _like("sum", sum, x, rows, cols, ld)
    py, ldy = _like("y", y, x, rows, cols, ld)
    if weight is not None:
        _vector_of("weight", weight, torch.float32, cols)
    if q is not None and (q.rows, q.cols) != (rows, cols):
        raise ValueError(f"x is {[rows, cols]}, the coded matrix {[q.rows, q.cols]}")
    s = _on(x.device, stream, residual, sum, y, weight, q)
    n = az_norm(rows, cols, x.data_ptr(), _float_type(x), eps, ld, pr, ldr, weight.data_ptr() if weight is not None else None,
                ps, lds, py, ldy, ctypes.addressof(q.c) if q is not None else None)
    return _call(x.device, az_rms_norm, n, s)


def norm_grad_tensors(dy, h, dx=None, dsum=None, weight=None, dw=None, eps: float = 1e-6, accumulate: bool = False,
                      workspace=None, stream=None) -> int:
    """az_rms_norm_grad: dx (the gradient of x and of the residual) and dw (float32 [cols]) from dy and h (float32 or bfloat16
    [rows][cols]), h the sum that the norm gave; dsum: what else reaches h.  dy, dsum and dx are like
    h.  A workspace is made for the call (torch's allocator, on the call's stream) unless a tensor is given."""
    torch = _modules["torch"]
    rows, cols, ld = _rows_of("h", h, (torch.float32, torch.bfloat16))
    pd, ldd = _like("dy", dy, h, rows, cols, ld)
    pr, ldr = _like("dsum", dsum, h, rows, cols, ld)
    px, ldx = _like("dx", dx, h, rows, cols, ld)
    for name, v in (("weight", weight), ("dw", dw)):
        if v is not None:
            _vector_of(name, v, torch.float32, cols)
    s = _on(h.device, stream, dy, dsum, dx, weight, dw)
    need = az_rms_norm_grad_workspace(rows, cols) if dw is not None else 0
    ws, size, keep = _workspace(workspace, need, h.device, stream)
    g = az_norm_grad(rows, cols, pd, _float_type(h), eps, ldd, h.data_ptr(), ld, weight.data_ptr() if weight is not None else None,
                     pr, ldr, px, ldx, dw.data_ptr() if dw is not None else None, accumulate)
    return _call(h.device, az_rms_norm_grad, g, ws, size, s)


def sample_tensors(logits, u, out, prob=None, temperature=None, top_k=None, top_p=None, min_p=None, stream=None) -> int:
    """az_logits_sample: an entry of each row of logits (float32 or bfloat16 [rows][vocab]) into out (int32 [rows]) and its
    probability into prob (float32 [rows]), from random numbers u in [0, 1); u, temperature, top_p and min_p
    float32 [rows], top_k int32 [rows]."""
    torch = _modules["torch"]
    b, v, ld = _rows_of("logits", logits, (torch.float32, torch.bfloat16))
    for name, t, dtype in (("u", u, torch.float32), ("out", out, torch.int32), ("prob", prob, torch.float32),
                           ("temperature", temperature, torch.float32), ("top_k", top_k, torch.int32),
                           ("top_p", top_p, torch.float32), ("min_p", min_p, torch.float32)):
        if t is not None:
            _vector_of(name, t, dtype, b)
    s = _on(logits.device, stream, u, out, prob, temperature, top_k, top_p, min_p)
    p = lambda x: x.data_ptr() if x is not None else None  # noqa: E731
    rows = az_sampling(p(logits), _float_type(logits), b, v, ld, p(u), p(temperature), p(top_k), p(top_p), p(min_p))
    return _call(logits.device, az_logits_sample, rows, p(out), p(prob), s)


AZ_PIPE_GRAPHS = 1
AZ_PIPE_COMPACT_POLICY = 2


def az_pipeline_create(net, max_batch: int, slots: int, flags: int = 0, max_legal: int = 0,
                       raise_on_error: bool = True):
    """Returns the pipeline handle, or (status) when raise_on_error is False and it fails."""
    out = ctypes.c_void_p()
    st = lib().az_pipeline_create(net, max_batch, slots, flags, max_legal, ctypes.byref(out))
    if st != AZ_OK and not raise_on_error:
        return st
    _check(st, "az_pipeline_create")
    return out


def az_pipeline_slot(p, slot: int):
    """Host pointers (planes, legal, policy, value, legal_count) of a slot."""
    ptrs = [ctypes.c_void_p() for _ in range(5)]
    _check(lib().az_pipeline_slot(p, slot, *[ctypes.byref(x) for x in ptrs]), "az_pipeline_slot")
    return tuple(x.value for x in ptrs)


def az_pipeline_submit(p, slot: int, B: int) -> int:
    return _check(lib().az_pipeline_submit(p, slot, B), "az_pipeline_submit")


def az_pipeline_query(p, slot: int) -> int:
    return _check(lib().az_pipeline_query(p, slot), "az_pipeline_query")


def az_pipeline_wait(p, slot: int) -> int:
    return _check(lib().az_pipeline_wait(p, slot), "az_pipeline_wait")


def az_pipeline_drive(p, workers: int, slots_per_worker: int, B: int, warmup: int, batches: int) -> float:
    """Wall seconds of `batches` native round-robin submissions per worker thread."""
    sec = ctypes.c_double()
    _check(lib().az_pipeline_drive(p, workers, slots_per_worker, B, warmup, batches, ctypes.byref(sec)),
           "az_pipeline_drive")
    return sec.value


def az_pipeline_free(p) -> None:
    lib().az_pipeline_free(p)


class Pipeline:
    """A pipeline with numpy views of its slots' pinned host buffers:
    views[k] = (planes, legal, policy, value, legal_count or None)."""

    def __init__(self, net, spec, max_batch: int, slots: int, use_graphs: bool = False,
                 max_legal: int = 0):
        flags = (AZ_PIPE_GRAPHS if use_graphs else 0) | (AZ_PIPE_COMPACT_POLICY if max_legal else 0)
        self.p = az_pipeline_create(net, max_batch, slots, flags, max_legal)
        n_moves = az_net_moves(net)
        f32 = ctypes.POINTER(ctypes.c_float)
        u8 = ctypes.POINTER(ctypes.c_uint8)
        i32 = ctypes.POINTER(ctypes.c_int32)
        self.views = []
        for k in range(slots):
            pp, lp, po, vp, cp = az_pipeline_slot(self.p, k)
            self.views.append((
                np.ctypeslib.as_array(ctypes.cast(pp, f32), (max_batch, spec.in_planes, 8, 8)),
                np.ctypeslib.as_array(ctypes.cast(lp, u8), (max_batch, n_moves)),
                np.ctypeslib.as_array(ctypes.cast(po, f32), (max_batch, max_legal or n_moves)),
                np.ctypeslib.as_array(ctypes.cast(vp, f32), (max_batch,)),
                np.ctypeslib.as_array(ctypes.cast(cp, i32), (max_batch,)) if max_legal else None,
            ))

    def submit(self, slot: int, B: int) -> None:
        az_pipeline_submit(self.p, slot, B)

    def wait(self, slot: int) -> None:
        az_pipeline_wait(self.p, slot)

    def query(self, slot: int) -> bool:
        return az_pipeline_query(self.p, slot) == 0

    def drive(self, workers: int, slots_per_worker: int, B: int, warmup: int, batches: int) -> float:
        return az_pipeline_drive(self.p, workers, slots_per_worker, B, warmup, batches)

    def close(self) -> None:
        if self.p is not None:
            az_pipeline_free(self.p)
            self.p = None
