"""Every kernel of the coded products and of the weight's gradient, in one part and in several, on
numbers whose sums are exact: results are compared for equality.

Entries are whole numbers of at most 3 times 2^-1, 1 or 2 (one of them a block).  A product is a multiple of 1/4
of at most 36, so that K <= 2^16 of them, in whatever order, are exact in fp32 (4 * 36 * K < 2^24); and
the e4m3 instruction, which cuts at 2^(E - 13) with 2^E <= 32 the largest product's binade, cuts nothing.  An
fp32 result is the exact one, a bf16 result its nearest bf16 value.
"""

import json
import os
import re
import tempfile

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _az():
    import torch

    import paper_2609_37447_amd as az
    return az, torch


def _whole(g, rows, cols):
    """Whole numbers in -3..3 times a power of two for each 128 x 128 block, float32 on the device."""
    import torch
    x = torch.randint(-3, 4, (rows, cols), generator=g, device="cuda").float()
    s = torch.exp2(torch.randint(-1, 2, (-(-rows // 128), -(-cols // 128)), generator=g, device="cuda").float())
    x *= s.repeat_interleave(128, dim=0)[:rows].repeat_interleave(128, dim=1)[:, :cols]
    return x


def _generator(*seed):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(int(np.random.SeedSequence(list(seed)).generate_state(1)[0]))
    return g


def _coded(x, scale_rows=1, pad=0, at=0):
    """x as a CodeMatrix with NaN codes past its columns and rows; its scales begin `at` bytes into a word."""
    az, torch = _az()
    rows, cols = x.shape
    ld = -(-cols // 16) * 16 + pad
    whole = torch.full((rows + 1, ld), 0x7F, dtype=torch.uint8, device="cuda")
    shape = (-(-rows // scale_rows), -(-cols // 128))
    scales = torch.full((shape[0] * shape[1] + 8,), 0xFF, dtype=torch.uint8, device="cuda")
    m = az.CodeMatrix(whole[:rows], scales[at:at + shape[0] * shape[1]].view(shape), cols, scale_rows)
    az.quantize_tensors(x, m)
    return m


def _rows(rows, cols, dtype, ld, offset=0, fill=7.0):
    """(view, whole): rows of `cols` in memory that is `fill` throughout."""
    import torch
    whole = torch.full((offset + rows * ld + 8,), fill, dtype=dtype, device="cuda")
    return whole[offset:offset + rows * ld].view(rows, ld)[:, :cols], whole


def _dot(a, b):
    """a b^T in float64, by rows that fit."""
    import torch
    bt = b.double().t().contiguous()
    return torch.cat([torch.mm(p.double(), bt) for p in a.split(4096)])


def _launched(call):
    """(name, grid) of each kernel of this library that call launches, from the profiler's trace."""
    import torch
    from torch.profiler import ProfilerActivity, profile
    found = []
    for _ in range(3):  # a trace without any kernel says nothing about the call
        torch.cuda.synchronize()
        with profile(activities=[ProfilerActivity.CPU, ProfilerActivity.CUDA]) as prof:
            call()
            torch.cuda.synchronize()
        with tempfile.TemporaryDirectory() as d:
            path = os.path.join(d, "trace.json")
            prof.export_chrome_trace(path)
            with open(path) as f:
                events = json.load(f)["traceEvents"]
        found = [(re.sub(r"\s", "", re.search(r"az_\w+(<[^()]*>)?", e["name"]).group(0)), e["args"]["grid"])
                 for e in events if e.get("cat") == "kernel" and "az_" in e.get("name", "")]
        if found:
            break
    return found


# --------------------------------------------------------------------------- #
# The weight's gradient
# --------------------------------------------------------------------------- #
COPY, MOVE, SHORT = 0, 1, 2
# rows, n, columns, and what runs them: (64 W columns and rows of a tile, parts of the rows)
GRADS = [((1, 13, 40), (2, 1)), ((65, 13, 129), (2, 1)), ((64, 3, 20), (2, 1)), ((130, 257, 200), (2, 1)),
         ((4097, 41, 33), (2, 22)), ((1000, 1881, 2050), (2, 1)), ((200, 4001, 4001), (4, 1)), ((65, 2051, 4101), (4, 1)),
         ((300, 3001, 4100), (4, 1)), ((11767, 1411, 1283), (4, 4))]


@pytest.mark.parametrize("shape,cut", GRADS)
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("feed,add,pad,offset", [("copy", False, 0, 0), ("copy", True, 8, 8), ("move", False, 1, 0), ("move", True, 3, 1)])
def test_weight_grad_is_exact_on_whole_numbers(shape, cut, out, feed, add, pad, offset):
    az, torch = _az()
    m, n, k = shape
    g = _generator(m, n, k, add)
    x, y = _whole(g, m, k), torch.randint(-3, 4, (m, n), generator=g, device="cuda").to(torch.bfloat16)
    xq = _coded(x, pad=16 * (pad % 2), at=pad % 4)
    # "copy": rows 16 bytes apart, whatever n is; past n they hold NaN
    ldy = -(-n // 8) * 8 + pad if feed == "copy" else (n | 1) + 2 * pad
    dy, _ = _rows(m, n, torch.bfloat16, ldy, offset, float("nan"))
    dy.copy_(y)
    dt = torch.float32 if out == "f32" else torch.bfloat16
    w0, b0 = _whole(g, n, k), torch.randint(-3, 4, (n,), generator=g, device="cuda").float()
    dw, whole = _rows(n, k, dt, k + pad, offset)
    dw.copy_(w0) if add else dw.fill_(float("nan"))
    db = b0.clone() if add else torch.full_like(b0, float("nan"))
    ws = torch.full((max(az.az_codes_weight_grad_workspace(m, n, k), 16),), 0xFF, dtype=torch.uint8, device="cuda")
    ran = _launched(lambda: az.weight_grad_tensors(dy, xq, dw, db=db, workspace=ws)) if not add else None
    if add:
        az.weight_grad_tensors(dy, xq, dw, db=db, accumulate=True, workspace=ws)
    want = _dot(y.float().t().contiguous(), x.t().contiguous())
    wb = y.double().sum(dim=0)
    if add:
        want, wb = want + w0.double(), wb + b0.double()
    assert torch.equal(dw, want.float().to(dt))
    assert torch.equal(db, wb.float())
    dw.fill_(7.0)
    assert bool((whole == 7.0).all())  # nothing past the rows was written
    if ran is not None:
        kind = COPY if feed == "copy" else MOVE if n >= 8 else SHORT
        f32 = str(out == "f32" or cut[1] > 1).lower()
        assert [(r[0], r[1][1]) for r in ran[:1]] == [(f"az_weight_grad<{cut[0]},{f32},{kind}>", cut[1])]
        assert [r[0] for r in ran[1:]] == ([f"az_join_parts<{str(out == 'f32').lower()}>"] if cut[1] > 1 else [])
