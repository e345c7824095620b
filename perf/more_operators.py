"""A dense layer served from 4 bits and trained in 8, from the residual stream to a chosen entry.

perf/operators.py measures the layer in 8 bits; here are the operators beside it:

  norm         root-mean-square norm of a residual stream with the residual's addition, its
               result e4m3 codes with a scale for each block of 128 (the product's operand)
               or a dense matrix
  norm_grad    its gradient: the stream's and the weight's
  checkpoint4  a matrix to 4-bit codes (e2m1) with a power-of-two scale for each block of 32
               columns and back, weights with the transposed matrix of the backward pass too
  matmul4      the product of 4-bit or e4m3 activations and 4-bit weights
  sample       one entry a row from logits, by temperature, top-k, top-p and min-p, from a
               given random number

Widths come from the library's networks: 128 x 64 and 160 x 64 trunk features, 4,672 and
1,880 policy entries, batches from one position to 1,024; the rest of the range is generic.
"""
import math

import torch

own = False  # False: elementary torch operations; True: the library's entry points

BLOCK8 = 128  # columns that share a scale in e4m3
BLOCK4 = 32   # and in e2m1
EPS = 1e-6


def listed():
    return [
        # One position's features on their way into an 8-bit head: latency is all.
        dict(name="norm_row_8192", op="norm", rows=1, cols=8192, dtype="bf16", residual=True, weight=True, codes=True),
        # A training step's residual stream into an 8-bit layer.
        dict(name="norm_16384x4096", op="norm", rows=16384, cols=4096, dtype="bf16", residual=True, weight=True, codes=True),
        # A ragged batch in fp32, dense results.
        dict(name="norm_333x10240_f32", op="norm", rows=333, cols=10240, dtype="f32", residual=False, weight=True, codes=False),
        # The gradient of a small batch.
        dict(name="norm_grad_64x10240", op="norm_grad", rows=64, cols=10240, dtype="bf16", residual=True, weight=True),
        # The gradient of a training step.
        dict(name="norm_grad_16384x4096", op="norm_grad", rows=16384, cols=4096, dtype="bf16", residual=True, weight=True),
        # A small batch's activation, saved in 4 bits and restored.
        dict(name="checkpoint4_64x10240", op="checkpoint4", rows=64, cols=10240, dtype="bf16", transposed=False),
        # The dense head's weights after an optimizer step, with their transposed copy for the backward pass.
        dict(name="checkpoint4_4672x8192", op="checkpoint4", rows=4672, cols=8192, dtype="f32", transposed=True),
        # One position through a dense head in 4 bits: the weights' bytes.
        dict(name="matmul4_1x4672x8192", op="matmul4", a="e4m3", m=1, n=4672, k=8192, out="bf16", bias=True),
        # A ragged batch with fp32 logits.
        dict(name="matmul4_333x1880x10240_f32", op="matmul4", a="e2m1", m=333, n=1880, k=10240, out="f32", bias=True),
        # The largest product.
        dict(name="matmul4_8192x8192x8192", op="matmul4", a="e2m1", m=8192, n=8192, k=8192, out="bf16", bias=False),
        # One position's move: temperature and min-p over the move planes.
        dict(name="sample_1x4672", op="sample", rows=1, vocab=4672, dtype="f32", top_k=0, top_p=False, min_p=True),
        # A full decoding batch over a large vocabulary with all of the filters.
        dict(name="sample_512x131072", op="sample", rows=512, vocab=131072, dtype="bf16", top_k=1000, top_p=True, min_p=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "norm", "norm_grad", "norm_grad", "checkpoint4", "matmul4", "matmul4", "matmul4", "sample", "sample", "sample"])
    while True:
        if op in ("norm", "norm_grad", "checkpoint4"):
            c = dict(op=op, rows=_log_int(rng, 1, 16384), cols=_log_int(rng, 16, 16384), dtype=rng.choice(["bf16", "f32"]))
            if op == "checkpoint4":
                c["transposed"] = rng.choice([False, True])
            else:
                c.update(residual=rng.choice([False, True]), weight=rng.choice([True, True, False]))
            if op == "norm":
                c["codes"] = rng.choice([False, True])
            # (fp32 has twice the bytes of the listed bf16)
            if c["rows"] * c["cols"] <= (4672 * 8192 if op == "checkpoint4" else 16384 * (4096 if c["dtype"] == "bf16" else 2048)):
                return c
        elif op == "matmul4":
            c = dict(op=op, a=rng.choice(["e4m3", "e2m1"]), m=_log_int(rng, 1, 8192), n=_log_int(rng, 16, 8192),
                     k=_log_int(rng, 16, 10240), out=rng.choice(["bf16", "bf16", "f32"]), bias=rng.choice([False, True]))
            if c["m"] * c["n"] * c["k"] <= 8192 ** 3:
                return c
        else:
            return dict(op=op, rows=_log_int(rng, 1, 512), vocab=_log_int(rng, 16, 131072), dtype=rng.choice(["bf16", "f32"]),
                        top_k=rng.choice([0, 0, 1, 1]) * _log_int(rng, 1, 2000), top_p=rng.choice([False, True]),
                        min_p=rng.choice([False, True]))


# --------------------------------------------------------------------------- #
# What a pass cannot do without
# --------------------------------------------------------------------------- #
_SIZE = {"f32": 4, "bf16": 2}


def _up(n, b):
    return -(-n // b)


def _stored8(rows, cols):
    """Bytes of an e4m3 matrix."""
    return rows * cols + rows * _up(cols, BLOCK8)


def _stored4(rows, cols):
    """Bytes of an e2m1 matrix."""
    return rows * _up(cols, 2) + rows * _up(cols, BLOCK4)


def work(case):
    c = case
    if c["op"] in ("norm", "norm_grad"):
        n, z = c["rows"] * c["cols"], _SIZE[c["dtype"]]
        if c["op"] == "norm":
            read = n * z * (3 if c["residual"] else 1)  # x; the residual and the sum
            return {"bytes": read + (_stored8(c["rows"], c["cols"]) if c["codes"] else n * z) + 4 * c["cols"] * c["weight"],
                    "flops": 5 * n}
        return {"bytes": n * z * (4 if c["residual"] else 3) + 8 * c["cols"] * c["weight"], "flops": 11 * n}
    if c["op"] == "checkpoint4":  # the codes are written by the one half and read by the other
        n = c["rows"] * c["cols"]
        return {"bytes": n * _SIZE[c["dtype"]] * (3 if c["transposed"] else 2) + 2 * _stored4(c["rows"], c["cols"]) +
                2 * _stored4(c["cols"], c["rows"]) * c["transposed"], "flops": 4 * n}
    if c["op"] == "matmul4":
        m, n, k = c["m"], c["n"], c["k"]
        return {"bytes": (_stored8 if c["a"] == "e4m3" else _stored4)(m, k) + _stored4(n, k) + m * n * _SIZE[c["out"]] + 4 * n * c["bias"],
                "flops": 2 * m * n * k}
    b, v = c["rows"], c["vocab"]
    return {"bytes": b * v * _SIZE[c["dtype"]] + 28 * b, "flops": 4 * b * v}


# --------------------------------------------------------------------------- #
# Inputs
# --------------------------------------------------------------------------- #
_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
_DEV = "cuda"


def _activations(g, rows, cols):
    """A stream whose channels differ in size, as layers of a trunk add it up."""
    x = torch.randn((rows, cols), generator=g, device=_DEV)
    return x * torch.exp(0.7 * torch.randn((1, cols), generator=g, device=_DEV))


def _weights(g, rows, cols):
    return torch.randn((rows, cols), generator=g, device=_DEV) * math.sqrt(2.0 / cols)


def _padded(x, to=16):
    """The matrix in rows of a multiple of `to` elements."""
    rows, cols = x.shape
    out = torch.zeros((rows, _up(cols, to) * to), dtype=x.dtype, device=x.device)
    out[:, :cols] = x
    return out


def _empty4(rows, cols):
    """Codes and scales of a 4-bit matrix, not yet written."""
    return (torch.zeros((rows, _up(cols, 32) * 16), dtype=torch.uint8, device=_DEV),
            torch.zeros((rows, _up(cols, 4 * BLOCK4) * 4), dtype=torch.uint8, device=_DEV))


def prepare(case, seed):
    c = case
    g = torch.Generator(device=_DEV)
    g.manual_seed(int(seed))
    s = dict(case=c)
    if c["op"] in ("norm", "norm_grad"):
        rows, cols, dt = c["rows"], c["cols"], _TORCH[c["dtype"]]
        s["x"] = _activations(g, rows, cols).to(dt)
        s["weight"] = 1.0 + 0.2 * torch.randn((cols,), generator=g, device=_DEV) if c["weight"] else None
        if c["op"] == "norm":
            s["residual"] = _activations(g, rows, cols).to(dt) if c["residual"] else None
            s["sum"] = torch.empty_like(s["x"]) if c["residual"] else None
            if c["codes"]:
                s["codes"] = _padded(torch.zeros((rows, cols), dtype=torch.uint8, device=_DEV))
                s["scales"] = torch.zeros((rows, _up(cols, BLOCK8)), dtype=torch.uint8, device=_DEV)
            else:
                s["y"] = torch.empty_like(s["x"])
        else:
            s["dy"] = (torch.randn((rows, cols), generator=g, device=_DEV) / rows).to(dt)
            s["dsum"] = (torch.randn((rows, cols), generator=g, device=_DEV) / rows).to(dt) if c["residual"] else None
            s["dx"] = torch.empty_like(s["x"])
            s["dw"] = torch.empty((cols,), device=_DEV) if c["weight"] else None
    elif c["op"] == "checkpoint4":
        rows, cols, dt = c["rows"], c["cols"], _TORCH[c["dtype"]]
        s["x"] = (_weights if c["transposed"] else _activations)(g, rows, cols).to(dt)
        s["q"], s["restored"] = _empty4(rows, cols), torch.empty_like(s["x"])
        if c["transposed"]:
            s["qt"], s["restored_t"] = _empty4(cols, rows), torch.empty((cols, rows), dtype=dt, device=_DEV)
    elif c["op"] == "matmul4":
        m, n, k = c["m"], c["n"], c["k"]
        x = _activations(g, m, k)
        if c["a"] == "e4m3":
            codes, scales = _quantize8(x)
            s["a"] = (_padded(codes), scales)
        else:
            s["a"] = _stored(x)
        s["b"] = _stored(_weights(g, n, k))
        s["bias"] = 0.1 * torch.randn((n,), generator=g, device=_DEV) if c["bias"] else None
        s["out"] = torch.empty((m, n), dtype=_TORCH[c["out"]], device=_DEV)
    else:
        b, v = c["rows"], c["vocab"]
        l = 3.0 * torch.randn((b, v), generator=g, device=_DEV)
        # Half of the rows allow some 30 entries, as a position does; one in eight has nothing to choose from.
        few = torch.rand((b, 1), generator=g, device=_DEV) < 0.5
        at = torch.arange(b, device=_DEV).unsqueeze(1)
        allowed = (~few | (torch.rand((b, v), generator=g, device=_DEV) < min(1.0, 30.0 / v))) & (at % 8 != 5)
        s["logits"] = torch.where(allowed, l, -math.inf).to(_TORCH[c["dtype"]])
        s["u"] = torch.rand((b,), generator=g, device=_DEV)
        # One row in eight takes the largest.
        warm = 0.5 + torch.rand((b,), generator=g, device=_DEV)
        s["temperature"] = torch.where(at[:, 0] % 8 == 3, 0.0, warm)
        s["top_k"] = torch.randint(1, c["top_k"] + 1, (b,), generator=g, device=_DEV, dtype=torch.int32) if c["top_k"] else None
        s["top_p"] = 0.5 + 0.5 * torch.rand((b,), generator=g, device=_DEV) if c["top_p"] else None
        s["min_p"] = 0.1 * torch.rand((b,), generator=g, device=_DEV) if c["min_p"] else None
        s["out"] = torch.empty((b,), dtype=torch.int32, device=_DEV)
        s["prob"] = torch.empty((b,), device=_DEV)
    return s


# --------------------------------------------------------------------------- #
# The plain forms
# --------------------------------------------------------------------------- #
def _power(e):
    """2^e in float32, -126 <= e <= 127."""
    return ((e + 127) << 23).view(torch.float32)


def _blocks(x, block):
    """x in blocks of columns, the last one filled up with zeros."""
    return torch.nn.functional.pad(x, (0, -x.shape[1] % block)).view(x.shape[0], -1, block)


def _quantize8(x):
    """e4m3 codes and scale bytes; the smallest scale that keeps a block within 448 = 7/8 * 2^9."""
    rows, cols = x.shape
    blocks = _blocks(x.float(), BLOCK8)
    f, e = torch.frexp(blocks.abs().amax(dim=2, keepdim=True))
    e = torch.where(f == 0, 0, (e - 9 + (f > 0.875).to(torch.int32)).clamp(-117, 119)).to(torch.int32)
    codes = (blocks * _power(-e)).clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)
    return codes.view(rows, -1)[:, :cols].contiguous(), (e[:, :, 0] + 127).to(torch.uint8)


def _value8(codes, scales, cols):
    values = _blocks(codes[:, :cols].contiguous().view(torch.float8_e4m3fn).float(), BLOCK8)
    return (values * _power(scales.to(torch.int32) - 127).unsqueeze(2)).view(codes.shape[0], -1)[:, :cols]


def _quantize4(x):
    """Values of the e2m1 codes [rows][blocks][32] and exponents; the smallest scale that keeps a block within 6 = 3/4 * 2^3."""
    blocks = _blocks(x.float(), BLOCK4)
    f, e = torch.frexp(blocks.abs().amax(dim=2, keepdim=True))
    e = torch.where(f == 0, 0, (e - 3 + (f > 0.75).to(torch.int32)).clamp(-125, 125)).to(torch.int32)
    y = (blocks * _power(-e)).clamp(-6.0, 6.0)
    size = y.abs()
    step = torch.where(size < 2.0, 0.5, torch.where(size < 4.0, 1.0, 2.0))
    return torch.copysign(torch.round(size / step) * step, y), e


def _restore4(x):
    """x by way of its 4-bit form, as it comes back."""
    codes, e = _quantize4(x)
    return (codes * _power(e)).view(x.shape[0], -1)[:, :x.shape[1]].to(x.dtype)


def _stored(x):
    """(codes two to a byte, scale bytes) of x, in rows of whole chunks of 16 bytes and words."""
    codes, e = _quantize4(x)
    rows = x.shape[0]
    size = codes.abs()
    bits = torch.where(size < 2.0, size * 2.0, torch.where(size < 4.0, size + 2.0, size / 2.0 + 4.0)).to(torch.uint8)
    bits = (bits | (torch.signbit(codes).to(torch.uint8) << 3)).view(rows, -1)
    return bits[:, 0::2] | (bits[:, 1::2] << 4), _padded((e[:, :, 0] + 127).to(torch.uint8), 4)


def _value4(codes, scales, cols):
    values = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=codes.device)
    bits = torch.stack([codes & 15, codes >> 4], dim=2).view(codes.shape[0], -1)[:, :cols]
    x = values[(bits & 7).int()]
    x = _blocks(torch.where(bits > 7, -x, x), BLOCK4)
    return (x * _power(scales[:, :x.shape[1]].to(torch.int32) - 127).unsqueeze(2)).view(codes.shape[0], -1)[:, :cols]


def _codes(codes, scales, cols):
    """e4m3 codes and scales as the values that they stand for."""
    return {"codes": codes[:, :cols].view(torch.float8_e4m3fn), "scales": scales.view(torch.float8_e8m0fnu)}


def _norm(s, c):
    h = s["x"] if s["residual"] is None else (s["x"].float() + s["residual"].float()).to(s["x"].dtype)
    out = {} if s["residual"] is None else {"sum": h}
    h = h.float()
    y = h * torch.rsqrt(h.square().mean(dim=1, keepdim=True) + EPS)
    if s["weight"] is not None:
        y = y * s["weight"]
    return {**out, **_codes(*_quantize8(y), c["cols"])} if c["codes"] else {**out, "y": y.to(s["x"].dtype)}


def _norm_grad(s, c):
    h, dy = s["x"].float(), s["dy"].float()
    r = torch.rsqrt(h.square().mean(dim=1, keepdim=True) + EPS)
    unit = h * r
    g = dy if s["weight"] is None else dy * s["weight"]
    dx = r * (g - unit * (g * unit).mean(dim=1, keepdim=True))
    if s["dsum"] is not None:
        dx = dx + s["dsum"].float()
    out = {"dx": dx.to(s["x"].dtype)}
    return out if s["weight"] is None else {**out, "dw": (dy * unit).sum(dim=0)}


def _sample(s, c):
    l, t = s["logits"].float(), s["temperature"].double().unsqueeze(1)
    l, at = torch.sort(l, dim=1, descending=True, stable=True)  # ties: the lowest index first
    top = l[:, :1]
    rank = torch.arange(c["vocab"], device=l.device)
    # The weights in 64 bits, so that an entry at a border falls where it belongs.
    w = torch.where(t > 0, torch.exp((l.double() - top) / t), (rank == 0).double())
    w = torch.where(top > -math.inf, w, 0.0)
    if s["top_k"] is not None:
        w = torch.where(rank < s["top_k"].unsqueeze(1), w, 0.0)
    if s["top_p"] is not None:
        before = torch.cumsum(w, dim=1) - w
        keep = before < s["top_p"].double().unsqueeze(1) * w.sum(dim=1, keepdim=True)
        w = torch.where(keep | (rank == 0), w, 0.0)
    if s["min_p"] is not None:
        w = torch.where(w >= s["min_p"].double().unsqueeze(1), w, 0.0)
    w = torch.zeros_like(w).scatter_(1, at, w)  # back in the order of the entries
    sums = torch.cumsum(w, dim=1)
    total = sums[:, -1]
    token = (sums <= (s["u"].double() * total).unsqueeze(1)).sum(dim=1).clamp(max=c["vocab"] - 1)
    prob = w.gather(1, token.unsqueeze(1))[:, 0] / total.clamp(min=1e-300)
    return {"token": torch.where(total > 0, token, -1).to(torch.int32), "prob": prob.float()}


def run(state):
    s, c = state, state["case"]
    if own:
        return _own(s, c)
    if c["op"] == "norm":
        return _norm(s, c)
    if c["op"] == "norm_grad":
        return _norm_grad(s, c)
    if c["op"] == "checkpoint4":
        out = {"restored": _restore4(s["x"])}
        if c["transposed"]:
            out["transposed"] = _restore4(s["x"].t())
        return out
    if c["op"] == "matmul4":
        out = (_value8 if c["a"] == "e4m3" else _value4)(*s["a"], c["k"]) @ _value4(*s["b"], c["k"]).t()
        return (out if s["bias"] is None else out + s["bias"]).to(_TORCH[c["out"]])
    return _sample(s, c)


# --------------------------------------------------------------------------- #
# The library's entry points
# --------------------------------------------------------------------------- #
def _own(s, c):
    import paper_2609_37447_amd as az
    if c["op"] == "norm":
        q = az.CodeMatrix(s["codes"], s["scales"], c["cols"]) if c["codes"] else None
        y = None if c["codes"] else s["y"]
        az.norm_tensors(s["x"], y=y, q=q, residual=s["residual"], sum=s["sum"], weight=s["weight"], eps=EPS)
        out = {} if s["sum"] is None else {"sum": s["sum"]}
        return {**out, **_codes(s["codes"], s["scales"], c["cols"])} if c["codes"] else {**out, "y": y}
    if c["op"] == "norm_grad":
        az.norm_grad_tensors(s["dy"], s["x"], s["dx"], dsum=s["dsum"], weight=s["weight"], dw=s["dw"], eps=EPS)
        return {"dx": s["dx"]} if s["dw"] is None else {"dx": s["dx"], "dw": s["dw"]}
    if c["op"] == "checkpoint4":
        q = az.Fp4Matrix(*s["q"], c["cols"])
        qt = az.Fp4Matrix(*s["qt"], c["rows"]) if c["transposed"] else None
        az.quantize_tensors(s["x"], q, qt)
        az.dequantize_tensors(q, s["restored"])
        if not c["transposed"]:
            return {"restored": s["restored"]}
        az.dequantize_tensors(qt, s["restored_t"])
        return {"restored": s["restored"], "transposed": s["restored_t"]}
    if c["op"] == "matmul4":
        a = az.CodeMatrix(*s["a"], c["k"]) if c["a"] == "e4m3" else az.Fp4Matrix(*s["a"], c["k"])
        az.matmul_tensors(a, az.Fp4Matrix(*s["b"], c["k"]), s["out"], bias=s["bias"])
        return s["out"]
    az.sample_tensors(s["logits"], s["u"], s["out"], prob=s["prob"], temperature=s["temperature"], top_k=s["top_k"],
                      top_p=s["top_p"], min_p=s["min_p"])
    return {"token": s["out"], "prob": s["prob"]}


# --------------------------------------------------------------------------- #
# The definition in 64 bits
# --------------------------------------------------------------------------- #
def _two_to(e):
    """2^e in float64 for whole e, from its bits."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _floor_log2(a):
    """The largest e with 2^e <= a, for normal a > 0."""
    return ((a.view(torch.int64) >> 52) - 1023).double()


def _grid(x, block, most, digits, least, low, high):
    """(codes' values, scales), float64, of x in blocks of columns: the format's largest value, the binary digits behind a
    code's first, the exponent of its smallest normal value, and the limits of a scale's exponent."""
    rows, cols = x.shape
    x = torch.nn.functional.pad(x, (0, -cols % block)).view(rows, -1, block)
    top = x.abs().amax(dim=2, keepdim=True)
    e = _floor_log2(top.clamp(min=1e-290) / most)
    e = torch.where(_two_to(e) * most < top, e + 1, e).clamp(low, high)
    scales = torch.where(top == 0, 1.0, _two_to(e))
    y = x / scales
    step = _two_to(_floor_log2(y.abs().clamp(min=2.0 ** least)) - digits)
    codes = (torch.round(y / step) * step).clamp(-most, most)
    return codes, scales


def _grid4(x):
    codes, scales = _grid(x, BLOCK4, 6.0, 1, 0, -125, 125)
    return (codes * scales).view(x.shape[0], -1)[:, :x.shape[1]].contiguous()


def _e4m3(byte):
    ex, man = (byte >> 3) & 15, byte & 7
    size = man / 8 * 2.0 ** -6 if ex == 0 else (1 + man / 8) * 2.0 ** (ex - 7)
    return math.nan if byte & 127 == 127 else -size if byte & 128 else size


def _e2m1(bits):
    ex, man = (bits >> 1) & 3, bits & 1
    size = man / 2 if ex == 0 else (1 + man / 2) * 2.0 ** (ex - 1)
    return -size if bits & 8 else size


def _decoded(codes, scales, cols, four):
    """Values of a coded matrix in float64, from the format's definition."""
    at = torch.arange(cols, device=codes.device)
    if four:
        table = torch.tensor(list(map(_e2m1, range(16))), dtype=torch.float64, device=codes.device)
        bits = (codes[:, at // 2].long() >> (4 * (at % 2))) & 15
    else:
        table = torch.tensor(list(map(_e4m3, range(256))), dtype=torch.float64, device=codes.device)
        bits = codes[:, :cols].long()
    return table[bits] * _two_to(scales.to(torch.int64) - 127)[:, at // (BLOCK4 if four else BLOCK8)]


def _drawn(l, u, t, k, p, floor):
    """(entry, its probability) of one row of logits in float64; (-1, 0) where nothing is allowed."""
    best = l.max()
    if not bool(best > -math.inf):
        return -1, 0.0
    order = torch.argsort(l, descending=True, stable=True)
    if not t > 0:
        return int(order[0]), 1.0
    e = torch.exp((l[order] - best) / t)
    if k is not None:
        e = e[:k]
    n = e.numel()
    if p is not None:
        n = max(1, int((torch.cat([e.new_zeros(1), e.cumsum(0)[:-1]]) < p * e.sum()).sum()))
    if floor is not None:
        n = min(n, int((e >= floor).sum()))
    kept, back = torch.sort(order[:n])
    e = e[:n][back]
    sums = e.cumsum(0)
    i = min(int(torch.searchsorted(sums, u * sums[-1], right=True)), n - 1)
    return int(kept[i]), float(e[i] / sums[-1])


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] == "norm":
        h, out = s["x"].double(), {}
        if s["residual"] is not None:
            h = h + s["residual"].double()
            out["sum"] = h
            h = h.to(s["x"].dtype).double()
        y = h / torch.sqrt((h * h).mean(dim=1, keepdim=True) + EPS)
        if s["weight"] is not None:
            y = y * s["weight"].double()
        if not c["codes"]:
            return {**out, "y": y}
        codes, scales = _grid(y, BLOCK8, 448.0, 3, -6, -117, 119)
        return {**out, "codes": codes.view(c["rows"], -1)[:, :c["cols"]].contiguous(), "scales": scales[:, :, 0]}
    if c["op"] == "norm_grad":
        h, dy = s["x"].double(), s["dy"].double()
        r = 1.0 / torch.sqrt((h * h).mean(dim=1, keepdim=True) + EPS)
        g = dy if s["weight"] is None else dy * s["weight"].double()
        dx = r * g - h * (r ** 3 * (g * h).mean(dim=1, keepdim=True))
        if s["dsum"] is not None:
            dx += s["dsum"].double()
        return {"dx": dx} if s["weight"] is None else {"dx": dx, "dw": (dy * (h * r)).sum(dim=0)}
    if c["op"] == "checkpoint4":
        x = s["x"].double()
        return {"restored": _grid4(x), "transposed": _grid4(x.t().contiguous())} if c["transposed"] else {"restored": _grid4(x)}
    if c["op"] == "matmul4":
        a, b = _decoded(*s["a"], c["k"], c["a"] == "e2m1"), _decoded(*s["b"], c["k"], True)
        out = torch.mm(a, b.t().contiguous())
        return out if s["bias"] is None else out + s["bias"].double()
    pick = lambda key, i: None if s[key] is None else s[key][i].item()  # noqa: E731
    got = [_drawn(s["logits"][i].double(), *(pick(key, i) for key in ("u", "temperature", "top_k", "top_p", "min_p")))
           for i in range(c["rows"])]
    return {"token": torch.tensor([t for t, _ in got]), "prob": torch.tensor([p for _, p in got], dtype=torch.float64)}
