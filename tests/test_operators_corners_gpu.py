"""Calls of the stand-alone operators at the corners of what they document: NaN in a gradient's operands, row
strides at their limits, workspaces made inside a call on another stream or in a captured graph, the longest
vocabulary, empty histories.  Sums are of small whole numbers (exact in fp32) where values are compared for equality."""

import pytest

from .test_codes_kernels_gpu import _az, _coded, _dot, _generator, _rows, _whole

pytestmark = pytest.mark.gpu


# --------------------------------------------------------------------------- #
# NaN
# --------------------------------------------------------------------------- #
@pytest.mark.parametrize("m,n,k", [(70, 40, 300), (200, 4001, 4001), (4097, 41, 300)])
@pytest.mark.parametrize("aligned", [True, False])
def test_nan_in_a_gradients_operands_stays_in_its_row_and_column(m, n, k, aligned):
    az, torch = _az()
    g = _generator(m, n, aligned)
    x = _whole(g, m, k)
    x[m - 3] = 0.0                                  # (a block of zeros is NaN as well if its scale is)
    xq = _coded(x)
    xq.codes[m - 1, 7] = 0x7F                       # column 7
    xq.scales[m - 3, 1] = 255                       # columns 128..255
    dy, _ = _rows(m, n, torch.bfloat16, -(-n // 8) * 8 if aligned else (n | 1) + 2, fill=float("nan"))
    dy.copy_(torch.randint(-3, 4, (m, n), generator=g, device="cuda"))
    dy[m // 2, n - 2] = float("nan")                # row n - 2
    dw, db = torch.zeros((n, k), device="cuda"), torch.zeros((n,), device="cuda")
    az.weight_grad_tensors(dy, xq, dw, db=db)
    want = torch.zeros((n, k), dtype=torch.bool, device="cuda")
    want[n - 2] = True
    want[:, 7] = True
    want[:, 128:256] = True
    assert torch.equal(torch.isnan(dw), want)
    assert torch.equal(torch.isnan(db).nonzero().flatten().cpu(), torch.tensor([n - 2]))
    back = torch.zeros((m, k), device="cuda")
    az.dequantize_tensors(xq, back)
    want = torch.zeros((m, k), dtype=torch.bool, device="cuda")
    want[m - 1, 7] = True
    want[m - 3, 128:256] = True
    assert torch.equal(torch.isnan(back), want)


# --------------------------------------------------------------------------- #
# Row strides at their limits
# --------------------------------------------------------------------------- #
def _far(x, ld):
    """x as a CodeMatrix whose rows are ld bytes apart, on memory that is otherwise not written."""
    az, torch = _az()
    rows, cols = x.shape
    codes = torch.empty((rows - 1) * ld + -(-cols // 16) * 16, dtype=torch.uint8, device="cuda").as_strided((rows, cols), (ld, 1))
    m = az.CodeMatrix(codes, torch.empty((rows, -(-cols // 128)), dtype=torch.uint8, device="cuda"))
    az.quantize_tensors(x, m)
    back = torch.empty_like(x)
    az.dequantize_tensors(m, back)
    assert torch.equal(back, x)
    return m


# tiles up to ld < 2^22, the kernel of few rows up to ld < 2^27
@pytest.mark.parametrize("m,n,k,ld", [(1501, 2051, 333, 2 ** 22 - 16), (40, 33, 1111, 2 ** 22), (17, 18, 300, 2 ** 27 - 16)])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_matmul_of_rows_far_apart(m, n, k, ld, out):
    az, torch = _az()
    g = _generator(m, n, k)
    x, w = _whole(g, m, k), _whole(g, n, k)
    o = torch.empty((m, n), dtype=torch.float32 if out == "f32" else torch.bfloat16, device="cuda")
    az.matmul_tensors(_far(x, ld), _far(w, ld), o)
    assert torch.equal(o, _dot(x, w).float().to(o.dtype))


# x: ld < 2^25; dy: copied up to ld < 2^23, through registers beyond
@pytest.mark.parametrize("ldx,ldy", [(2 ** 25 - 16, 2 ** 23 - 8), (1024, 2 ** 23), (1024, 2 ** 23 + 1)])
def test_weight_grad_of_rows_far_apart(ldx, ldy):
    az, torch = _az()
    m, n, k = 130, 67, 300
    g = _generator(ldx & 0xfff, ldy & 0xfff)
    x = _whole(g, m, k)
    dy = torch.empty((m - 1) * ldy + n, dtype=torch.bfloat16, device="cuda").as_strided((m, n), (ldy, 1))
    dy.copy_(torch.randint(-3, 4, (m, n), generator=g, device="cuda"))
    dw, db = torch.empty((n, k), device="cuda"), torch.empty((n,), device="cuda")
    az.weight_grad_tensors(dy, _far(x, ldx), dw, db=db)
    y = dy.float()
    assert torch.equal(dw, _dot(y.t().contiguous(), x.t().contiguous()).float())
    assert torch.equal(db, y.sum(dim=0))


def test_strides_past_the_limits_are_refused():
    az, torch = _az()
    one = torch.zeros((1, 1), dtype=torch.uint8, device="cuda")
    a = az.CodeMatrix(torch.empty(2 ** 27 + 16, dtype=torch.uint8, device="cuda").as_strided((2, 16), (2 ** 27, 1)), one.repeat(2, 1))
    b = az.CodeMatrix.empty(3, 16)
    with pytest.raises(az.AzError) as e:
        az.matmul_tensors(a, b, torch.empty((2, 3), device="cuda"))
    assert e.value.status == az.AZ_ERR_UNSUPPORTED
    with pytest.raises(az.AzError) as e:
        az.weight_grad_tensors(torch.empty((2, 3), dtype=torch.bfloat16, device="cuda"), a, torch.empty((3, 16), device="cuda"))
    assert e.value.status == az.AZ_ERR_UNSUPPORTED


# --------------------------------------------------------------------------- #
# Workspaces made inside a call
# --------------------------------------------------------------------------- #
class _Sums:
    """A product and a gradient that are both cut into parts, and a policy in chunks, on workspaces of their calls."""

    def __init__(self):
        az, torch = _az()
        g = _generator(21)
        self.az = az
        self.x, self.w = _whole(g, 65, 3001), _whole(g, 4101, 3001)
        self.a, self.b = _coded(self.x), _coded(self.w, 128)
        self.s = _whole(g, 4097, 200)
        self.sq = _coded(self.s)
        self.dy = torch.randint(-3, 4, (4097, 40), generator=g, device="cuda").to(torch.bfloat16)
        self.logits = torch.randn((3, 50000), generator=g, device="cuda")
        self.o = torch.empty((65, 4101), device="cuda")
        self.dw, self.db = torch.empty((40, 200), device="cuda"), torch.empty((40,), device="cuda")
        self.p = torch.empty_like(self.logits)
        assert az.az_codes_matmul_workspace(self.a.c, self.b.c, az.AZ_F32) and az.az_codes_weight_grad_workspace(4097, 40, 200)

    def clear(self):
        for t in (self.o, self.dw, self.db, self.p):
            t.fill_(float("nan"))

    def call(self, stream=None):
        self.az.matmul_tensors(self.a, self.b, self.o, stream=stream)
        self.az.weight_grad_tensors(self.dy, self.sq, self.dw, db=self.db, stream=stream)
        self.az.policy_tensors(self.logits, self.p, stream=stream)

    def check(self):
        import torch
        assert torch.equal(self.o, _dot(self.x, self.w).float())
        assert torch.equal(self.dw, _dot(self.dy.float().t().contiguous(), self.s.t().contiguous()).float())
        assert torch.equal(self.db, self.dy.float().sum(dim=0))
        assert bool(((self.p.double() - torch.softmax(self.logits.double(), dim=1)).abs() < 1e-7).all())  # (each p below 0.01)


def test_a_given_stream_and_workspaces_of_the_call():
    import torch
    c, s = _Sums(), torch.cuda.Stream()
    for _ in range(3):
        c.clear()
        s.wait_stream(torch.cuda.current_stream())
        c.call(stream=s)
        s.synchronize()
        c.check()


def test_captured_calls_with_workspaces_of_their_own():
    import torch
    c = _Sums()
    c.call()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        c.call()
    for _ in range(4):
        c.clear()
        g.replay()
        torch.cuda.synchronize()
        c.check()
        c.clear()
        c.call()  # the program's own eager work between the replays
        torch.cuda.synchronize()
        c.check()


# --------------------------------------------------------------------------- #
# The policy
# --------------------------------------------------------------------------- #
def test_the_longest_vocabulary():
    import torch

    import paper_2609_37447_amd as az
    v = 1 << 24
    g = _generator(22)
    x = torch.randn((2, v), generator=g, device="cuda")
    out = torch.empty_like(x)
    az.policy_tensors(x, out)
    want = torch.softmax(x.double(), dim=1)
    # 22 * max |l| + 8 half steps, and the sum's: 16 a thread, 512 threads, 2,048 chunks of a row in 64 lanes
    off = 22 * float(x.abs().max()) + 8 + 16 + 6 + 8 + 2048 / 64 + 6
    assert bool(((out.double() - want).abs() <= want * 2.0 ** -24 * off).all())


@pytest.mark.parametrize("vocab", [33, 4700, 20001])
def test_bits_past_the_vocabulary_do_not_matter(vocab):
    import torch

    import paper_2609_37447_amd as az
    x = torch.randn((4, vocab), generator=_generator(vocab), device="cuda")
    mask = torch.full((4, -(-vocab // 32)), -1, dtype=torch.int32, device="cuda")
    out, want = torch.empty_like(x), torch.empty_like(x)
    az.policy_tensors(x, out, mask=mask)
    az.policy_tensors(x, want)
    assert torch.equal(out, want)


def test_a_history_of_no_entries():
    import torch

    import paper_2609_37447_amd as az
    x = torch.randn((3, 100), generator=_generator(23), device="cuda")
    out, want = torch.empty_like(x), torch.empty_like(x)
    az.policy_tensors(x, want)
    pen = torch.tensor([[1.5, 0.5, 0.5]] * 3, device="cuda")
    az.policy_tensors(x, out, history=torch.empty((3, 0), dtype=torch.int32, device="cuda"), penalties=pen)
    assert torch.equal(out, want)
    lengths = torch.zeros((3,), dtype=torch.int32, device="cuda")
    az.policy_tensors(x, out.fill_(0), history=torch.zeros((3, 5), dtype=torch.int32, device="cuda"), lengths=lengths, penalties=pen)
    assert torch.equal(out, want)
