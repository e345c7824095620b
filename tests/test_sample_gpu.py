"""The entry drawn from logits on the GPU against its float64 definition (oracle/layer.py).

Entries are compared where the definition's decisions are not nearer than 1e-9 of the whole sum to going the other
way; weights are whole multiples of 2^-S, S >= 38, each off by half of one (vocab 2^24), 45 for 2^17: sums of 2^17 of them
are within 2^17 * 2^-46 < 2e-9 of the largest weight, sums of fewer entries nearer.  Probabilities: half a step of fp32 beside that.
"""

import numpy as np
import pytest

from oracle import layer as O

from .test_codes_gpu import _az, _rng, _strided

pytestmark = pytest.mark.gpu


def _logits(rng, rows, vocab, dtype, spread=3.0):
    import torch
    t = torch.from_numpy((spread * rng.standard_normal((rows, vocab))).astype(np.float32))
    return t.to(torch.bfloat16) if dtype == "bf16" else t


def _run(t, u, pad=0, offset=0, **kw):
    az, torch = _az()
    td, _ = _strided(t, pad, offset=offset)
    dev = lambda a, d: torch.from_numpy(np.asarray(a, d)).cuda()  # noqa: E731
    out = torch.full((t.shape[0],), 77, dtype=torch.int32, device="cuda")
    prob = torch.full((t.shape[0],), 77.0, device="cuda")
    types = {"top_k": np.int32}
    az.sample_tensors(td, dev(u, np.float32), out, prob=prob, **{k: dev(v, types.get(k, np.float32)) for k, v in kw.items()})
    return out.cpu().numpy(), prob.double().cpu().numpy()


def _check(t, u, **kw):
    got, prob = _run(t, u, **kw)
    kw = {k: v for k, v in kw.items() if k not in ("pad", "offset")}
    names = {"temperature": np.float32, "top_k": np.int64, "top_p": np.float32, "min_p": np.float32}
    compared = 0
    for i in range(t.shape[0]):
        par = {k: names[k](v[i]).item() for k, v in kw.items()}
        want, p, near = O.draw(t[i].double().numpy(), float(np.float32(u[i])), **par)
        if near < 1e-9:
            continue
        compared += 1
        assert got[i] == want, (i, got[i], want, near, par)
        assert abs(prob[i] - p) <= (2.0 ** -24 + 1e-8) * p
    assert compared >= 0.9 * t.shape[0]


VOCABS = [1, 2, 7, 8, 9, 63, 100, 1000, 2049, 4096, 4097, 4672, 8191, 8193, 20000, 70001, 131072]


@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("filters", ["none", "k", "p", "m", "kp", "kpm"])
def test_draw(vocab, dtype, filters):
    rng = _rng(vocab, len(filters), 1)
    rows = 6
    t = _logits(rng, rows, vocab, dtype)
    kw = {"temperature": rng.uniform(0.3, 2.0, rows)}
    if "k" in filters:
        kw["top_k"] = np.maximum(1, np.exp(rng.uniform(0, np.log(vocab + 1), rows)).astype(np.int64))
    if "p" in filters:
        kw["top_p"] = rng.uniform(0.05, 0.999, rows)
    if "m" in filters:
        kw["min_p"] = rng.uniform(0.0, 0.2, rows)
    _check(t, rng.random(rows), pad=vocab % 3, offset=vocab % 2, **kw)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [300, 4672, 20000])
def test_ties_go_by_index(dtype, vocab):
    """A handful of values: thousands of equal logits at every border."""
    import torch
    rng = _rng(vocab, 2)
    rows = 12
    t = torch.from_numpy(rng.integers(-2, 3, (rows, vocab)).astype(np.float32)) * 0.5
    t[1] = 1.25                       # all equal
    t[2, : vocab // 2] = -0.0         # zeros of both signs are equal
    t = t.to(torch.bfloat16) if dtype == "bf16" else t
    for seed in range(3):
        r = _rng(vocab, seed, 3)
        _check(t, r.random(rows), top_k=r.integers(1, vocab, rows), top_p=r.uniform(0.1, 0.99, rows))
        _check(t, r.random(rows), top_k=r.integers(1, vocab, rows))
        _check(t, r.random(rows), top_p=r.uniform(0.1, 0.99, rows))


@pytest.mark.parametrize("vocab", [50, 4672, 30000])
def test_every_entry_has_its_part(vocab):
    """u in the middle of an entry's part draws that entry."""
    import torch
    rng = _rng(vocab, 4)
    l = _logits(rng, 1, vocab, "f32")
    at, w, _ = O.kept(l[0].double().numpy(), top_p=0.9)
    cum = np.cumsum(w) / w.sum()
    pick = np.unique(rng.integers(0, len(at), 40))
    pick = pick[w[pick] / w.sum() > 2.0 ** -18]
    mid = (cum - w / w.sum() / 2)[pick]
    t = l.expand(len(pick), vocab).contiguous()
    got, prob = _run(t, mid, top_p=np.full(len(pick), 0.9))
    assert np.array_equal(got, at[pick])
    assert np.all(np.abs(prob - (w / w.sum())[pick]) <= 1e-6 * prob)
    # the ends of the range
    got, _ = _run(l.expand(5, vocab).contiguous(), [0.0, 1.0 - 2.0 ** -24, 1.0, 7.0, float("nan")], top_p=np.full(5, 0.9))
    assert got.tolist() == [at[0], at[-1], at[-1], at[-1], at[0]]


@pytest.mark.parametrize("vocab", [9, 4672, 20000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_special_rows(vocab, dtype):
    import torch
    rng = _rng(vocab, 5)
    t = _logits(rng, 12, vocab, dtype)
    ninf = float("-inf")
    t[0] = ninf                                # nothing is allowed
    t[1, 3] = float("nan")
    t[2, 3] = float("inf")
    t[3, :] = ninf
    t[3, vocab - 1] = -3e38                    # one entry, far down
    t[4, vocab // 2:] = ninf
    t[5, :] = -1e30                            # far from each other
    t[5, 2] = 1e30
    t[6, :] = ninf
    t[6, 0], t[6, vocab - 1] = 1.0, 1.0
    got, prob = _run(t, np.full(12, 0.7), top_p=np.full(12, 0.95))
    assert got[:4].tolist() == [-1, -1, -1, vocab - 1] and prob[:4].tolist() == [0.0, 0.0, 0.0, 1.0]
    assert got[5] == 2 and prob[5] == 1.0 and got[6] == vocab - 1 and prob[6] == 0.5
    _check(t[4:], np.full(8, 0.3), top_p=np.full(8, 0.95))
    # parameters that mean no limit, or the largest alone
    t = t[7:]
    top = [int(np.argmax(r.double().numpy())) for r in t]
    n = len(t)
    for kw in ({"temperature": [0.0, -1.0, float("nan"), 1e-30, 0.0]}, {"top_k": [1] * n}, {"top_p": [0.0, -3.0, 1e-9, float("-inf"), 0.0]},
               {"min_p": [1.0, 5.0, float("inf"), 1.0, 2.0]}):
        got, prob = _run(t, np.full(n, 0.999), **kw)
        assert got.tolist() == top and np.all(prob == 1.0), kw
    plain = _run(t, np.full(n, 0.6))
    for kw in ({"top_k": [0, -5, 2 ** 31 - 1, vocab, vocab + 1]}, {"top_p": [1.0, 2.0, float("nan"), float("inf"), 1.0]},
               {"min_p": [0.0, -1.0, float("nan"), float("-inf"), 0.0]}):
        got = _run(t, np.full(n, 0.6), **kw)
        assert np.array_equal(got[0], plain[0]) and np.array_equal(got[1], plain[1]), kw
    # an infinite temperature: every allowed entry alike
    got, prob = _run(torch.zeros((1, vocab)) + t[:1].float(), [0.5], temperature=[float("inf")])
    assert got[0] == vocab // 2 and abs(prob[0] - 1.0 / vocab) < 1e-7 / vocab + 1e-12


@pytest.mark.parametrize("vocab", [100, 4672, 20001])
@pytest.mark.parametrize("temperature", [float("inf"), 3e38, 1e-38])
def test_temperatures_at_the_ends_with_filters(vocab, temperature):
    """The filters keep their beginning where all weights are alike, or all but one nothing."""
    rng = _rng(vocab, 8)
    t = _logits(rng, 10, vocab, "f32")
    t[5:, 7:] = float("-inf")                  # fewer allowed than top_k asks for
    u, heat = rng.random(10), np.full(10, temperature)
    for kw in ({}, {"top_k": np.full(10, 33)}, {"top_p": np.full(10, 0.6)}, {"top_k": np.full(10, 50), "top_p": np.full(10, 0.41), "min_p": np.full(10, 0.5)}):
        _check(t, u, temperature=heat, **kw)


@pytest.mark.parametrize("vocab", [3, 100, 4672, 20001])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("temperature", [1e37, 9e37, 3e38, float("inf")])
def test_logits_as_far_apart_as_they_can_be(vocab, dtype, temperature):
    """Distances past the largest fp32 number, at temperatures for which they still have a weight."""
    import torch
    rng = _rng(vocab, 9)
    t = torch.from_numpy(rng.uniform(-3.3e38, 3.3e38, (10, vocab)).astype(np.float32))
    t[:, 1] = 3.35e38
    t[5:, vocab // 2 + 1:] = float("-inf")
    t = t.to(torch.bfloat16) if dtype == "bf16" else t
    u, heat, k = rng.random(10), np.full(10, temperature), max(1, vocab // 3)
    for kw in ({}, {"top_k": np.full(10, k)}, {"top_p": rng.uniform(0.3, 0.999, 10)}, {"min_p": np.full(10, 0.013)},
               {"top_k": np.full(10, k), "top_p": np.full(10, 0.91371), "min_p": np.full(10, 0.0017)}):
        _check(t, u, temperature=heat, **kw)


def test_a_distance_past_fp32_keeps_its_weight():
    import torch
    big = 3e38
    t = torch.tensor([[big, -big], [big, -big]])
    got, prob = _run(t, [0.99, 0.5], temperature=[big, big], top_p=[0.95, 0.95])  # weights 1 and exp(-2)
    assert got.tolist() == [1, 0] and np.all(np.abs(prob - np.array([0.1192029, 0.8807971])) <= 1e-6)
    t = torch.tensor([[big, -big, -3.1e38], [-3.1e38, -big, big]])
    got, prob = _run(t, [1.0, 0.0], temperature=[1e38, 1e38], top_k=[2, 2])       # weights 1, exp(-6), and one that goes
    assert got.tolist() == [1, 1] and np.all(np.abs(prob - 0.002472623) <= 1e-6 * 0.002472623 + 1e-9)
    got, prob = _run(t, [1.0, 0.0], temperature=[1e38, 1e38], top_p=[0.99999, 0.99999])  # the last has 0.0022
    assert got.tolist() == [2, 0]


@pytest.mark.parametrize("vocab", [100, 4672, 131072, 1 << 24])
@pytest.mark.parametrize("filters", [{}, {"top_p": [1.0 - 2.0 ** -24]}])
def test_a_peak_over_a_flat_tail(vocab, filters):
    """Each weight is off by at most half a step 2^-S of the largest, S = 62 - ceil(log2 vocab) and at most 51: a tail of equal entries just
    below half a step has none, and one of one and a half steps counts as two."""
    import torch
    s = min(62 - int(np.ceil(np.log2(vocab))), 51)
    for tail, step in ((0.4999, 0), (1.5001, 2), (3.0, 3)):
        l = torch.full((1, vocab), float(np.float32(np.log(tail) - s * np.log(2.0))), device="cuda")
        l[0, vocab // 2] = 0.0
        got, prob = _run(l, [0.5], **filters)
        assert got[0] == vocab // 2
        true = 1.0 / (1.0 + (vocab - 1) * np.exp(float(l[0, 0])))
        # (half a step of fp32, and at most 2^-24 of the sum that top_p leaves out)
        assert abs(prob[0] - 1.0 / (1.0 + (vocab - 1) * step * 2.0 ** -s)) <= 2.0 ** -23
        assert abs(prob[0] - true) <= vocab * 2.0 ** -(s + 1) + 2.0 ** -23


def test_frequencies():
    """Equally spaced u give every entry its share, to one draw."""
    import torch
    rng = _rng(6)
    l = _logits(rng, 1, 100, "f32", 1.0)
    n = 4096
    got, _ = _run(l.expand(n, 100).contiguous(), (np.arange(n) + 0.5) / n, top_k=np.full(n, 20))
    at, w, _ = O.kept(l[0].double().numpy(), top_k=20)
    share = np.bincount(got, minlength=100) / n
    want = np.zeros(100)
    want[at] = w / w.sum()
    assert np.all(np.abs(share - want) <= 1.01 / n)


def test_equal_calls_give_equal_results():
    rng = _rng(7)
    t = _logits(rng, 64, 50000, "bf16")
    kw = dict(top_k=rng.integers(1, 2000, 64), top_p=rng.uniform(0.3, 1.0, 64), min_p=rng.uniform(0, 0.1, 64))
    u = rng.random(64)
    a = _run(t, u, **kw)
    for _ in range(3):
        b = _run(t, u, **kw)
        assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])
