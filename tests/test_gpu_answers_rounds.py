"""topk, log_prob and entropy of rows that a workgroup reads in several rounds,
alone or as one of a row's segments, against the oracle (64 bits).

Tolerance: a term of the softmax's sum is off by 88 x 2^-24 as test_gpu_answers
derives (the exponents' differences add up to the term's own, however many rounds
carry it on).  A thread adds up to 32 values, its wave's lanes in 6 steps, then
every round the 8 waves one after another and, where the maximum grew, a
rescaling of what was there: an exponential of 2^-23 and a product.  The join adds
6 steps and one rescaling.  32 rounds: 88 + 32 + 6 + 32 (8 + 3) + 9 = 487 x 2^-24
< 3e-5 of s, and so of log s absolutely, and of t / s, which is at most the
entropy, twice that; the last steps round to 2^-23 of their results."""
import numpy as np
import pytest

import oracle
from workloads import DTYPE_FP16, DTYPE_FP32

from gpu_util import log, run_gpu
from test_gpu_answers import questions, same

pytestmark = pytest.mark.gpu


def check_rows(x, k, given, rows, dtype):
    """All questions about x, compared for the given rows."""
    desc, _ = questions(x, k, given, dtype)
    _, (top, lp, h, lg), _ = run_gpu(desc, materialize_all=False)
    z = np.asarray(desc["ops"][0]["data"]).reshape(x.shape)[rows].astype(np.float64)
    ref = oracle.topk(z, k)
    np.testing.assert_array_equal(top[rows], ref)
    with np.errstate(invalid="ignore"):
        for got, r in ((lp[rows], oracle.log_prob(z, ref)), (lg[rows], oracle.log_prob(z, np.asarray(given)[rows]))):
            same(got, r, 3e-5 + 2.0 ** -21 * np.abs(r))
        r = oracle.entropy(z)
        same(h[rows].reshape(r.shape), r, 3e-5 * (1 + 2 * np.abs(r)))


def special_rows(x, k, rng):
    """Rows whose best, masks or infinities lie in one stretch or another."""
    rows, cols = x.shape
    x[0] = -np.inf
    x[1, : cols - 1] = -np.inf                      # one channel is left, the last
    x[2, rng.random(cols) < 0.9] = -np.inf
    x[3] = np.arange(cols) * 1e-3                   # every round has larger ones
    x[4] = -np.arange(cols) * 1e-3
    x[5] = 1.5                                      # all equal
    x[6, cols // 2:] = 9.0                          # a crowd above all before it
    x[7, -1:] = np.nan
    x[8, cols - 3] = np.inf
    x[9] = np.finfo(np.float16).min
    x[9, cols - 2] = -60000.0
    x[10, : cols // 3] = -np.inf                    # the first rounds have nothing
    x[11, : k // 2] = 8.0                           # half of the best at the start, more of them at the end
    x[11, -k:] = 8.0
    return x


@pytest.mark.parametrize("rows,cols,k,dtype", [
    (85, 191584, 5, DTYPE_FP32),                    # three segments of four rounds
    (100, 100003, 20, DTYPE_FP16), (100, 100003, 64, DTYPE_FP32), (64, 150001, 1, DTYPE_FP32),
    (20, 1 << 19, 64, DTYPE_FP32),                  # twelve segments of three
    (128, 70001, 33, DTYPE_FP16),                   # two of three
    (129, 262145, 7, DTYPE_FP32),                   # one of 17
])
def test_rounds(rows, cols, k, dtype):
    rng = np.random.default_rng(cols + k)
    log(f"[case] {rows} x {cols}, k {k}, type {dtype}")
    x = special_rows(rng.standard_normal((rows, cols), dtype=np.float32) * 3, k, rng)
    given = rng.integers(0, cols, (rows, 3))
    given[:, 0] = cols - 1
    check_rows(x, k, given, np.r_[0:min(rows, 20), rows - 1], dtype)


def test_the_most_rounds():
    # 32 of them: the longest rows, more of them than half of the compute units
    rng = np.random.default_rng(32)
    rows, cols, k = 129, 1 << 19, 40
    log(f"[case] {rows} x {cols}, k {k}")
    x = special_rows(rng.standard_normal((rows, cols), dtype=np.float32) * 3, k, rng).astype(np.float16)
    check_rows(x, k, rng.integers(0, cols, (rows, 2)), np.r_[0:13, rows - 1], DTYPE_FP16)


@pytest.mark.parametrize("cols", [4097, 6001, 8192])
@pytest.mark.parametrize("k", [1, 16])
def test_rows_of_four_waves(cols, k):
    rng = np.random.default_rng(cols)
    log(f"[case] 300 x {cols}, k {k}")
    x = special_rows(rng.standard_normal((300, cols), dtype=np.float32) * 3, k, rng)
    for dtype in (DTYPE_FP32, DTYPE_FP16):
        check_rows(x, k, rng.integers(0, cols, (300, 2)), np.arange(300), dtype)


@pytest.mark.parametrize("rows,cols", [(85, 191584), (20, 300000)])
def test_runs_repeat_and_replay(rows, cols):
    import torch
    from paper_1907_01989_amd import engine
    rng = np.random.default_rng(rows)
    x = special_rows(rng.standard_normal((rows, cols), dtype=np.float32), 20, rng)
    desc, _ = questions(x, 20, rng.integers(0, cols, (rows, 2)))
    log(f"[case] {rows} x {cols} repeated and captured")
    plan = engine.Plan(desc)
    xs = plan.input_tensors()
    bits = lambda ts: [t.view(torch.int32).clone() for t in ts]  # noqa: E731
    first = bits(plan.run(xs))
    out = plan.capture(xs)
    for rep in range(4):
        for o in out:
            o.fill_(-1)
        plan.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(first, bits(out))), rep
        xs[0].neg_()
        plan.run(xs)
        xs[0].neg_()
        torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(first, bits(plan.run(xs))))
