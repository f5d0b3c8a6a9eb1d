"""topk, log_prob and entropy against the oracle (64 bits).

Indices have to be equal.  Tolerances of the others: with d = x - m, a term
exp(d) of the softmax's sum s is off by 2.5 |d| 2^-24 (the difference, the
product with log2 e, that constant) + 2^-23, and terms weigh exp(d), so |d| up
to 35 counts at 2^19 channels: 88 x 2^-24.  A sum passes at most 64 values of a
thread, 6 + 3 steps of the workgroup and 64 segments: 137 x 2^-24.  So s, and
log s absolutely, is off by 225 x 2^-24 < 2e-5 at the most, and t / s, which is
at most the entropy, by twice that of itself; the last steps round to 2^-23 of
their results."""
import numpy as np
import pytest

import oracle
from workloads import ACT_NONE, DTYPE_FP16, DTYPE_FP32, NetBuilder

from gpu_util import log, run_gpu

pytestmark = pytest.mark.gpu

LOWEST = np.finfo(np.float32).min


def questions(x, k, given=None, dtype=DTYPE_FP32, shape=None):
    """A graph that asks everything about the rows of x (rows, channels)."""
    b = NetBuilder()
    n, h, w = shape or (len(x), 1, 1)
    t = b.input(n, h, w, x.shape[1], 0, 1, dtype=dtype)
    b.ops[t]["data"] = x.astype(np.float16 if dtype == DTYPE_FP16 else np.float32).astype(np.float32).reshape(n, h, w, -1)
    top = b.topk(t, k)
    outs = [top, b.log_prob(t, top), b.entropy(t)]
    if given is not None:
        outs.append(b.log_prob(t, b.index_input(np.asarray(given).reshape(n, h, w, -1))))
    for o in outs:
        b.mark_output(o)
    return b.graph("questions"), outs


def same(got, ref, tol):
    got = got.astype(np.float64)
    # (differences of logits of 3e38 reach 6e38: -inf in the outputs' fp32, whose largest value is 3.4e38)
    ref = np.where(np.abs(ref) > np.finfo(np.float32).max, np.sign(ref) * np.inf, ref)
    for test in (np.isnan, np.isposinf, np.isneginf):
        np.testing.assert_array_equal(test(got), test(ref))
    f = np.isfinite(ref)
    off = np.abs(got[f] - ref[f]) - (tol[f] if np.ndim(tol) else tol)
    assert off.size == 0 or off.max() <= 0, f"worst by {off.max():.3e}"


def check(desc, outs, got):
    ref = oracle.run_graph(desc, keep=outs)
    ref = [ref[t].reshape(g.shape) for t, g in zip(outs, got)]
    assert got[0].dtype == np.int32
    np.testing.assert_array_equal(got[0], ref[0])
    with np.errstate(invalid="ignore"):
        for g, r in list(zip(got, ref))[1:]:
            same(g, r, 2e-5 * (1 + 2 * np.abs(r)) if g.shape[-1] == 1 and g is got[2] else 2e-5 + 2.0 ** -21 * np.abs(r))


def ask(x, k, given=None, dtype=DTYPE_FP32, shape=None, **kw):
    desc, outs = questions(x, k, given, dtype, shape)
    _, got, _ = run_gpu(desc, materialize_all=False, **kw)
    check(desc, outs, got)
    return got


CASES = [(1, 1, 1), (3, 2, 2), (2, 3, 1), (5, 7, 7), (1, 64, 64), (4, 63, 5), (9, 255, 5), (6, 256, 3), (7, 257, 64),
         (70, 300, 5), (64, 1000, 5), (33, 1001, 10), (3, 1200, 20), (300, 2049, 1), (3, 4099, 64), (2, 8193, 7),
         (260, 9000, 5), (257, 20011, 64), (2, 49999, 50), (1, 131077, 64), (1, 131077, 1), (600, 37, 3),
         (1, 1 << 19, 64), (257, 70001, 5)]


@pytest.mark.parametrize("rows,cols,k", CASES)
@pytest.mark.parametrize("dtype", [DTYPE_FP32, DTYPE_FP16])
def test_random_rows(rows, cols, k, dtype):
    rng = np.random.default_rng(cols)
    log(f"[case] {rows} x {cols}, k {k}, type {dtype}")
    ask(rng.standard_normal((rows, cols)) * 3, k, rng.integers(0, cols, (rows, 3)), dtype)


@pytest.mark.parametrize("rows,cols,k", [(3, 10, 4), (2, 1000, 20), (2, 2500, 64), (1, 40000, 64), (257, 33001, 30)])
def test_equal_values(rows, cols, k):
    # few different values, rows of one value, zeros of both signs, rising and falling rows
    rng = np.random.default_rng(rows)
    log(f"[case] ties {rows} x {cols}")
    ask(rng.integers(-2, 3, (rows, cols)).astype(float), k)
    ask(np.full((rows, cols), -7.5), k)
    ask(np.where(rng.random((rows, cols)) < 0.5, 0.0, -0.0), k)
    ask(np.broadcast_to(np.arange(cols) * 1e-3, (rows, cols)), k)
    ask(np.broadcast_to(-np.arange(cols) * 1e-3, (rows, cols)), k)
    # all but one or a few below a crowd of equals
    x = np.full((rows, cols), 1.0)
    x[:, cols // 2] = 2.0
    x[:, : cols // 3] = 0.0
    ask(x, k)


@pytest.mark.parametrize("cols,k", [(1, 1), (12, 5), (1000, 5), (5000, 64), (50000, 40)])
def test_masked_rows(cols, k):
    rng = np.random.default_rng(cols)
    x = rng.standard_normal((9, cols)) * 2
    x[0] = -np.inf                                  # no channel is left
    x[1, 1:] = -np.inf                              # one is
    x[2, rng.permutation(cols)[: cols // 2]] = -np.inf
    x[3] = LOWEST                                   # a mask of the type's lowest value: all equal
    x[4, 1:] = LOWEST
    x[5, rng.permutation(cols)[: max(1, cols - k + 1)]] = -np.inf
    x[6, : cols - 1] = -np.inf
    x[7, cols // 2] = np.nan
    x[8, cols // 2] = np.inf
    log(f"[case] masks, {cols} channels")
    got = ask(x, k, rng.integers(0, cols, (9, 4)))
    assert got[2][0] == 0 and (got[1][0] == -np.inf).all() and np.isnan(got[2][7:]).all()
    if cols > 1:
        ask(np.where(np.isin(np.arange(cols), [0, cols - 1]), x, -np.inf), k)
        ask(np.where(rng.random((9, cols)) < 0.3, np.nan, x), k)


def test_large_and_small_logits():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((6, 3000))
    x[0] *= 1e30
    x[1] *= 1e-30
    x[2] += 60000
    x[3] = np.float32(3e38) * np.sign(x[3])
    x[4] *= 1e-41                                   # denormal numbers
    log("[case] magnitudes")
    ask(x.astype(np.float32), 20, rng.integers(0, 3000, (6, 2)))


def test_indices_that_name_no_channel():
    log("[case] indices outside the channels")
    x = np.random.default_rng(2).standard_normal((3, 100))
    got = ask(x, 2, [[-1, 0, 99], [100, 5, 5], [2 ** 31 - 1, -2 ** 31, 7]])
    assert np.isnan(got[3]).tolist() == [[True, False, False], [True, False, False], [True, True, False]]


@pytest.mark.parametrize("shape,c", [((2, 5, 3), 21), ((1, 33, 33), 19), ((3, 1, 700), 150)])
def test_pixels(shape, c):
    rng = np.random.default_rng(c)
    n = int(np.prod(shape))
    log(f"[case] pixels {shape} x {c}")
    ask(rng.standard_normal((n, c)) * 2, 4, rng.integers(0, c, (n, 1)), shape=shape)


def test_sliced_logits_and_argmax_labels():
    # a convolution's output, held in 16 bits: asked about as the values it stores
    b = NetBuilder(seed=3)
    x = b.conv(b.input(2, 6, 5, 16, -1, 1), 21, 1, act=ACT_NONE)
    a = b.argmax(x)
    outs = [b.topk(x, 3), b.log_prob(x, a), b.entropy(x), x, a]
    for t in outs:
        b.mark_output(t)
    desc = b.graph("sliced")
    log("[case] sliced logits")
    plan, got, _ = run_gpu(desc, materialize_all=False)
    z = got[3].astype(np.float64)
    np.testing.assert_array_equal(got[0], oracle.topk(z, 3))
    np.testing.assert_array_equal(got[4], got[0][..., 0])
    same(got[1], oracle.log_prob(z, got[4][..., None]), 2e-5)
    same(got[2], oracle.entropy(z), 2e-4)
    _, again, _ = run_gpu(desc, materialize_all=True)
    for p, q in zip(got, again):
        np.testing.assert_array_equal(p, q)


@pytest.mark.parametrize("ask_for", ["topk", "entropy", "log_prob"])
@pytest.mark.parametrize("rows,cols", [(3, 700), (1, 30000)])
def test_one_question_alone(ask_for, rows, cols):
    rng = np.random.default_rng(rows)
    b = NetBuilder()
    t = b.input(rows, 1, 1, cols, -4, 4, dtype=DTYPE_FP32)
    o = b.topk(t, 6) if ask_for == "topk" else b.entropy(t) if ask_for == "entropy" else \
        b.log_prob(t, b.index_input(rng.integers(0, cols, (rows, 1, 1, 700))))
    b.mark_output(o)
    desc = b.graph(ask_for)
    log(f"[case] {ask_for} alone, {rows} x {cols}")
    plan, got, _ = run_gpu(desc, materialize_all=False)
    assert [n["kind"] for n in plan.nodes()] == [ask_for]
    ref = oracle.run_graph(desc, keep=[o])[o].reshape(got[0].shape)
    if ask_for == "topk":
        np.testing.assert_array_equal(got[0], ref)
    else:
        same(got[0], ref, 2e-5 + 4e-5 * np.abs(ref))


@pytest.mark.parametrize("rows,cols,k", [(1, 50000, 20), (40, 1000, 5), (3, 70000, 64)])
def test_repeated_captured_and_without_allocation(rows, cols, k):
    import torch
    from paper_1907_01989_amd import _binding as B, engine
    rng = np.random.default_rng(5)
    desc, outs = questions(rng.standard_normal((rows, cols)), k, rng.integers(0, cols, (rows, 2)))
    log(f"[case] {rows} x {cols} repeated, captured, without allocation")
    plan = engine.Plan(desc)
    xs = plan.input_tensors()
    first = [o.clone() for o in plan.run(xs)]
    torch.cuda.synchronize()
    check(desc, outs, [o.cpu().numpy() for o in first])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = plan.run(xs)
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(first, again))
    out = plan.capture(xs)
    for rep in range(4):
        for o in out:
            o.fill_(-1)
        plan.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(first, out)), rep
        xs[0].neg_()
        plan.run(xs)
        xs[0].neg_()
        torch.cuda.synchronize()
    for rep in range(2):
        got = plan.alloc_outputs()
        B.mgi_plan_run_noalloc(plan.handle, [x.data_ptr() for x in xs], [o.data_ptr() for o in got],
                               torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(first, got)), rep


def test_inputs_off_16_bytes():
    import torch
    from paper_1907_01989_amd import engine
    for dtype, tt in ((DTYPE_FP32, torch.float32), (DTYPE_FP16, torch.float16)):
        x = np.random.default_rng(6).standard_normal((5, 1003)) * 2
        desc, outs = questions(x, 9, dtype=dtype)
        log(f"[case] logits off 16 bytes, type {dtype}")
        plan = engine.Plan(desc)
        xs = plan.input_tensors()
        room = torch.zeros(xs[0].numel() + 1, dtype=tt, device="cuda:0")
        room[1:] = xs[0].reshape(-1)
        got = plan.run([room[1:].view(xs[0].shape)])
        torch.cuda.synchronize()
        check(desc, outs, [o.cpu().numpy() for o in got])


def test_outputs_over_inputs_are_refused():
    import torch
    from paper_1907_01989_amd import _binding as B, engine
    b = NetBuilder()
    t = b.input(4, 1, 1, 64, -1, 1, dtype=DTYPE_FP32)
    ix = b.index_input(np.zeros((4, 1, 1, 64)))
    b.mark_output(b.log_prob(t, ix))
    plan = engine.Plan(b.graph("overlap"))
    xs = plan.input_tensors()
    log("[case] outputs over inputs")
    for x in xs:
        with pytest.raises(B.MgiError) as e:
            plan.run(xs, [x.view(torch.float32).view(4, 64)])
        assert e.value.status == 1 and "overlaps" in str(e.value)
    plan.run(xs)
    torch.cuda.synchronize()


def test_a_head_with_its_answers():
    # features -> 4-bit layer -> answers, as a program uses them, with the logits for the check
    b = NetBuilder(seed=7)
    x = b.gap(b.conv(b.input(12, 7, 7, 64, -1, 1), 320, 1))
    z = b.fc_int4(x, 1000, 64, True)
    top = b.topk(z, 5)
    given = b.index_input(np.random.default_rng(7).integers(0, 1000, (12, 1, 1, 1)))
    outs = [z, top, b.log_prob(z, top), b.log_prob(z, given), b.entropy(z)]
    for t in outs:
        b.mark_output(t)
    desc = b.graph("head")
    log("[case] a 4-bit head with its answers")
    plan, got, _ = run_gpu(desc, materialize_all=False)
    assert [n["kind"] for n in plan.nodes()][-2:] == ["fc_int4", "answers"]
    logits = got[0].astype(np.float64)
    ref = oracle.run_graph(desc, keep=[z])[z].reshape(logits.shape)
    assert (np.linalg.norm(logits - ref, axis=1) <= 1e-2 * np.linalg.norm(ref, axis=1)).all()
    np.testing.assert_array_equal(got[1], oracle.topk(logits, 5))
    same(got[2], oracle.log_prob(logits, got[1]), 2e-5)
    same(got[3], oracle.log_prob(logits, np.asarray(desc["ops"][given]["data"]).reshape(12, 1)), 2e-5)
    same(got[4], oracle.entropy(logits), 3e-4)
    for kw in ({"fuse": False}, {"materialize_all": True}):
        _, again, _ = run_gpu(desc, **{"materialize_all": False, **kw})
        np.testing.assert_array_equal(got[1], again[1])


def test_writes_stay_inside_the_buffers():
    from test_gpu_guards import check_guards, guarded_plan
    rng = np.random.default_rng(8)
    for rows, cols, k in ((1, 40000, 64), (5, 1000, 5), (300, 10, 10)):
        desc, _ = questions(rng.standard_normal((rows, cols)), k, rng.integers(0, cols, (rows, 3)))
        log(f"[case] guards {rows} x {cols}")
        plan, outs, raw, ws, lead = guarded_plan(desc)
        xs = plan.input_tensors()
        for _ in range(2):
            plan.run(xs, outs)
        check_guards(plan, raw, ws, lead, f"{rows} x {cols}")
    b = NetBuilder(seed=8)
    b.mark_output(b.fc_int4(b.input(19, 1, 1, 1000, -1, 1), 77, 96, True))
    plan, outs, raw, ws, lead = guarded_plan(b.graph("fc"))
    plan.run(plan.input_tensors(), outs)
    check_guards(plan, raw, ws, lead, "fc_int4")


@pytest.mark.parametrize("k", [1, 13, 41, 64])
def test_crowds_in_a_later_stretch(k):
    # rows that a workgroup reads in rounds: a later one holds more equal values,
    # larger than all before them, than there is room for
    x = np.random.default_rng(k).standard_normal((300, 70001)) * 0.1
    x[:, 20000:50000] = 2.0
    x[1, 40000:] = 3.0
    x[2, 60000:60020] = 2.0
    x[3:, 14008:] = 2.0                             # (from the second of five stretches on)
    log(f"[case] crowds, k {k}")
    ask(x, k)


def test_two_captured_heads_replayed_on_two_streams_and_tuned():
    # plans of the same description share nothing but their inputs
    import torch
    from paper_1907_01989_amd import engine
    b = NetBuilder(seed=11)
    x = b.input(3, 1, 1, 203, -1, 1, dtype=DTYPE_FP32)
    z = b.fc_int4(x, 30000, 96, True)
    top = b.topk(z, 33)
    for t in (top, b.log_prob(z, top), b.entropy(z)):
        b.mark_output(t)
    desc = b.graph("twice")
    log("[case] two captured heads")
    plans = [engine.Plan(desc) for _ in range(2)]
    xs = plans[0].input_tensors()
    want = [o.clone() for o in plans[0].run(xs)]
    plans[1].autotune(xs)
    outs = [p.capture(xs) for p in plans]
    streams = [torch.cuda.Stream() for _ in plans]
    torch.cuda.synchronize()
    for rep in range(6):
        for o in outs[0] + outs[1]:
            o.fill_(-1)
        torch.cuda.synchronize()
        for p, s in zip(plans, streams):
            p.replay(s)
        torch.cuda.synchronize()
        for got in outs:
            assert all(torch.equal(a, w) for a, w in zip(got, want)), rep
        assert torch.equal(plans[rep % 2].run(xs)[0], want[0])
        torch.cuda.synchronize()


@pytest.mark.parametrize("cols", [1, 3, 57, 64])
def test_every_channel_is_asked_for(cols):
    rng = np.random.default_rng(cols)
    x = rng.standard_normal((70, cols))
    x[3] = np.nan
    x[5, cols // 2] = np.inf
    x[7, : cols // 2] = -np.inf
    log(f"[case] all {cols} channels")
    ask(x, cols, rng.integers(-2, cols + 2, (70, 700)))


def test_more_rows_than_one_grid_dimension_has_threads_for():
    # 2^26 rows of one wave each: 2^32 threads
    import torch
    from paper_1907_01989_amd import engine
    rows = 2 ** 26 + 5
    desc = {"ops": [{"op": "input", "shape": (rows, 1, 1, 2), "dtype": DTYPE_FP16}, {"op": "topk", "in": 0, "k": 1},
                    {"op": "log_prob", "in": 0, "index": 1}, {"op": "entropy", "in": 0}], "outputs": [1, 2, 3]}
    log(f"[case] {rows} x 2")
    plan = engine.Plan(desc)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.randn((rows, 1, 1, 2), generator=g, device="cuda", dtype=torch.float16)
    top, lp, h = plan.run([x], [o.fill_(-7) for o in plan.alloc_outputs()])
    torch.cuda.synchronize()
    for r in range(0, rows, 2 ** 24):
        z = x[r:r + 2 ** 24].reshape(-1, 2).double()
        assert torch.equal(top[r:r + 2 ** 24, 0], (z[:, 1] > z[:, 0]).int()), r
        p = torch.log_softmax(z, 1)
        assert ((lp[r:r + 2 ** 24, 0] - p.amax(1)).abs() <= 2e-5).all(), r
        assert ((h[r:r + 2 ** 24, 0] + (p.exp() * p).sum(1)).abs() <= 5e-5).all(), r


def test_a_launch_of_too_many_threads_is_an_error():
    # (a softmax takes a wave to a row too; only the count of threads is wrong, no access is)
    import torch
    from paper_1907_01989_amd import _binding as B, engine
    rows = 2 ** 26 + 5
    desc = {"ops": [{"op": "input", "shape": (rows, 1, 1, 2), "dtype": DTYPE_FP16}, {"op": "softmax", "in": 0}], "outputs": [1]}
    log(f"[case] softmax of {rows} x 2")
    plan = engine.Plan(desc)
    x = torch.zeros((rows, 1, 1, 2), device="cuda", dtype=torch.float16)
    with pytest.raises(B.MgiError, match="softmax.*InvalidConfiguration"):
        plan.run([x])
    torch.cuda.synchronize()
