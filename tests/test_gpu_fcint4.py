"""Fully connected layer with 4-bit weights against the oracle (64 bits).

The scales of these graphs are exact in both storage types and the inputs are
too, so the only roundings are those of fp32 sums.  At most ``K / 32`` partial
sums follow one another (matrix instructions of 32 products, group sums), then
those of the waves and workgroups that share K, the bias and the product with a
power of two; an instruction adds its 32 products in an order of its own.  With
a whole step of 2^-23 for each (half a step if every one rounds to nearest):
    |error| <= (K / 32 + 32 + 32) 2^-23 sum |w x|.
"""
import numpy as np
import pytest

import oracle
import workloads
from workloads import ACT_NONE, ACT_RELU, ACT_RELU6, DTYPE_FP16, DTYPE_FP32, NetBuilder

from gpu_util import log, run_gpu

pytestmark = pytest.mark.gpu


def layer(n, cin, cout, group=32, zeros=False, dtype=DTYPE_FP16, act=ACT_NONE, seed=0):
    b = NetBuilder(seed=seed + n + cin + cout + group)
    t = b.fc_int4(b.input(n, 1, 1, cin, -2, 2, dtype=dtype), cout, group, zeros)
    if act != ACT_NONE:
        t = b.activation(t, act)
    b.mark_output(t)
    return b.graph(f"fc_int4_{n}x{cin}x{cout}_g{group}{'z' if zeros else ''}"), t


def bound(desc):
    """The allowed error of the layer's outputs, (n, cout)."""
    op = next(o for o in desc["ops"] if o["op"] == "fc_int4")
    x = np.abs(np.asarray(desc["ops"][op["in"]]["data"], np.float64)).reshape(-1, desc["ops"][op["in"]]["shape"][3])
    eye = np.eye(x.shape[1]).reshape(x.shape[1], 1, 1, -1)
    w = np.abs(oracle.fc_int4(eye, op["q"], op["scales"], op["zeros"], op["group"], None)).reshape(x.shape[1], -1)
    b = 0.0 if op["b"] is None else np.abs(op["b"])
    return (x.shape[1] / 32 + 64) * 2.0 ** -23 * (x @ w + b)


def check(desc, t, got):
    ref = oracle.run_graph(desc, keep=[t])[t].reshape(got.shape)
    off = np.abs(got.astype(np.float64) - ref) - bound(desc)
    assert np.isfinite(got).all() and (off <= 0).all(), \
        f"{int((off > 0).sum())} of {got.size} out of bound, worst by {off.max():.3e}"


CASES = [
    # n, cin, cout, group, zeros
    (1, 1, 1, 32, True), (1, 31, 17, 32, False), (3, 33, 16, 32, True), (2, 127, 5, 64, True),
    (1, 129, 40, 128, True), (5, 130, 33, 64, False), (16, 256, 64, 32, True), (17, 257, 50, 96, True),
    (31, 500, 31, 160, True), (33, 512, 100, 128, False), (1, 1280, 1000, 32, False), (64, 1024, 1000, 32, True),
    (65, 640, 48, 64, True), (130, 320, 24, 256, True), (1, 4096, 1000, 128, True), (2, 2001, 503, 96, True),
    (1, 96, 9000, 32, True), (16, 4128, 333, 1024, True), (257, 160, 272, 32, False), (4, 8192, 64, 64, False),
]


@pytest.mark.parametrize("n,cin,cout,group,zeros", CASES)
def test_layer(n, cin, cout, group, zeros):
    desc, t = layer(n, cin, cout, group, zeros)
    log(f"[case] {desc['name']}")
    _, outs, _ = run_gpu(desc, materialize_all=False)
    check(desc, t, outs[0])


@pytest.mark.parametrize("n,cin,cout,group,zeros", CASES[::3])
def test_layer_bf16_from_fp32(n, cin, cout, group, zeros):
    desc, t = layer(n, cin, cout, group, zeros, dtype=DTYPE_FP32, seed=1)
    desc = workloads.as_bf16_graph(desc)
    log(f"[case] {desc['name']}")
    _, outs, _ = run_gpu(desc, materialize_all=False, dtype=1)
    check(desc, t, outs[0])


@pytest.mark.parametrize("n,cin,cout,group,zeros", CASES[1::4])
def test_layer_fp16_from_fp32_and_materialised(n, cin, cout, group, zeros):
    desc, t = layer(n, cin, cout, group, zeros, dtype=DTYPE_FP32, seed=2)
    log(f"[case] {desc['name']}")
    _, a, _ = run_gpu(desc, materialize_all=False)
    check(desc, t, a[0])
    _, b, nodes = run_gpu(desc, materialize_all=True, fuse=False)
    np.testing.assert_array_equal(a[0], b[0])
    np.testing.assert_array_equal(nodes[t].reshape(a[0].shape), a[0])


@pytest.mark.parametrize("act", [ACT_RELU, ACT_RELU6])
def test_fused_activation_and_no_bias(act):
    desc, t = layer(6, 200, 70, act=act)
    desc["ops"][1]["b"] = None
    log(f"[case] {desc['name']} act {act}")
    plan, outs, _ = run_gpu(desc, materialize_all=False)
    assert [n["kind"] for n in plan.nodes()][-1] == "fc_int4"
    desc["ops"][1]["b"] = np.zeros(70)
    check(desc, t, outs[0])


@pytest.mark.parametrize("dtype", [0, 1])
def test_scales_far_from_one(dtype):
    # scales of 2^-60 .. 2^60 from channel to channel, zeros and both signs among them
    desc, t = layer(3, 160, 64, 32, True)
    if dtype == 1:
        desc = workloads.as_bf16_graph(desc)
    op = desc["ops"][1]
    e = np.linspace(-60, 60, 64).round()[:, None]
    op["scales"] = (op["scales"] * 2.0 ** e).astype(np.float32)
    op["scales"][5] = 0
    op["scales"][7:20] *= -1
    op["scales"][:, 2] = 0
    op["b"] = np.zeros(64)
    log(f"[case] scales 2^-60 .. 2^60, storage type {dtype}")
    _, outs, _ = run_gpu(desc, materialize_all=False, dtype=dtype)
    check(desc, t, outs[0])
    assert (outs[0][:, 5] == 0).all()


@pytest.mark.parametrize("dtype", [0, 1])
def test_scales_are_rounded_to_the_storage_type(dtype):
    # half a step: 2^-11 (fp16), 2^-8 (bf16), of each group's part
    desc, t = layer(4, 256, 48, 64, True)
    if dtype == 1:
        desc = workloads.as_bf16_graph(desc)
    rng = np.random.default_rng(3)
    op = desc["ops"][1]
    op["scales"] = (op["scales"] * (1 + rng.random(op["scales"].shape) * 0.01)).astype(np.float32)
    log(f"[case] scales of 24 bits, storage type {dtype}")
    _, outs, _ = run_gpu(desc, materialize_all=False, dtype=dtype)
    ref = oracle.run_graph(desc, keep=[t])[t].reshape(outs[0].shape)
    full = bound(desc)
    step = full / ((256 / 32 + 64) * 2.0 ** -23) * 2.0 ** (-8 if dtype else -11)
    assert (np.abs(outs[0] - ref) <= full + step).all()


@pytest.mark.parametrize("dtype", [0, 1])
def test_infinite_and_nan_features(dtype):
    # one infinity beside the end of a ragged K: its class rows are infinite, with
    # the weight's sign, or NaN where the weight is zero; other rows are untouched
    desc, t = layer(18, 203, 40, 32, True, dtype=DTYPE_FP32)
    if dtype == 1:
        desc = workloads.as_bf16_graph(desc)
    x = desc["ops"][0]["data"]
    x[3, 0, 0, 202] = np.inf
    x[5, 0, 0, 0] = -np.inf
    x[17, 0, 0, 100] = np.nan
    log(f"[case] infinities, storage type {dtype}")
    _, outs, _ = run_gpu(desc, materialize_all=False, dtype=dtype)
    with np.errstate(invalid="ignore"):
        ref = oracle.run_graph(desc, keep=[t])[t].reshape(outs[0].shape)
    np.testing.assert_array_equal(np.isnan(outs[0]), np.isnan(ref))
    np.testing.assert_array_equal(np.isinf(outs[0]), np.isinf(ref))
    inf = np.isinf(ref)
    np.testing.assert_array_equal(outs[0][inf], ref[inf])
    assert inf[3].any() and inf[5].any() and np.isnan(ref[17]).all() and np.isfinite(outs[0][4]).all()


def test_largest_products_do_not_overflow():
    # 65504 times 15 times 512 channels is far inside fp32
    desc, t = layer(2, 512, 32, 64, True)
    desc["ops"][0]["data"][:] = 65504.0
    op = desc["ops"][1]
    op["q"][:] = 0xFF
    op["zeros"][:] = 0
    op["scales"][:] = 1.0
    log("[case] largest products")
    _, outs, _ = run_gpu(desc, materialize_all=False)
    np.testing.assert_allclose(outs[0], 65504.0 * 15 * 512, rtol=1e-6)


def test_features_from_a_network():
    # pooled features of a small network, with a last channel slice that is not full
    b = NetBuilder(seed=9)
    x = b.gap(b.conv(b.input(5, 9, 9, 8, -1, 1), 44, 1))
    t = b.fc_int4(x, 30, 32, True)
    b.mark_output(t)
    desc = b.graph("pooled")
    log("[case] pooled features")
    plan, outs, nodes = run_gpu(desc, materialize_all=True, fuse_pool=False)
    pooled = nodes[x].astype(np.float64)
    op = desc["ops"][t]
    ref = oracle.fc_int4(pooled, op["q"], op["scales"], op["zeros"], 32, op["b"]).reshape(outs[0].shape)
    w = np.abs(oracle.fc_int4(np.eye(44).reshape(44, 1, 1, 44), op["q"], op["scales"], op["zeros"], 32, None)).reshape(44, -1)
    assert (np.abs(outs[0] - ref) <= (44 / 32 + 64) * 2.0 ** -23 * (np.abs(pooled.reshape(5, -1)) @ w + np.abs(op["b"]))).all()


@pytest.mark.parametrize("n,cin,cout", [(1, 4096, 96), (20, 1000, 48)])
def test_runs_repeat_and_replay(n, cin, cout):
    import torch
    from paper_1907_01989_amd import engine
    desc, t = layer(n, cin, cout, 64, True)
    log(f"[case] {desc['name']} repeated and captured")
    plan = engine.Plan(desc)
    xs = plan.input_tensors()
    first = plan.run(xs)[0].clone()
    check(desc, t, first.cpu().numpy())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = plan.run(xs)[0]
    torch.cuda.synchronize()
    assert torch.equal(first, again)
    out = plan.capture(xs)[0]
    for rep in range(4):
        out.fill_(-1)
        plan.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first), rep
        xs[0].neg_()
        eager = plan.run(xs)[0]
        xs[0].neg_()
        torch.cuda.synchronize()
        assert not torch.equal(eager, first)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("src", [DTYPE_FP16, DTYPE_FP32])
@pytest.mark.parametrize("n,cin,cout", [(1, 7, 5), (1, 8, 20), (16, 9, 4200), (3, 15, 16), (5, 127, 4100), (9, 129, 33),
                                        (13, 250, 4500), (16, 1027, 16), (7, 2001, 5003), (2, 1289, 16500)])
def test_rows_read_as_they_are(n, cin, cout, src, dtype):
    # few rows of fp32 or of odd fp16 length are converted by the layer itself:
    # the same values as through a converted copy, also at the rows' ends
    import torch
    from paper_1907_01989_amd import engine
    desc, t = layer(n, cin, cout, 64, True, dtype=src, seed=4)
    if dtype == 1:
        desc = workloads.as_bf16_graph(desc)
    log(f"[case] {desc['name']} inputs {src}, storage type {dtype}")
    plan = engine.Plan(desc, dtype=dtype)
    (x,) = plan.input_tensors()
    got = plan.run([x])[0].clone()
    check(desc, t, got.cpu().numpy())
    # an array off 16 bytes, and one that the output overlaps, are converted first
    apart = torch.empty(x.numel() + 4, dtype=x.dtype, device=x.device)
    off = apart[1:1 + x.numel()].view(x.shape)
    off.copy_(x)
    assert torch.equal(plan.run([off])[0], got)
    room = torch.empty(max(x.numel() * x.element_size(), got.numel() * 4), dtype=torch.uint8, device=x.device)
    same = room[:x.numel() * x.element_size()].view(x.dtype).view(x.shape)
    same.copy_(x)
    over = room[:got.numel() * 4].view(torch.float32).view(got.shape)
    plan.run([same], [over])
    assert torch.equal(over, got)
    x[n - 1, ..., cin - 1] = float("inf")
    last = plan.run([x])[0]
    assert torch.equal(last[:n - 1], got[:n - 1])
    op = desc["ops"][1]
    codes = op["q"][:, (cin - 1) // 2] >> (4 * ((cin - 1) % 2)) & 15
    w = torch.as_tensor((codes.astype(np.float64) - op["zeros"][:, -1]) * op["scales"][:, -1], device=x.device)
    row = last[n - 1].reshape(-1).double()
    assert torch.isnan(row[w == 0]).all() and torch.equal(row[w != 0], torch.sign(w[w != 0]) * float("inf"))


@pytest.mark.parametrize("src,dtype", [(DTYPE_FP16, 0), (DTYPE_FP32, 0), (DTYPE_FP32, 1)])
@pytest.mark.parametrize("n,cin,cout,group,zeros", [(1000, 1030, 1030, 64, True), (1030, 1024, 1000, 128, False),
                                                    (2050, 1288, 500, 96, True), (70, 1152, 8200, 32, False),
                                                    (321, 2000, 3000, 256, True)])
def test_many_rows(n, cin, cout, group, zeros, src, dtype):
    import torch
    from paper_1907_01989_amd import engine
    desc, t = layer(n, cin, cout, group, zeros, dtype=src, seed=5)
    if dtype == 1:
        desc = workloads.as_bf16_graph(desc)
    log(f"[case] {desc['name']} inputs {src}, storage type {dtype}")
    plan = engine.Plan(desc, dtype=dtype)
    xs = plan.input_tensors()
    got = plan.run(xs)[0].clone()
    check(desc, t, got.cpu().numpy())
    for _ in range(3):
        assert torch.equal(plan.run(xs)[0], got)


@pytest.mark.parametrize("dtype", [0, 1])
def test_a_group_far_longer_than_the_rows(dtype):
    # one scale per channel, whatever multiple of 32 the group is
    desc, t = layer(3, 100, 40, 128, True, seed=6)
    if dtype == 1:
        desc = workloads.as_bf16_graph(desc)
    desc["ops"][1]["group"] = 2 ** 31 - 32
    log(f"[case] group 2^31 - 32, storage type {dtype}")
    _, outs, _ = run_gpu(desc, materialize_all=False, dtype=dtype)
    check(desc, t, outs[0])


@pytest.mark.parametrize("n,cout,group", [(3, 40, 32), (20, 50, 64), (9, 4200, 128)])
@pytest.mark.parametrize("dtype", [0, 1])
def test_scales_far_apart_within_a_channel(dtype, n, cout, group):
    # groups of one channel with scales 2^24 apart, and features that make up for
    # it: every group counts in the sum.  Scales of 24 bits, so each group's part
    # is off by half a step of the storage type (2^-11, 2^-8).
    desc, t = layer(n, 4 * group, cout, group, True, seed=7)
    if dtype == 1:
        desc = workloads.as_bf16_graph(desc)
    rng = np.random.default_rng(cout)
    op, x = desc["ops"][1], desc["ops"][0]["data"]
    order = rng.permuted(np.tile(np.arange(4), (cout, 1)), axis=1)
    order[::2] = np.arange(4)
    op["scales"] = (op["scales"] / 16 * (1 + rng.random((cout, 4)) * 0.01) * 2.0 ** (-8 * order)).astype(np.float32)
    x[:] = (x.reshape(n, 4, group) * 2.0 ** (8 * np.arange(4) - 12)[:, None]).reshape(x.shape)
    x[:] = x.astype(np.float16)
    op["b"] = np.zeros(cout)
    log(f"[case] {desc['name']}, scales 2^24 apart, storage type {dtype}")
    _, outs, _ = run_gpu(desc, materialize_all=False, dtype=dtype)
    ref = oracle.run_graph(desc, keep=[t])[t].reshape(outs[0].shape)
    full = bound(desc)
    step = full / ((4 * group / 32 + 64) * 2.0 ** -23) * 2.0 ** (-8 if dtype else -11)
    assert (np.abs(outs[0] - ref) <= full + step).all()


@pytest.mark.parametrize("n,cin,cout,group", [(3, 2048, 40, 128), (20, 2048, 50, 64), (9, 2000, 4200, 32),
                                              (700, 2048, 1500, 128)])
def test_large_bf16_features(n, cin, cout, group):
    # features up to 2^116 of one sign and the largest codes: what one scale's
    # stretch of at most 128 inputs sums to stays below 128 * 15 * 2^116 < 2^127,
    # and the scales bring that back before more is added
    desc, t = layer(n, cin, cout, group, True, dtype=DTYPE_FP32, seed=8)
    desc = workloads.as_bf16_graph(desc)
    op, x = desc["ops"][1], desc["ops"][0]["data"]
    x[:] = workloads.bf16_round(2.0 ** 115 * (1 + np.abs(x) / 2.1))
    op["q"][:] = 0xFF
    op["zeros"][:] = 0
    op["scales"] = (op["scales"] * 2.0 ** -30).astype(np.float32)
    log(f"[case] {desc['name']}, features of 2^115")
    _, outs, _ = run_gpu(desc, materialize_all=False, dtype=1)
    check(desc, t, outs[0])


def test_scales_at_the_ends_of_the_range():
    # the largest floats do not round to infinity, the smallest not to zero
    for dtype in (0, 1):
        desc, t = layer(2, 160, 64, 32, True, seed=9)
        if dtype == 1:
            desc = workloads.as_bf16_graph(desc)
        op = desc["ops"][1]
        op["b"] = np.zeros(64)
        big = np.float32(np.finfo(np.float32).max) / 2 ** 12
        small = np.float32(2.0 ** -120)
        op["scales"][:32], op["scales"][32:] = big, small
        desc["ops"][0]["data"][:] *= 2.0 ** -5
        log(f"[case] scales of 8e34 and 2^-120, storage type {dtype}")
        _, outs, _ = run_gpu(desc, materialize_all=False, dtype=dtype)
        ref = oracle.run_graph(desc, keep=[t])[t].reshape(outs[0].shape)
        full = bound(desc)
        # (half a step of each scale; results below the normal numbers in steps of 2^-149)
        step = full / ((160 / 32 + 64) * 2.0 ** -23) * 2.0 ** (-8 if dtype else -11) + 2.0 ** -149
        assert np.isfinite(outs[0]).all() and (np.abs(outs[0] - ref) <= full + step).all()
