"""Every kernel form of the 4-bit layer, against the oracle (64 bits).

The tile kernels differ by rows (16 or 32), channels (32, or 64 above 16384),
groups of waves along K (one to four), inputs that share a scale (32, 64 or 128
to a step) and how they get their rows: fp16 read in place, converted by the
layer (up to 16 rows), or slices.  The bound is the one of test_gpu_fcint4."""
import numpy as np
import pytest

import oracle
import workloads
from workloads import DTYPE_FP16, DTYPE_FP32, NetBuilder

from gpu_util import log, run_gpu
from test_gpu_fcint4 import bound, check, layer

pytestmark = pytest.mark.gpu

TILES = [
    # n, cin, cout, group, zeros
    # 32 rows, four groups along K, an uneven share of its blocks among them
    (64, 4096, 1000, 128, False), (40, 2100, 300, 96, True), (17, 2049, 33, 32, True), (33, 2056, 500, 64, False),
    (31, 1921, 47, 256, True), (32, 2048, 1000, 32, False),
    # ... two and one
    (50, 1152, 700, 128, True), (60, 264, 100, 128, False),
    # 16 rows x 64 channels, two groups and one
    (8, 2048, 16500, 128, False), (16, 1096, 16400, 96, True), (3, 136, 17000, 128, True),
    # 16 rows x 32 channels, four to one
    (16, 1024, 5000, 128, True), (9, 776, 4300, 128, False), (5, 640, 4200, 64, False), (1, 520, 4100, 64, True),
    (2, 384, 4112, 32, True),
]


@pytest.mark.parametrize("src,dtype", [(DTYPE_FP16, 0), (DTYPE_FP32, 0), (DTYPE_FP32, 1)])
@pytest.mark.parametrize("n,cin,cout,group,zeros", TILES)
def test_each_tile(n, cin, cout, group, zeros, src, dtype):
    import torch
    from paper_1907_01989_amd import engine
    desc, t = layer(n, cin, cout, group, zeros, dtype=src, seed=10)
    if dtype == 1:
        desc = workloads.as_bf16_graph(desc)
    log(f"[case] {desc['name']} inputs {src}, storage type {dtype}")
    plan = engine.Plan(desc, dtype=dtype)
    (x,) = plan.input_tensors()
    got = plan.run([x])[0].clone()
    check(desc, t, got.cpu().numpy())
    assert torch.equal(plan.run([x])[0], got)
    # off 16 bytes the rows are converted to slices first: the same values and sums
    apart = torch.empty(x.numel() + 4, dtype=x.dtype, device=x.device)
    off = apart[1:1 + x.numel()].view(x.shape)
    off.copy_(x)
    assert torch.equal(plan.run([off])[0], got)


@pytest.mark.parametrize("n,cout", [(20, 300), (6, 5000)])
def test_softmax_behind_the_layer(n, cout):
    # the layer's logits as an output beside their softmax, and the softmax alone
    b = NetBuilder(seed=12)
    z = b.fc_int4(b.input(n, 1, 1, 200, -1, 1, dtype=DTYPE_FP32), cout, 64, True)
    y = b.softmax(z)
    b.mark_output(z)
    b.mark_output(y)
    desc = b.graph("softmax")
    log(f"[case] softmax behind {n} x 200 x {cout}")
    plan, (logits, probs), _ = run_gpu(desc, materialize_all=False)
    assert [k["kind"] for k in plan.nodes()][-2:] == ["fc_int4", "softmax"]
    check(desc, z, logits)
    ref = oracle.softmax(logits.astype(np.float64).reshape(n, 1, 1, cout)).reshape(n, cout)
    # a term's exponent is off by |x - m| 2^-23 and its exponential by 2^-22, the sum and
    # the quotient round as often: |x - m| below 40, up to cout / 64 + 16 sums
    d = logits.max(1, keepdims=True) - logits
    assert d.max() < 40
    assert (np.abs(probs - ref) <= ref * (2 * 40 + 8 + cout / 64 + 16) * 2.0 ** -23).all()
    _, (alone,), _ = run_gpu({**desc, "outputs": [y]}, materialize_all=False)
    np.testing.assert_array_equal(alone, probs)
    _, again, _ = run_gpu(desc, materialize_all=True, fuse=False)
    np.testing.assert_array_equal(again[1], probs)
