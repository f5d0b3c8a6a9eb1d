"""Questions about tensors of every kind that a graph has, in graphs that use
them otherwise too: against the oracle's topk, log_prob and entropy (64 bits) of
the values that the plan itself hands out.  Tolerances as in test_gpu_answers."""
import numpy as np
import pytest

import oracle
from workloads import ACT_NONE, DTYPE_FP16, DTYPE_FP32, NetBuilder

from gpu_util import log, run_gpu
from test_gpu_answers import same

pytestmark = pytest.mark.gpu


def check(z, top, lp, h, given, lg):
    z = z.astype(np.float64)
    np.testing.assert_array_equal(top, oracle.topk(z, top.shape[-1]))
    for got, ref in ((lp, oracle.log_prob(z, top)), (lg, oracle.log_prob(z, given))):
        same(got, ref, 2e-5 + 2.0 ** -21 * np.abs(ref))
    ref = oracle.entropy(z)
    same(h, ref, 2e-5 * (1 + 2 * np.abs(ref)))


def tensors(b):
    """One tensor of each kind, all of them graph outputs."""
    x = b.input(3, 7, 5, 24, -2, 2)
    c = b.conv(x, 21, 1, act=ACT_NONE)
    d = b.dw(x)
    a = b.add(c, b.conv(x, 21, 1, act=ACT_NONE))
    r = b.resize(c, 9, 8, align_corners=False)
    p = b.gap(b.conv(x, 40, 1))
    z = b.fc(p, 100)
    q = b.fc_int4(p, 101)
    return {"conv": c, "depthwise": d, "add": a, "resize": r, "concat": b.concat([c, d]), "pool": p, "fc": z,
            "fc_int4": q, "softmax": b.softmax(z)}


@pytest.mark.parametrize("kind", ["conv", "depthwise", "add", "resize", "concat", "pool", "fc", "fc_int4", "softmax"])
@pytest.mark.parametrize("dtype", [0, 1])
def test_each_kind_of_tensor(kind, dtype):
    b = NetBuilder(seed=21)
    t = tensors(b)[kind]
    n, (h, w, c) = 3, b.hwc(t)
    given = np.random.default_rng(3).integers(-1, c + 1, (n, h, w, 2))
    top = b.topk(t, 4)
    outs = [t, top, b.log_prob(t, top), b.entropy(t), b.log_prob(t, b.index_input(given))]
    for o in outs:
        b.mark_output(o)
    desc = b.graph(kind)
    log(f"[case] questions about a {kind}, storage type {dtype}")
    _, got, _ = run_gpu(desc, materialize_all=False, dtype=dtype)
    flat = lambda v: v.reshape(n * h * w, -1)  # noqa: E731
    check(flat(got[0]), flat(got[1]), flat(got[2]), flat(got[3]), flat(given), flat(got[4]))
    # the tensor no output, and no fusion: the same answers
    for kw in ({"outputs": outs[1:]}, {"outputs": [outs[2], outs[4]]}):
        _, again, _ = run_gpu({**desc, **kw}, materialize_all=False, dtype=dtype)
        for o, v in zip(kw["outputs"], again):
            np.testing.assert_array_equal(v, got[outs.index(o)])
    _, again, nodes = run_gpu(desc, materialize_all=True, fuse=False, dtype=dtype)
    z = flat(again[0])
    check(z, flat(again[1]), flat(again[2]), flat(again[3]), flat(given), flat(again[4]))
    for o, v in zip(outs[1:], again[1:]):
        np.testing.assert_array_equal(flat(nodes[o]), flat(v))


@pytest.mark.parametrize("planner", [0, 1, 2])
@pytest.mark.parametrize("rows,classes", [(1, 30000), (40, 1001)])
def test_answers_that_only_other_answers_read(planner, rows, classes):
    # topk is no output: its place in the arena is written all the same, and so
    # are the segments' parts, beside logits that the kernel still reads
    b = NetBuilder(seed=22)
    x = b.input(rows, 1, 1, 64, -1, 1, dtype=DTYPE_FP32)
    z = b.fc_int4(x, classes, 32, True)
    top, small = b.topk(z, 20), b.topk(z, 3)
    y = b.fc(x, classes)
    outs = [b.log_prob(z, top), b.log_prob(z, small), b.log_prob(y, top), b.log_prob(y, b.topk(y, 7)), b.entropy(y), z, y]
    for o in outs:
        b.mark_output(o)
    desc = b.graph("inner")
    log(f"[case] inner answers, {rows} x {classes}, planner {planner}")
    _, got, _ = run_gpu(desc, materialize_all=False, planner=planner)
    lz, ly = got[5].astype(np.float64), got[6].astype(np.float64)
    for g, l, i in ((got[0], lz, oracle.topk(lz, 20)), (got[1], lz, oracle.topk(lz, 3)), (got[2], ly, oracle.topk(lz, 20)),
                    (got[3], ly, oracle.topk(ly, 7))):
        same(g, oracle.log_prob(l, i), 2e-5 + 2.0 ** -21 * np.abs(oracle.log_prob(l, i)))
    h = oracle.entropy(ly)
    same(got[4], h, 2e-5 * (1 + 2 * np.abs(h)))
    _, alone, _ = run_gpu({**desc, "outputs": outs[:5]}, materialize_all=False, planner=planner)
    for p, q in zip(got, alone):
        np.testing.assert_array_equal(p, q)


def test_one_index_input_for_two_tensors_and_two_answers_from_one_index():
    b = NetBuilder(seed=23)
    x, y = b.input(5, 1, 1, 300, -3, 3, dtype=DTYPE_FP32), b.input(5, 1, 1, 77, -3, 3, dtype=DTYPE_FP16)
    ix = b.index_input(np.random.default_rng(1).integers(0, 90, (5, 1, 1, 4)))
    outs = [b.log_prob(x, ix), b.log_prob(y, ix), b.log_prob(x, ix)]
    for o in outs:
        b.mark_output(o)
    desc = b.graph("shared")
    log("[case] shared indices")
    _, got, _ = run_gpu(desc, materialize_all=False)
    ref = oracle.run_graph(desc, keep=outs)
    for o, g in zip(outs, got):
        r = ref[o].reshape(g.shape)
        same(g, r, 2e-5 + 2.0 ** -21 * np.abs(r))
    assert np.isnan(got[1]).any()
