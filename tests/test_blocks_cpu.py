"""Host-side tests of the attention block's operators: refusals, what finalize
makes of them, 16-bit inputs and outputs, and the oracle's definitions on small
hand-made cases."""
import ctypes
import math

import numpy as np
import pytest

import oracle
from workloads import NetBuilder
from paper_1907_01989_amd import _binding as B
from paper_1907_01989_amd import engine


def status(fn, *a, **k):
    with pytest.raises(B.MgiError) as e:
        fn(*a, **k)
    return e.value.status


@pytest.fixture
def g():
    g = B.mgi_graph_create()
    yield g
    B.mgi_graph_destroy(g)


def codes(cout, cin, v=0x38):
    return np.full((cout, cin), v, np.uint8)


def test_norm_and_quantize_refusals(g):
    x = B.mgi_graph_add_input(g, 1, 4, 4, 40)
    ix = B.mgi_graph_add_index_input(g, 1, 4, 4, 40)
    wide = B.mgi_graph_add_input(g, 1, 1, 1, 2 ** 14 + 1)
    large = B.mgi_graph_add_input(g, 2 ** 15, 2 ** 10, 2 ** 8, 8)
    for add in (B.mgi_graph_add_rms_norm, B.mgi_graph_add_quantize):
        assert status(add, g, 99) == 1
        assert status(add, g, -1) == 1
        assert status(add, g, ix) == 3
        assert status(add, g, wide) == 3
        assert status(add, g, large) == 3
    label = B.mgi_graph_add_argmax(g, x)
    assert status(B.mgi_graph_add_quantize, g, label) == 3
    for eps in (-1e-6, math.inf, math.nan):
        assert status(B.mgi_graph_add_rms_norm, g, x, None, eps) == 1
    out, L = ctypes.c_int(), B.lib()
    assert L.mgi_graph_add_rms_norm(g, x, None, 1e-6, 2, ctypes.byref(out)) == 1
    assert L.mgi_graph_add_rms_norm(g, x, None, 1e-6, 0, None) == 1
    assert L.mgi_graph_add_rms_norm(None, x, None, 1e-6, 0, ctypes.byref(out)) == 1
    assert L.mgi_graph_add_quantize(g, x, None) == 1
    # an 8-bit tensor feeds the 8-bit layer only
    for q in (B.mgi_graph_add_quantize(g, x), B.mgi_graph_add_rms_norm(g, x, to8=True)):
        for add in (B.mgi_graph_add_rms_norm, B.mgi_graph_add_quantize, B.mgi_graph_add_softmax, B.mgi_graph_add_argmax,
                    B.mgi_graph_add_global_avgpool, B.mgi_graph_add_entropy):
            assert status(add, g, q) == 3
        assert status(B.mgi_graph_add_add, g, x, q, 0) == 3
        assert status(B.mgi_graph_add_concat, g, [x, q]) == 3
        assert status(B.mgi_graph_add_fc, g, q, 4, np.zeros((4, 40)), None) == 3
        assert status(B.mgi_graph_add_rotary, g, q, 1, 8, [1] * 4, [1.0] * 4) == 3
        assert status(B.mgi_graph_add_attention, g, x, q, x, 1, 1, 8) == 3
        B.mgi_graph_add_pointwise_fp8(g, q, 5, codes(5, 40), np.ones(1))


def test_pointwise_fp8_refusals(g):
    x = B.mgi_graph_add_input(g, 1, 4, 4, 40)
    q = B.mgi_graph_add_quantize(g, x)
    add = lambda *a, **k: status(B.mgi_graph_add_pointwise_fp8, g, *a, **k)  # noqa: E731
    one = np.ones((1, 1), np.float32)
    assert add(99, 5, codes(5, 40), one) == 1
    assert add(x, 5, codes(5, 40), one) == 3             # not held in 8 bits
    assert add(q, 0, codes(1, 40), one) == 1
    assert add(q, -3, codes(1, 40), one) == 1
    assert add(q, 5, codes(5, 40), one, None, 9) == 1    # no such activation
    for bad in (np.inf, np.nan):
        assert add(q, 5, codes(5, 40), one * np.float32(bad)) == 1
    for bad in (0x7f, 0xff):
        c = codes(5, 40)
        c[4, 39] = bad
        assert add(q, 5, c, one) == 1
    assert add(q, 5, None, one) == 1
    assert add(q, 5, codes(5, 40), None) == 1


def test_rotary_refusals(g):
    x = B.mgi_graph_add_input(g, 1, 4, 4, 40)
    p = B.mgi_graph_add_index_input(g, 1, 4, 4, 2)
    other = B.mgi_graph_add_index_input(g, 1, 4, 5, 2)
    many = B.mgi_graph_add_index_input(g, 1, 4, 4, 9)
    add = lambda *a, **k: status(B.mgi_graph_add_rotary, g, *a, **k)  # noqa: E731
    ax, f = [1, 2], [1.0, 0.5]
    assert add(99, 1, 8, ax, f) == 1
    assert add(p, 1, 8, ax, f) == 3
    assert add(x, 0, 8, ax, f) == 1
    assert add(x, 1, 0, ax, f) == 1
    assert add(x, 1, 12, ax, f) == 3
    assert add(x, 1, 8, ax, f, first=4) == 3
    assert add(x, 1, 8, ax, f, first=-8) == 1
    assert add(x, 1, 8, [0] * 5, [1.0] * 5) == 2         # more pairs than half a head
    assert add(x, 6, 8, ax, f) == 2                      # past the last channel
    assert add(x, 2 ** 30, 8, ax, f) == 2
    assert add(x, 5, 8, ax, f, first=8) == 2
    assert add(x, 1, 8, [0, 3], f) == 1
    assert add(x, 1, 8, [-1, 0], f) == 1
    assert add(x, 1, 8, ax, [1.0, math.inf]) == 1
    assert add(x, 1, 8, ax, f, positions=p) == 1         # two axes: no axis 2
    assert add(x, 1, 8, [0, 1], f, positions=other) == 2
    assert add(x, 1, 8, [0, 1], f, positions=many) == 3
    assert add(x, 1, 8, [0, 1], f, positions=x) == 1
    assert add(x, 1, 8, [0, 1], f, positions=77) == 1
    assert add(x, 1, 8, [0, 1], f, positions=-2) == 1
    d = B.RotaryDesc(1, 8, 0, 2, 2)
    out = ctypes.c_int()
    axes, freqs = (ctypes.c_int * 2)(0, 1), (ctypes.c_double * 2)(1, 1)
    assert B.lib().mgi_graph_add_rotary(g, x, ctypes.byref(d), axes, freqs, -1, ctypes.byref(out)) == 1
    d.adjacent = 0
    assert B.lib().mgi_graph_add_rotary(g, x, ctypes.byref(d), None, freqs, -1, ctypes.byref(out)) == 1
    assert B.lib().mgi_graph_add_rotary(g, x, None, axes, freqs, -1, ctypes.byref(out)) == 1
    assert B.lib().mgi_graph_add_rotary(g, x, ctypes.byref(d), axes, freqs, -1, ctypes.byref(out)) == 0


def test_more_workgroups_than_a_launch_has_are_refused(g):
    # (sequences or images times heads of keys)
    wide = B.mgi_graph_add_input(g, 1, 1, 1, 2 ** 23, 0)
    most = B.mgi_graph_add_index_input(g, 1, 1, 1, 2 ** 16 + 1)
    few = B.mgi_graph_add_index_input(g, 1, 1, 1, 2)
    assert status(B.mgi_graph_add_attention, g, wide, wide, wide, 2 ** 20, 2 ** 20, 8, bounds=most) == 3
    assert B.mgi_graph_add_attention(g, wide, wide, wide, 2 ** 20, 2 ** 20, 8, bounds=few) == 3
    many = B.mgi_graph_add_input(g, 2 ** 23, 1, 1, 16, 0)
    assert status(B.mgi_graph_add_attention, g, many, many, many, 2, 2, 8) == 3
    assert B.mgi_graph_add_attention(g, many, many, many, 2, 1, 8) == 5


def test_rotary_takes_arrays():
    from paper_1907_01989_amd import engine
    ops = [{"op": "input", "shape": (1, 2, 2, 16)},
           {"op": "rotary", "in": 0, "heads": 1, "head_dim": 16, "axes": np.array([0, 1, 2]),
            "freqs": np.array([1, 0.5, 0.25], np.float32)}]
    B.mgi_graph_destroy(engine.build_graph({"ops": ops, "outputs": [1]}))


def test_attention_refusals(g):
    q = B.mgi_graph_add_input(g, 2, 4, 4, 64)
    k = B.mgi_graph_add_input(g, 2, 2, 2, 32)
    k3 = B.mgi_graph_add_input(g, 3, 2, 2, 32)
    row = B.mgi_graph_add_input(g, 1, 1, 32, 32)
    ix = B.mgi_graph_add_index_input(g, 1, 1, 1, 4)
    ix5 = B.mgi_graph_add_index_input(g, 1, 1, 1, 5)
    single = B.mgi_graph_add_index_input(g, 1, 1, 1, 1)
    lots = B.mgi_graph_add_index_input(g, 1, 1, 1, 2 ** 16 + 2)
    add = lambda *a, **kw: status(B.mgi_graph_add_attention, g, *a, **kw)  # noqa: E731
    assert add(99, k, k, 8, 4, 8) == 1
    assert add(ix, k, k, 8, 4, 8) == 3
    assert add(q, k, k, 8, 3, 8) == 1                    # no whole groups
    assert add(q, k, k, 0, 1, 8) == 1
    assert add(q, k, k, 8, 0, 8) == 1
    assert add(q, k, k, 8, 4, 0) == 1
    assert add(q, k, k, 2, 1, 12) == 3
    assert add(q, k, k, 1, 1, 136) == 3
    assert add(q, k, k, 1, 1, 8, q_from=4) == 3
    assert add(q, k, k, 1, 1, 8, v_from=-8) == 1
    assert add(q, k, k, 8, 8, 8) == 2                    # k has four heads of eight
    assert add(q, k, k, 2 ** 30, 2 ** 30, 8) == 2
    assert add(q, k, k, 8, 4, 8, q_from=8) == 2
    assert add(q, k, k, 8, 4, 8, k_from=8) == 2
    assert add(q, k, k3, 8, 4, 8) == 2                   # k and v differ
    assert add(q, k3, k3, 8, 4, 8) == 2                  # images differ
    assert add(q, k, k, 8, 4, 8, scale=math.nan) == 1
    assert add(q, k, k, 8, 4, 8, scale=math.inf) == 1
    assert add(q, k, k, 8, 4, 8, bounds=ix) == 2         # pixels differ, no k_bounds
    assert add(q, k, k, 8, 4, 8, bounds=q) == 1
    assert add(q, k, k, 8, 4, 8, k_bounds=ix) == 1       # without bounds
    assert add(q, k, k, 8, 4, 8, bounds=ix, k_bounds=ix5) == 2
    assert add(q, k, k, 8, 4, 8, bounds=ix, k_bounds=k) == 1
    assert add(q, row, row, 8, 4, 8, bounds=single) == 2
    assert add(q, row, row, 8, 4, 8, bounds=lots) == 3
    assert B.mgi_graph_add_attention(g, q, row, row, 8, 4, 8, bounds=ix) == 8
    assert B.mgi_graph_add_attention(g, q, k, k, 8, 4, 8, bounds=ix, k_bounds=ix) == 9
    d = B.AttentionDesc(8, 4, 8, 0, 0, 0, 2, 0.0)
    out = ctypes.c_int()
    assert B.lib().mgi_graph_add_attention(g, q, k, k, ctypes.byref(d), -1, -1, ctypes.byref(out)) == 1
    assert B.lib().mgi_graph_add_attention(g, q, k, k, None, -1, -1, ctypes.byref(out)) == 1


def test_array_sizes_are_checked_by_the_engine():
    b = NetBuilder()
    x = b.input(1, 4, 4, 136, -1, 1)
    n = b.rms_norm(x)
    q = b.quantize(x)
    p = b.pointwise_fp8(q, 200)
    r = b.rotary(x, 2, 64, [1] * 16, [1.0] * 16)
    a = b.attention(r, r, r, 2, 2, 64)
    for t in (n, p, a):
        b.mark_output(t)
    good = b.graph("sizes")
    plan = engine.Plan(good, bind=False)
    assert [s for s, _, _ in plan.outputs_info] == [(1, 4, 4, 136), (1, 4, 4, 200), (1, 4, 4, 128)]
    for t, name, bad in ((n, "w", np.ones(135)), (p, "q", np.zeros((200, 128), np.uint8)), (p, "q", np.zeros((200, 136), np.int32)),
                         (p, "scales", np.ones(2)), (p, "b", np.ones(199)), (r, "freqs", [1.0] * 15)):
        desc = b.graph("sizes")
        desc["ops"] = [dict(op) for op in desc["ops"]]
        desc["ops"][t][name] = bad
        with pytest.raises(ValueError, match=name):
            engine.Plan(desc, bind=False)


def test_types_of_inputs_and_outputs():
    b = NetBuilder()
    x = b.input(1, 4, 4, 16, -1, 1, dtype=B.DTYPE_BF16)
    c = b.conv(x, 24, 1)
    b.mark_output(c)
    with pytest.raises(B.MgiError, match="bf16"):
        engine.Plan(b.graph("bf16"), bind=False)
    plan = engine.Plan(b.graph("bf16"), bind=False, dtype=B.DTYPE_BF16)
    assert plan.inputs_info[0] == ((1, 4, 4, 16), B.DTYPE_BF16, 512)
    assert plan.outputs_info[0][1:] == (B.DTYPE_FP32, 4 * 384)
    for dtype in (B.DTYPE_FP16, B.DTYPE_BF16):
        desc = {**b.graph("out"), "output_dtypes": {c: dtype}}
        desc["ops"] = [dict(desc["ops"][0], dtype=B.DTYPE_FP32)] + desc["ops"][1:]
        plan = engine.Plan(desc, bind=False, dtype=dtype)
        assert plan.outputs_info[0][1:] == (dtype, 2 * 384)
        with pytest.raises(B.MgiError, match="storage type"):
            engine.Plan(desc, bind=False, dtype=1 - dtype)


def test_16_bit_outputs_are_refused_for_tensors_of_32(g):
    x = B.mgi_graph_add_input(g, 2, 1, 1, 8)
    flat = [B.mgi_graph_add_fc(g, x, 4, np.zeros((4, 8)), None), B.mgi_graph_add_softmax(g, x), B.mgi_graph_add_argmax(g, x),
            B.mgi_graph_add_topk(g, x, 2), B.mgi_graph_add_entropy(g, x)]
    for t in flat:
        assert status(B.mgi_graph_mark_output_as, g, t, B.DTYPE_FP16) == 3
        B.mgi_graph_mark_output_as(g, t, B.DTYPE_FP32)
        assert status(B.mgi_graph_mark_output, g, t) == 1
    assert status(B.mgi_graph_mark_output_as, g, flat[0], B.DTYPE_INT32) == 3
    assert status(B.mgi_graph_mark_output_as, g, x, B.DTYPE_FP16) == 3
    assert status(B.mgi_graph_mark_output_as, g, 77, B.DTYPE_FP16) == 1


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("form", ["relu", "none", "two", "behind one", "int4"])
def test_16_bit_outputs_are_refused_for_activations_of_logits(form, dtype):
    # (the layer takes the activation along and writes fp32 values: twice the bytes of such an output)
    b = NetBuilder()
    x = b.input(2, 1, 1, 64, -1, 1)
    f = b.fc_int4(x, 8) if form == "int4" else b.fc(x, 8)
    if form == "behind one":
        f = b.concat([f])
    if form == "two":
        f = b.activation(f, 0)
    a = b.activation(f, 0 if form == "none" else 1)
    wide = engine.Plan({"ops": b.ops, "outputs": [a]}, bind=False, dtype=dtype)
    assert wide.outputs_info[0][1:] == (B.DTYPE_FP32, 64)
    with pytest.raises(B.MgiError, match="16 bits") as e:
        engine.Plan({"ops": b.ops, "outputs": [a], "output_dtypes": {a: dtype}}, bind=False, dtype=dtype)
    assert e.value.status == 3


def kinds(b, outputs, **kw):
    plan = engine.Plan({"ops": b.ops, "outputs": outputs}, bind=False, **kw)
    return [n["kind"] for n in plan.nodes() if n["kind"] not in ("ingest", "export")]


def test_a_norm_takes_the_add_before_it_along():
    b = NetBuilder()
    x, y = b.input(1, 4, 4, 40, -1, 1), b.input(1, 4, 4, 40, -1, 1)
    s = b.add(x, y)
    n = b.rms_norm(s)
    m = b.rms_norm(s, to8=True)
    p = b.pointwise_fp8(m, 8)
    assert kinds(b, [n]) == ["add_rms_norm"]
    assert kinds(b, [s, n]) == ["add_rms_norm"]
    assert kinds(b, [n, p]) == ["add_rms_norm", "rms_norm", "pointwise_fp8"]     # one of two norms
    assert kinds(b, [n], fuse=False) == ["add", "rms_norm"]
    assert kinds(b, [n], materialize_all=True) == ["add", "rms_norm"]
    # not a residual that a convolution takes
    c = b.add(b.conv(x, 40, 1, act=0), y)
    assert kinds(b, [b.rms_norm(c)]) == ["pw_gemm", "rms_norm"]


def test_oracle_definitions():
    # 8 bits: the least power of two that holds the block, ties to even, steps below 2^-6
    x = np.zeros((1, 1, 1, 130))
    x[..., :6] = [448, 17, 19, 2.0 ** -10, 3 * 2.0 ** -10, -0.3]
    x[..., 128:] = [449, 1]
    assert oracle.block_exponents(x).reshape(-1).tolist() == [0, 1]
    q = oracle.quantize(x).reshape(-1)
    assert q[:6].tolist() == [448, 16, 20, 0, 2.0 ** -8, -0.3125] and q[128:].tolist() == [448, 1]
    assert oracle.e4m3_values([0x7e, 0xfe, 0x08, 0x07, 0x01, 0x38]).tolist() == [448, -448, 2.0 ** -6, 7 * 2.0 ** -9, 2.0 ** -9, 1]
    # a quarter of a turn takes (1, 0) to (0, 1)
    y = oracle.rotary(np.array([1.0, 0, 5, 7, 1, 0, 5, 7]).reshape(1, 1, 1, 8), 1, 8, [0], [np.pi / 2], np.ones((1, 1, 1, 1), int), adjacent=True)
    np.testing.assert_allclose(y.reshape(-1), [0, 1, 5, 7, 1, 0, 5, 7], atol=1e-15)
    y = oracle.rotary(np.arange(8.0).reshape(1, 1, 1, 8), 1, 8, [0, 0], [np.pi / 2] * 2, np.ones((1, 1, 1, 1), int))
    np.testing.assert_allclose(y.reshape(-1), [-2, -3, 0, 1, 4, 5, 6, 7], atol=1e-14)
    # equal scores: means of what is seen; queries that see nothing: zeros
    v = np.arange(24.0).reshape(1, 1, 3, 8)
    z = oracle.attention(np.zeros((1, 1, 4, 8)), np.ones((1, 1, 3, 8)), v, 1, 1, 8, causal=True)
    np.testing.assert_allclose(z[0, 0], [np.zeros(8), v[0, 0, 0], v[0, 0, :2].mean(0), v[0, 0].mean(0)])
    assert oracle.attention_spans(10, 10, 1, [2, 5, 4, 99]) == [(2, 5, 2, 5), (5, 5, 5, 5), (5, 10, 5, 10)]


@pytest.mark.parametrize("planner", [B.PLANNER_GREEDY, B.PLANNER_MCFP])
@pytest.mark.parametrize("layer", ["rotary", "pointwise_fp8"])
def test_the_workspace_does_not_grow_with_the_blocks(layer, planner):
    # each block's sum feeds its norm alone: a fused sum is no tensor
    def workspace(blocks, fuse):
        b = NetBuilder()
        h = b.input(1, 32, 32, 256, -1, 1, dtype=B.DTYPE_FP16)
        for _ in range(blocks):
            y = b.rotary(h, 4, 64, [1, 2] * 8, [0.5] * 16) if layer == "rotary" else b.pointwise_fp8(b.quantize(h), 256)
            h = b.rms_norm(b.add(h, y))
        plan = engine.Plan({"ops": b.ops, "outputs": [h]}, bind=False, fuse=fuse, planner=planner)
        assert ("add_rms_norm" in [n["kind"] for n in plan.nodes()]) == fuse
        return plan.workspace_bytes

    assert workspace(12, True) == workspace(4, True) <= workspace(4, False) == workspace(12, False)
    assert workspace(1, True) <= workspace(1, False)


def test_a_fused_sum_in_a_concatenation_needs_no_copy():
    def plan(fuse):
        b = NetBuilder()
        x = b.input(1, 32, 32, 64, -1, 1, dtype=B.DTYPE_FP16)
        s = b.add(b.conv(x, 64, 1), b.conv(x, 64, 1, act=0))
        t = b.add(b.dw(x), b.dw(x, act=0))
        n = b.rms_norm(t)
        return engine.Plan({"ops": b.ops, "outputs": [b.conv(b.concat([s, t, n]), 16)]}, bind=False, fuse=fuse)

    p = plan(True)
    assert "add_rms_norm" in [n["kind"] for n in p.nodes()]
    # the three parts lie in the concatenation, beside it the input's sliced copy and the two summands: with one
    # of the parts copied the workspace holds that twice
    whole, part = 32 * 32 * 192 * 2, 32 * 32 * 64 * 2
    assert p.workspace_bytes <= whole + 3 * part and p.memory_report()[1] <= plan(False).memory_report()[1]
