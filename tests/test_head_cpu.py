"""Host-side tests of the 4-bit fully connected layer and of the questions about
logits (topk, log_prob, entropy): refusals, what finalize makes of them, and the
oracle's own definitions on small hand-made cases."""
import ctypes
import math

import numpy as np
import pytest

import oracle
import workloads
from workloads import ACT_NONE, ACT_RELU, NetBuilder
from paper_1907_01989_amd import _binding as B
from paper_1907_01989_amd import engine


def status(fn, *a, **k):
    with pytest.raises(B.MgiError) as e:
        fn(*a, **k)
    return e.value.status


@pytest.fixture
def graph():
    g = B.mgi_graph_create()
    yield g
    B.mgi_graph_destroy(g)


def codes(cout, cin):
    return np.full((cout, (cin + 1) // 2), 0x88, np.uint8)


def test_fc_int4_refusals(graph):
    g, L = graph, B.lib()
    x = B.mgi_graph_add_input(g, 2, 1, 1, 40)
    wide = B.mgi_graph_add_input(g, 2, 3, 1, 40)
    ix = B.mgi_graph_add_index_input(g, 2, 1, 1, 40)
    q, s = codes(5, 40), np.ones((5, 2), np.float32)
    add = lambda *a, **k: status(B.mgi_graph_add_fc_int4, g, *a, **k)  # noqa: E731
    assert add(9, 5, 32, q, s) == 1                       # no such tensor
    assert add(x, 0, 32, q, s) == 1                       # no classes
    assert add(x, 5, 0, q, s) == 1                        # no group
    assert add(x, 5, -32, q, s) == 1
    assert add(x, 5, 48, q, s) == 3                       # not a multiple of 32
    assert add(wide, 5, 32, q, s) == 3                    # not 1x1
    assert add(ix, 5, 32, q, s) == 3                      # indices
    assert add(x, 5, 32, q, s * np.float32(np.inf)) == 1
    assert add(x, 5, 32, q, s * np.float32(np.nan)) == 1
    z = np.full((5, 2), 15, np.uint8)
    z[4, 1] = 16
    assert add(x, 5, 32, q, s, z) == 1
    out = ctypes.c_int()
    assert L.mgi_graph_add_fc_int4(g, x, 5, 32, None, None, None, None, ctypes.byref(out)) == 1
    assert L.mgi_graph_add_fc_int4(None, x, 5, 32, None, None, None, None, ctypes.byref(out)) == 1
    assert "mgi_graph_add_fc_int4" in B.mgi_last_error()
    assert B.mgi_graph_add_fc_int4(g, x, 5, 32, q, s) == 3
    assert B.mgi_graph_add_fc_int4(g, x, 5, 64, q, np.ones((5, 1), np.float32), np.full((5, 1), 15, np.uint8)) == 4
    many = B.mgi_graph_add_input(g, 2 ** 24 + 1, 1, 1, 40)
    assert add(many, 5, 32, q, s) == 3                    # more images than offsets reach


def test_fc_int4_array_sizes_are_checked_by_the_engine():
    b = NetBuilder()
    t = b.fc_int4(b.input(1, 1, 1, 33, -1, 1), 7, 32, zeros=True)
    b.mark_output(t)
    for name, bad in (("q", np.zeros((7, 16), np.uint8)), ("scales", np.ones((7, 1), np.float32)),
                      ("zeros", np.zeros((7, 3), np.uint8)), ("b", np.zeros(6, np.float32)),
                      ("q", np.zeros((7, 17), np.int32))):
        desc = b.graph("sizes")
        desc["ops"] = [dict(op) for op in desc["ops"]]
        desc["ops"][t][name] = bad
        with pytest.raises(ValueError, match=name):
            engine.Plan(desc, bind=False)


def one_group(group, cout=300):
    b = NetBuilder()
    x = b.input(2, 1, 1, 64, -1, 1)
    t = b.fc_int4(x, cout, 64, zeros=True)
    b.ops[t]["group"] = group
    b.mark_output(t)
    return b.graph(f"group_{group}"), t


def test_a_group_may_be_far_longer_than_the_rows():
    # (the number of groups is counted without adding to the largest int)
    plans = [engine.Plan(one_group(g)[0], bind=False) for g in (96, 2 ** 31 - 32)]
    assert plans[0].weight_bytes == plans[1].weight_bytes


@pytest.mark.parametrize("group", [2 ** 32 + 32, 2 ** 32 + 64, -2 ** 32 + 64])
def test_a_group_that_no_int_holds_is_refused(group):
    # (as a C int these are groups of 32 and 64: other sizes than the arrays were checked for)
    with pytest.raises(ValueError, match="group"):
        engine.Plan(one_group(group)[0], bind=False)


@pytest.mark.parametrize("operand", [1, 2, 100, -1])
def test_an_operand_that_is_no_earlier_tensor_is_refused_by_the_library(operand):
    desc, t = one_group(64)
    desc["ops"] = [dict(op) for op in desc["ops"]]
    desc["ops"][t]["in"] = operand
    assert status(engine.Plan, desc, bind=False) == 1


@pytest.mark.parametrize("cin,n,cout,ok", [(32, 2 ** 24, 512, True), (32, 2 ** 24, 2000, False), (1024, 2 ** 23, 1024, True),
                                           (1024, 2 ** 24, 2000, False), (32, 2 ** 22, 2 ** 11, True), (32, 2 ** 22, 2 ** 14, False)])
def test_layers_that_no_launch_has_threads_for_are_refused(cin, n, cout, ok):
    ops = [{"op": "input", "shape": (n, 1, 1, cin), "dtype": B.DTYPE_FP16},
           {"op": "fc_int4", "in": 0, "cout": cout, "group": 32, "q": codes(cout, cin),
            "scales": np.ones((cout, cin // 32), np.float32), "zeros": None, "b": None}]
    desc = {"ops": ops, "outputs": [1]}
    if ok:
        assert kinds(engine.Plan(desc, bind=False))[-1] == "fc_int4"
    else:
        assert status(engine.Plan, desc, bind=False) == 3


def test_question_refusals(graph):
    g, L = graph, B.lib()
    x = B.mgi_graph_add_input(g, 2, 1, 1, 100)
    ix = B.mgi_graph_add_index_input(g, 2, 1, 1, 3)
    other = B.mgi_graph_add_index_input(g, 3, 1, 1, 3)
    tall = B.mgi_graph_add_index_input(g, 2, 2, 1, 3)
    assert status(B.mgi_graph_add_index_input, g, 0, 1, 1, 3) == 1
    assert status(B.mgi_graph_add_topk, g, x, 0) == 1
    assert status(B.mgi_graph_add_topk, g, x, 101) == 2
    assert status(B.mgi_graph_add_topk, g, x, 65) == 3
    assert status(B.mgi_graph_add_topk, g, ix, 1) == 3
    top = B.mgi_graph_add_topk(g, x, 64)
    assert status(B.mgi_graph_add_log_prob, g, x, x) == 1          # no indices
    assert status(B.mgi_graph_add_log_prob, g, x, other) == 2
    assert status(B.mgi_graph_add_log_prob, g, x, tall) == 2
    assert status(B.mgi_graph_add_log_prob, g, top, ix) == 3       # indices have no softmax
    assert status(B.mgi_graph_add_log_prob, g, x, 77) == 1
    assert status(B.mgi_graph_add_entropy, g, top) == 3
    assert status(B.mgi_graph_add_entropy, g, -1) == 1
    # indices are read by log_prob alone
    for fn in (B.mgi_graph_add_softmax, B.mgi_graph_add_argmax, B.mgi_graph_add_global_avgpool):
        assert status(fn, g, ix) == 3
        assert status(fn, g, top) == 3
    assert status(B.mgi_graph_add_activation, g, ix, 0) == 3
    assert status(B.mgi_graph_add_add, g, ix, ix) == 3
    assert status(B.mgi_graph_add_concat, g, [ix]) == 3
    assert status(B.mgi_graph_add_pad, g, ix, 1, 1, 1, 1) == 3
    assert status(B.mgi_graph_add_conv2d, g, ix, B.conv_desc(1, 1, cout=1), np.zeros((1, 1, 1, 3), np.float32)) == 3
    assert status(B.mgi_graph_mark_output, g, ix) == 3             # a graph input
    many = B.mgi_graph_add_input(g, 1, 1, 1, (1 << 19) + 1)
    assert status(B.mgi_graph_add_entropy, g, many) == 3
    arg = B.mgi_graph_add_argmax(g, x)
    assert status(B.mgi_graph_add_topk, g, arg, 1) == 3
    assert B.mgi_graph_add_log_prob(g, x, arg) >= 0                # argmax's labels may be asked about
    assert L.mgi_graph_add_topk(g, x, 1, None) == 1
    assert L.mgi_graph_add_index_input(None, 1, 1, 1, 1, None) == 1


def kinds(plan):
    return [n["kind"] for n in plan.nodes()]


def head(n=2, c=32, classes=100, k=5, **kw):
    b = NetBuilder(seed=1)
    x = b.input(n, 1, 1, c, -1, 1, **kw)
    z = b.fc_int4(x, classes)
    e = b.entropy(z)
    top = b.topk(z, k)
    given = b.index_input(np.zeros((n, 1, 1, 2)))
    outs = [b.log_prob(z, given), b.log_prob(z, top), e, top]
    for t in outs:
        b.mark_output(t)
    return b, outs


def test_questions_about_one_tensor_are_one_node():
    b, _ = head()
    plan = engine.Plan(b.graph("head"), bind=False)
    assert kinds(plan) == ["ingest", "fc_int4", "answers"]
    assert plan.nodes()[2]["n_fused"] == 4
    assert [i[1] for i in plan.inputs_info] == [B.DTYPE_FP16, B.DTYPE_INT32]
    assert [(i[0], i[1]) for i in plan.outputs_info] == [((2, 1, 1, 2), 2), ((2, 1, 1, 5), 2), ((2, 1, 1, 1), 2), ((2, 1, 1, 5), 3)]
    for kw in ({"fuse": False}, {"materialize_all": True}):
        plan = engine.Plan(b.graph("head"), bind=False, **kw)
        assert sorted(kinds(plan)) == sorted(["ingest", "fc_int4", "entropy", "topk", "log_prob", "log_prob"])
    for planner in (B.PLANNER_NAIVE, B.PLANNER_MCFP):
        assert kinds(engine.Plan(b.graph("head"), bind=False, planner=planner)) == ["ingest", "fc_int4", "answers"]


def test_questions_join_only_where_their_indices_are_ready():
    b = NetBuilder(seed=2)
    x, y = b.input(2, 1, 1, 40, -1, 1), b.input(2, 1, 1, 40, -1, 1)
    ex = b.entropy(x)
    ty = b.topk(y, 3)
    outs = [ex, b.log_prob(x, ty), b.log_prob(y, ty)]      # x at y's best: waits for y's node
    for t in outs:
        b.mark_output(t)
    plan = engine.Plan(b.graph("cross"), bind=False)
    assert kinds(plan) == ["entropy", "answers", "log_prob"]
    # a second topk, a second entropy and a fifth list start nodes of their own
    b = NetBuilder(seed=3)
    x = b.input(1, 1, 1, 40, -1, 1)
    ix = [b.index_input(np.zeros((1, 1, 1, 1))) for _ in range(5)]
    outs = [b.topk(x, 2), b.topk(x, 3), b.entropy(x), b.entropy(x)] + [b.log_prob(x, i) for i in ix]
    for t in outs:
        b.mark_output(t)
    assert kinds(engine.Plan(b.graph("many"), bind=False)) == ["answers", "answers"]


def test_activation_joins_the_layer_and_logits_may_be_an_output_too():
    b = NetBuilder(seed=4)
    z = b.activation(b.fc_int4(b.input(3, 1, 1, 64, -1, 1), 20), ACT_RELU)
    b.mark_output(z)
    b.mark_output(b.topk(z, 2))
    b.mark_output(b.softmax(z))
    assert kinds(engine.Plan(b.graph("act"), bind=False)) == ["ingest", "fc_int4", "topk", "softmax"]


def test_questions_about_a_sliced_tensor_share_one_copy():
    b = NetBuilder(seed=5)
    y = b.conv(b.input(1, 5, 4, 48, -1, 1), 21, 1, act=ACT_NONE)
    for t in (b.entropy(y), b.topk(y, 3)):
        b.mark_output(t)
    assert kinds(engine.Plan(b.graph("pixels"), bind=False)) == ["ingest", "pw_gemm", "export", "answers"]


def test_weights_take_half_a_byte():
    n = 4096
    b = NetBuilder()
    x = b.input(1, 1, 1, n, -1, 1)
    ops = [b.ops[0], {"op": "fc_int4", "in": 0, "cout": n, "group": 128, "q": codes(n, n),
                      "scales": np.ones((n, n // 128), np.float32), "zeros": None, "b": None}]
    plan = engine.Plan({"ops": ops, "outputs": [1]}, bind=False)
    assert x == 0 and plan.weight_bytes <= n * n // 2 + 2 * n * n // 128 + 8 * n + 4096


# ---------------------------------------------------------------- the oracle
def test_oracle_fc_int4_by_hand():
    # two classes, three channels in groups of two: codes 1 2 | 15 and 8 0 | 7
    q = np.array([[0x21, 0xFF], [0x08, 0xF7]], np.uint8)
    y = oracle.fc_int4(np.array([[[[1.0, 10.0, 100.0]]]]), q, np.array([[0.5, 2.0], [1.0, 4.0]]),
                       np.array([[1, 15], [8, 0]]), 2, np.array([0.25, -1.0]))
    assert y.tolist() == [[[[0.5 * 10 + 0.25, -8 * 10 + 4 * 7 * 100 - 1.0]]]]
    y = oracle.fc_int4(np.ones((1, 1, 1, 3)), q, np.ones((2, 1)), None, 32, None)
    assert y.tolist() == [[[[-7 - 6 + 7, 0 - 8 - 1]]]]


def test_oracle_questions_by_hand():
    ninf = -np.inf
    x = np.array([[1.0, 3.0, 3.0, ninf], [ninf, ninf, ninf, ninf], [0.0, np.nan, 5.0, 5.0], [2.0, np.inf, 0.0, 1.0]])
    assert oracle.topk(x, 4).tolist() == [[1, 2, 0, 3], [0, 1, 2, 3], [2, 3, 0, 1], [1, 0, 3, 2]]
    lp = oracle.log_prob(x, np.array([[0, 3, 4], [0, 1, -1], [0, 2, 3], [0, 1, 2]]))
    s = math.log(2 * math.exp(3) + math.exp(1))
    np.testing.assert_allclose(lp[0, :1], 1 - s)
    assert lp[0, 1] == ninf and np.isnan(lp[0, 2])
    assert lp[1, 0] == ninf and lp[1, 1] == ninf and np.isnan(lp[1, 2])
    assert np.isnan(lp[2:]).all()
    h = oracle.entropy(x)
    p = np.array([math.exp(1 - s), math.exp(3 - s), math.exp(3 - s)])
    np.testing.assert_allclose(h[0], -(p * np.log(p)).sum())
    assert h[1] == 0 and np.isnan(h[2:]).all()


def test_oracle_runs_a_head():
    b, outs = head()
    r = oracle.run_graph(b.graph("head"), keep=outs)
    assert r[outs[3]].shape == (2, 1, 1, 5) and (np.diff(r[outs[1]], axis=-1) <= 0).all()
    assert workloads.NetBuilder is NetBuilder and (r[outs[2]] <= math.log(100)).all()


def test_a_subset_of_the_batch_keeps_its_own_indices():
    b, outs = head(n=4)
    for op in b.ops:
        if op["op"] == "index_input":
            op["data"] = np.arange(8, dtype=np.int32).reshape(4, 1, 1, 2)
    desc = b.graph("head")
    full, part = oracle.run_graph(desc, keep=outs), oracle.run_graph(workloads.subset_batch(desc, [2, 0]), keep=outs)
    for t in outs:
        np.testing.assert_array_equal(part[t], full[t][[2, 0]])
