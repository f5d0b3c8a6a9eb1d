"""The attention block's operators together, as a program has them: a norm in 8
bits, one layer for queries, keys and values, rotary positions, attention, the
layer behind it, the residual and the next norm; eager, captured and replayed, in
the no-allocation workspace, on another stream, and with buffers of every kind."""
import numpy as np
import pytest

import oracle
from gpu_util import log

pytestmark = pytest.mark.gpu

HEADS, KV, DIM, C = 4, 2, 32, 96


def block(dtype, n=2, h=5, w=7, src=None, bounds=None, seed=0):
    from block_util import builder, given, stored
    b = builder(seed + 5)
    x = given(b, stored(np.random.default_rng(seed).standard_normal((n, h, w, C)), dtype), dtype if src is None else src)
    tokens = b.rms_norm(x, to8=True)
    qkv = b.pointwise_fp8(tokens, (HEADS + 2 * KV) * DIM)
    b.ops[qkv]["scales"] = b.ops[qkv]["scales"] * 0.5
    half = DIM // 2
    turned = b.rotary(qkv, HEADS + KV, DIM, [1 + i % 2 for i in range(half)], [0.5 ** i for i in range(half)])
    extra = {} if bounds is None else {"bounds": b.index_input(np.asarray(bounds).reshape(1, 1, 1, -1))}
    y = b.attention(turned, turned, qkv, HEADS, KV, DIM, k_from=HEADS * DIM, v_from=(HEADS + KV) * DIM, **extra)
    o = b.pointwise_fp8(b.quantize(y), C)
    s = b.add(x, o, act=0)
    z = b.rms_norm(s)
    return b, dict(x=x, tokens=tokens, qkv=qkv, turned=turned, y=y, o=o, s=s, z=z)


def plan_of(b, outputs, dtype, **kw):
    from paper_1907_01989_amd import engine
    return engine.Plan({"name": "block", "ops": b.ops, "outputs": outputs, "output_dtypes": {t: dtype for t in outputs}}, dtype=dtype, **kw)


@pytest.mark.parametrize("dtype,src", [(0, 0), (1, 1), (1, 2)])
def test_block(dtype, src):
    from block_util import HALF, run
    b, t = block(dtype, src=src)
    log(f"[case] block type {dtype} from {src}")
    want = [t[k] for k in ("qkv", "turned", "y", "o", "s", "z")]
    got, plan = run(b, want, dtype)
    # each operator on the operands that the plan itself made (the norm's codes are tested alone)
    vals = dict(zip(want, got))
    vals[t["x"]] = np.asarray(b.ops[t["x"]]["data"])
    for k in ("turned", "y", "s", "z"):
        op = b.ops[t[k]]
        ref = oracle.eval_op(op, [vals[u] for u in oracle.op_inputs(op)])
        # one rounding to 16 bits, one of the weights, and fp32
        assert np.abs(vals[t[k]] - ref).max() <= (2 * HALF[dtype] + 2.0 ** -12) * np.abs(ref).max(), k
    ref = oracle.eval_op(b.ops[t["o"]], [oracle.quantize(vals[t["y"]])])
    assert np.abs(vals[t["o"]] - ref).max() <= 2 * HALF[dtype] * np.abs(ref).max()
    assert [i["kind"] for i in plan.nodes() if i["kind"] not in ("export", "ingest")] == [
        "rms_norm", "pointwise_fp8", "rotary", "attention", "quantize", "pointwise_fp8", "add_rms_norm"]
    # unfused, with every tensor kept: the same bits
    again, _ = run(b, want, dtype, fuse=False)
    kept, plan = run(b, want, dtype, materialize_all=True)
    for a, c, d in zip(got, again, kept):
        np.testing.assert_array_equal(a, c)
        np.testing.assert_array_equal(a, d)


def test_packed_block_replayed_and_without_allocation():
    import torch
    from block_util import inputs
    from paper_1907_01989_amd import _binding as B
    # rows of keys long enough to be shared by several workgroups
    b, t = block(0, 1, 1, 3001, bounds=[0, 2990, 2991, 2991, 3000])
    outs = [t["z"], t["y"]]
    plan = plan_of(b, outs, 0)
    xs = inputs(plan)
    log("[case] block replayed")
    eager = [o.clone() for o in plan.run(xs)]
    assert all(torch.isfinite(o).all() for o in eager) and (eager[1].reshape(3001, -1)[3000:] == 0).all()
    g = plan.capture(xs)
    other = plan_of(b, outs, 0)
    xs2 = [x if x.dtype == torch.int32 else x * 0.5 for x in xs]
    ref2 = [o.clone() for o in other.run(xs2)]
    h = other.capture(xs2)
    for _ in range(4):
        for o in list(g) + list(h):
            o.fill_(-3)
        plan.replay()
        other.replay()
        more = plan.run(xs)
        torch.cuda.synchronize()
        for a, c, d in zip(g, eager, more):
            assert torch.equal(a, c) and torch.equal(d, c)
        for a, c in zip(h, ref2):
            assert torch.equal(a, c)
    # new values in the same buffers
    xs[0].copy_(xs2[0])
    plan.replay()
    torch.cuda.synchronize()
    for a, c in zip(g, ref2):
        assert torch.equal(a, c)
    outs = plan.alloc_outputs()
    for _ in range(2):
        for o in outs:
            o.fill_(7)
        B.mgi_plan_run_noalloc(plan.handle, [x.data_ptr() for x in xs], [o.data_ptr() for o in outs],
                               torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        for a, c in zip(outs, ref2):
            assert torch.equal(a, c)


def test_another_stream_and_many_runs():
    import torch
    from block_util import inputs
    b, t = block(1, 1, 1, 2500, seed=3)
    plan = plan_of(b, [t["z"]], 1)
    xs = inputs(plan)
    ref = plan.run(xs)[0].clone()
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    log("[case] block on another stream")
    with torch.cuda.stream(st):
        outs = [plan.run(xs)[0] for _ in range(5)]
    st.synchronize()
    for o in outs:
        assert torch.equal(o, ref)


@pytest.mark.parametrize("dtype", [0, 1])
def test_buffers_off_16_bytes(dtype):
    import torch
    from block_util import inputs
    b, t = block(dtype, 1, 6, 6)
    outs = [t["y"], t["s"], t["z"], t["turned"]]
    plan = plan_of(b, outs, dtype)
    xs = inputs(plan)
    ref = [o.clone() for o in plan.run(xs)]
    log(f"[case] block, buffers off 16 bytes, type {dtype}")

    def off(x, fill=None):
        y = torch.full((x.numel() + 9,), 3.0, dtype=x.dtype, device=x.device)
        v = y[1:x.numel() + 1].view(x.shape)
        v.copy_(x if fill is None else torch.full_like(x, fill))
        return y, v

    ys = [off(r, -1) for r in ref]
    plan.run([off(x)[1] for x in xs], [v for _, v in ys])
    torch.cuda.synchronize()
    for (whole, v), r in zip(ys, ref):
        assert torch.equal(v, r)
        assert (whole[:1] == 3).all() and (whole[r.numel() + 1:] == 3).all()


def test_outputs_over_inputs():
    import torch
    from block_util import builder, given, inputs, stored
    from paper_1907_01989_amd import _binding as B, engine
    x = stored(np.random.default_rng(2).standard_normal((1, 4, 8, 64)), 0)
    b = builder()
    t = b.rms_norm(given(b, x, 0))
    plan = engine.Plan({"ops": b.ops, "outputs": [t], "output_dtypes": {t: 0}})
    xs = inputs(plan)
    ref = plan.run(xs)[0].clone()
    log("[case] in place")
    plan.run(xs, [xs[0]])                                  # in place: by conversions
    torch.cuda.synchronize()
    assert torch.equal(xs[0], ref)
    # positions and bounds are read while outputs are written: refused
    b = builder()
    xi = given(b, x, 0)
    p = b.index_input(np.zeros((1, 4, 8, 1), np.int32))
    t = b.rotary(xi, 1, 64, [0] * 32, [1.0] * 32, positions=p)
    plan = engine.Plan({"ops": b.ops, "outputs": [t], "output_dtypes": {t: 0}})
    xs = inputs(plan)
    with pytest.raises(B.MgiError, match="overlaps"):
        plan.run(xs, [xs[0]])


def test_bf16_inputs_of_other_operators():
    # a stem, a depthwise layer, a convolution, a 4-bit layer, a pool and questions, from bf16 and from fp32 arrays
    import workloads
    from workloads import NetBuilder
    from gpu_util import run_gpu

    def net(dtype):
        b = NetBuilder(seed=4)
        a = b.input(2, 12, 12, 3, -1, 1, dtype=dtype)
        c = b.input(2, 8, 8, 24, -1, 1, dtype=dtype)
        d = b.input(2, 1, 1, 64, -1, 1, dtype=dtype)
        e = b.input(2, 1, 1, 37, -1, 1, dtype=dtype)
        outs = [b.conv(a, 16, 3, 2), b.dw(c), b.conv(c, 40, 3), b.fc_int4(d, 50), b.fc_int4(e, 50), b.gap(c), b.topk(d, 3),
                b.entropy(e), b.softmax(e)]
        for o in outs:
            b.mark_output(o)
        return workloads.as_bf16_graph(b.graph("bf16_inputs"))

    log("[case] bf16 inputs of other operators")
    _, a, _ = run_gpu(net(1), materialize_all=False, dtype=1)
    _, r, _ = run_gpu(net(2), materialize_all=False, dtype=1)
    for x, y in zip(a, r):
        np.testing.assert_array_equal(x, y)


def test_16_bit_outputs_of_other_operators():
    import torch
    from workloads import NetBuilder
    from paper_1907_01989_amd import engine
    b = NetBuilder(seed=6)
    x = b.input(2, 9, 9, 24, -1, 1)
    outs = [b.conv(x, 30, 1), b.conv(x, 40, 3, 2), b.dw(x), b.add(x, x), b.gap(x)]
    log("[case] 16-bit outputs of other operators")
    for dtype, kind in ((0, torch.float16), (1, torch.bfloat16)):
        desc = {"ops": b.ops, "outputs": outs}
        wide = engine.Plan(desc, dtype=dtype)
        narrow = engine.Plan({**desc, "output_dtypes": {t: dtype for t in outs}}, dtype=dtype)
        a, c = wide.run(wide.input_tensors()), narrow.run(narrow.input_tensors())
        torch.cuda.synchronize()
        for p, q in zip(a, c):
            assert q.dtype == kind and torch.equal(p, q.float())


def test_operators_write_inside_their_buffers():
    from block_util import inputs
    from test_gpu_guards import check_guards, guarded_plan
    # long rows (keys split over workgroups) and odd widths (sliced outputs that are exported)
    for dtype, kw in ((0, dict(n=1, h=1, w=3001, bounds=[0, 2990, 2991, 2991, 3000])), (1, dict(n=3, h=5, w=7))):
        b, t = block(dtype, **kw)
        odd = b.pointwise_fp8(t["tokens"], 77)
        b.ops[odd]["scales"] = b.ops[odd]["scales"] * 0.5
        outs = [t["z"], t["y"], t["turned"], t["tokens"], odd, b.quantize(odd), b.rms_norm(odd)]
        types = {o: dtype for o in outs[:2] + outs[4:]}
        log(f"[case] block guards, type {dtype}")
        for extra in ({}, {"materialize_all": True}, {"fuse": False}):
            plan, ys, raw, ws, lead = guarded_plan({"name": "block", "ops": b.ops, "outputs": outs, "output_dtypes": types}, dtype=dtype, **extra)
            xs = inputs(plan)
            for _ in range(2):
                plan.run(xs, ys)
            check_guards(plan, raw, ws, lead, f"block {dtype} {extra}")


def test_nodes_can_be_read_and_timed():
    import torch
    from block_util import inputs
    from paper_1907_01989_amd import _binding as B
    b, t = block(0, 1, 1, 2600)
    want = ["tokens", "qkv", "turned", "y", "o", "s", "z"]
    plan = plan_of(b, [t["z"]], 0, materialize_all=True)
    xs = inputs(plan)
    log("[case] block, nodes read and timed")
    plan.run(xs)
    read = {info["tensor"]: plan.read_node(i)[1] for i, info in enumerate(plan.nodes()) if info["tensor"] >= 0}
    other = plan_of(b, [t[k] for k in want if k != "tokens"], 0)
    ys = other.run(xs)
    torch.cuda.synchronize()
    for k, y in zip([k for k in want if k != "tokens"], ys):
        assert torch.equal(read[t[k]].reshape(y.shape), y.float()), k
    assert torch.isfinite(read[t["tokens"]]).all()
    # every node's kernels between two events (attention's keys are split: two kernels)
    kinds = [n["kind"] for n in other.nodes()]
    events = [[torch.cuda.Event(enable_timing=True) for _ in kinds] for _ in range(2)]
    for e in events[0] + events[1]:
        e.record()
    again = other.alloc_outputs()
    B.mgi_plan_run_timed(other.handle, [x.data_ptr() for x in xs], [y.data_ptr() for y in again],
                         [e.cuda_event for e in events[0]], [e.cuda_event for e in events[1]], torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    for y, z in zip(again, ys):
        assert torch.equal(y, z)
    times = {k: a.elapsed_time(z) for k, a, z in zip(kinds, *events)}
    assert times["attention"] > 0.005 and all(v < 100 for v in times.values()), times


def test_a_tensor_added_to_itself_and_one_sum_for_two_norms():
    from block_util import HALF, builder, given, run, stored, within
    x = stored(np.random.default_rng(3).standard_normal((1, 3, 5, 72)), 0)
    b = builder()
    s = b.add(given(b, x, 0), 0, act=0)
    n, m = b.rms_norm(s), b.rms_norm(s, eps=0.5)
    log("[case] a tensor added to itself")
    (sv, nv, mv), _ = run(b, [s, n, m], 0, {s: 0})
    np.testing.assert_array_equal(sv, 2 * x)
    for t, v in ((n, nv), (m, mv)):
        ref = oracle.rms_norm(sv, b.ops[t]["w"], b.ops[t]["eps"])
        within(v, ref, (HALF[0] + 2.0 ** -17) * np.abs(ref) + 2.0 ** -25)


@pytest.mark.parametrize("dtype", [0, 1])
def test_channels_past_the_last_stay_zero(dtype):
    import torch
    from block_util import builder, given, inputs, stored
    from paper_1907_01989_amd import _binding as B
    b = builder()
    x = given(b, stored(np.random.default_rng(4).standard_normal((2, 5, 9, 77)), dtype), dtype)
    n = b.rms_norm(x)
    p = b.pointwise_fp8(b.quantize(n), 45)
    s = b.add(n, x, act=0)
    plan = plan_of(b, [p, s], dtype, materialize_all=True)
    plan.run(inputs(plan))
    log(f"[case] padding lanes, type {dtype}")
    seen = 0
    for i, info in enumerate(plan.nodes()):
        if info["tensor"] not in (n, p, s):
            continue
        c = info["shape"][3]
        raw = torch.empty(B.mgi_plan_read_node_raw(plan.handle, i), dtype=torch.uint8, device="cuda:0")
        B.mgi_plan_read_node_raw(plan.handle, i, raw.data_ptr(), torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        lanes = raw.view(torch.int16).reshape(-1, 90, 8)
        assert (lanes[-1, :, c % 8:] == 0).all() and (lanes[-1, :, :c % 8] != 0).any()
        seen += 1
    assert seen == 3


@pytest.mark.parametrize("dtype", [0, 1])
def test_a_trunk_before_and_a_head_behind_tuned_and_captured(dtype):
    # convolutions before the block, its tensors in a concatenation, a depthwise layer, a resize and a head
    from block_util import builder, given, inputs, run, stored
    from paper_1907_01989_amd import engine
    b = builder(11)
    x = given(b, stored(np.random.default_rng(4).uniform(0, 1, (2, 33, 29, 3)), dtype), dtype)
    p = b.conv(b.dw(b.conv(x, 32, 3, 2)), 64)
    n = b.rms_norm(p, to8=True)
    qkv = b.pointwise_fp8(n, 3 * 64)
    r = b.rotary(qkv, 4, 32, [1 + i % 2 for i in range(12)], [0.7 ** i for i in range(12)])
    y = b.attention(r, r, qkv, 2, 2, 32, k_from=64, v_from=128)
    o = b.pointwise_fp8(b.quantize(y), 64, 1)
    s = b.add(p, o)
    z = b.rms_norm(s)
    joined = b.concat([y, z, s])
    d = b.dw(joined)
    small = b.resize(y, 9, 9)
    label = b.argmax(b.conv(small, 24, act=0))
    logits = b.fc(b.gap(b.conv(d, 128)), 40)
    outs = [logits, label, y, z, small, joined]
    log(f"[case] block between a trunk and a head, type {dtype}")
    want, _ = run(b, outs, dtype, fuse=False)
    kept, _ = run(b, outs, dtype, materialize_all=True)
    plan = engine.Plan({"name": "trunk", "ops": b.ops, "outputs": outs}, dtype=dtype)
    xs = inputs(plan)

    def same(ys):
        for a, c in zip(ys, want):
            np.testing.assert_array_equal(a.double().cpu().numpy().reshape(c.shape), c)

    for a, c in zip(kept, want):
        np.testing.assert_array_equal(a, c)
    same(plan.run(xs))
    plan.autotune(xs, reps=2)
    same(plan.run(xs))
    held = plan.capture(xs)
    for _ in range(3):
        for o in held:
            o.fill_(-3)
        plan.replay()
        same(held)


@pytest.mark.parametrize("dtype", [0, 1])
def test_nodes_that_write_16_bit_outputs_are_read_as_fp32(dtype):
    import torch
    from block_util import builder, given, inputs, stored
    b = builder()
    x = given(b, stored(np.random.default_rng(4).standard_normal((1, 3, 5, 77)), dtype), dtype)
    s = b.add(x, x, act=0)
    q = b.quantize(s)
    plan = plan_of(b, [s, q], dtype, materialize_all=True)
    ys = plan.run(inputs(plan))
    log(f"[case] export nodes read, type {dtype}")
    nodes = [i for i, n in enumerate(plan.nodes()) if n["kind"] == "export"]
    assert len(nodes) == 2
    for i, y in zip(nodes, ys):
        assert y.dtype == (torch.float16, torch.bfloat16)[dtype]
        assert torch.equal(plan.read_node(i)[1], y.float())


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("m", [12, 90, 1200])
def test_channels_past_the_last_stay_zero_beside_nan(m, dtype):
    # rows of zeros (whose factor without eps is infinite), with NaN and with infinities
    import torch
    from block_util import builder, given, inputs, stored
    from paper_1907_01989_amd import _binding as B
    b = builder()
    x = stored(np.random.default_rng(4).standard_normal((1, 1, m, 77)), dtype)
    x[0, 0, 1], x[0, 0, 2, 5], x[0, 0, 3, 76] = 0, np.nan, np.inf
    x = given(b, x, dtype)
    n, e = b.rms_norm(x), b.rms_norm(x, eps=0.0)
    s = b.rms_norm(b.add(n, e))
    ps = [b.pointwise_fp8(b.quantize(t), 45) for t in (x, n, e)]
    log(f"[case] {m} rows, padding lanes beside NaN, type {dtype}")
    for kw in ({"materialize_all": True}, {"materialize_all": True, "fuse": False}):
        plan = plan_of(b, [s] + ps, dtype, **kw)
        plan.run(inputs(plan))
        seen = 0
        for i, info in enumerate(plan.nodes()):
            if info["tensor"] not in [n, e, s] + ps:
                continue
            c = info["shape"][3]
            raw = torch.empty(B.mgi_plan_read_node_raw(plan.handle, i), dtype=torch.uint8, device="cuda:0")
            B.mgi_plan_read_node_raw(plan.handle, i, raw.data_ptr(), torch.cuda.current_stream().cuda_stream)
            torch.cuda.synchronize()
            lanes = raw.view(torch.int16).reshape(-1, m, 8)
            assert (lanes[-1, :, c % 8:] == 0).all(), (info, torch.nonzero(lanes[-1, :, c % 8:])[:5])
            seen += 1
        assert seen == 6
