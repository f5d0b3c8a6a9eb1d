"""Helpers of the attention block's tests: graph inputs with given values, runs,
and the roundings that results may differ by."""
import numpy as np
import torch

from workloads import NetBuilder

# half a step of each storage type relative to the value, and of its subnormals
HALF = {0: 2.0 ** -11, 1: 2.0 ** -8}
TINY = {0: 2.0 ** -25, 1: 2.0 ** -133}
TORCH = {0: torch.float16, 1: torch.bfloat16}


def stored(x, dtype):
    """The values of x in the storage type (0 fp16, 1 bf16), as float64."""
    return torch.from_numpy(np.asarray(x, np.float64)).to(TORCH[dtype]).double().numpy()


def given(b, x, dtype):
    """A graph input with these values; ``dtype``: its element type (0 fp16, 1 bf16, 2 fp32)."""
    x = np.asarray(x, np.float64)
    return b._push({"op": "input", "name": f"input{len(b.ops)}", "shape": x.shape, "data": x, "dtype": dtype}, x.shape[1:])


def run(b, outputs, dtype, types=None, **kw):
    """The outputs of a fresh plan as float64 arrays of the tensors' shapes, and the plan."""
    from paper_1907_01989_amd import engine
    import oracle
    desc = {"name": "block", "ops": b.ops, "outputs": list(outputs), "output_dtypes": types or {}}
    plan = engine.Plan(desc, dtype=dtype, **kw)
    got = plan.run(inputs(plan))
    torch.cuda.synchronize()
    shapes = oracle.tensor_shapes(desc)
    return [g.double().cpu().numpy().reshape(shapes[t]) for g, t in zip(got, outputs)], plan


def inputs(plan):
    """Device copies of the description's input arrays (also of values that only bf16 has)."""
    xs = []
    for op in plan.desc["ops"]:
        if op["op"] == "input":
            dt = {0: torch.float16, 1: torch.bfloat16, 2: torch.float32}[op["dtype"]]
            xs.append(torch.from_numpy(np.ascontiguousarray(op["data"])).to(dt).to(plan.device))
        elif op["op"] == "index_input":
            xs.append(torch.from_numpy(np.ascontiguousarray(op["data"], dtype=np.int32)).to(plan.device))
    return xs


def within(got, ref, bound, what=""):
    """Every value within its bound of the reference's; NaN and infinities where that has them."""
    got, ref = np.asarray(got, np.float64), np.asarray(ref, np.float64)
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    fine = np.isfinite(ref)
    np.testing.assert_array_equal(np.isnan(got), np.isnan(ref), err_msg=what)
    np.testing.assert_array_equal(got[~fine & ~np.isnan(ref)], ref[~fine & ~np.isnan(ref)], err_msg=what)
    off = np.where(fine, np.abs(np.where(fine, got, 0) - np.where(fine, ref, 0)) - bound, -1)
    assert (off <= 0).all(), f"{what}: {int((off > 0).sum())} of {off.size} out of bound, worst by {off.max():.3e} at {np.unravel_index(off.argmax(), off.shape)}"


def builder(seed=0):
    return NetBuilder(seed=seed)
