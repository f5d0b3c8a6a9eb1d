"""rms_norm, quantize and their fusion with add, against the oracle (64 bits).

fp32 roundings of a norm: a thread adds at most 8 * 2 * 8 squares one after the
other, then six steps across lanes and up to sixteen waves' sums, 150 half steps
of 2^-24 relative to the sum, of which the root halves the effect; the root, the
reciprocal and two products add less than eight: 2^-17 relative to the value
holds them all (128 half steps).  Then one rounding to 16 bits.  A code of 8 bits
may be that of any value within 2^-17 of the exact one.
"""
import numpy as np
import pytest

import oracle
from gpu_util import log

pytestmark = pytest.mark.gpu

FP32 = 2.0 ** -17


def case(n, h, w, c, seed=0, spread=1.0):
    rng = np.random.default_rng([seed, n * h * w, c])
    return rng.standard_normal((n, h, w, c)) * np.exp(rng.standard_normal((n, h, w, 1)) * spread)


def check8(got, y, what):
    """`got`: values of an 8-bit tensor of y, where y is known to FP32."""
    lo, hi = None, None
    for a in (1 - FP32, 1, 1 + FP32):
        for e in (oracle.block_exponents(y * (1 - FP32)), oracle.block_exponents(y * (1 + FP32))):
            v = oracle.quantize(y * a, e)
            lo = v if lo is None else np.minimum(lo, v)
            hi = v if hi is None else np.maximum(hi, v)
    bad = ~((got >= lo) & (got <= hi))
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.size}, first at {np.argwhere(bad)[0]}"
    # (nearly all are the exact one's codes)
    assert (got != oracle.quantize(y)).mean() < 2e-3, what


CASES = [(1, 1, 1, 8), (1, 1, 1, 1), (1, 7, 9, 24), (2, 5, 5, 136), (3, 1, 1, 128), (1, 9, 9, 1000), (1, 1, 63, 181),
         (1, 1, 64, 120), (1, 8, 9, 2048), (1, 1, 3, 4096), (1, 1, 1, 8192), (1, 3, 25, 5000), (1, 1, 1, 16384), (1, 1, 66, 16384),
         (5, 13, 7, 77)]


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("n,h,w,c", CASES)
def test_norm(n, h, w, c, dtype):
    from block_util import HALF, TINY, builder, given, run, stored, within
    log(f"[case] norm {n}x{h}x{w}x{c} type {dtype}")
    x = stored(case(n, h, w, c), dtype)
    b = builder(c)
    t = b.rms_norm(given(b, x, dtype))
    ref = oracle.rms_norm(x, b.ops[t]["w"], b.ops[t]["eps"])
    bound = (HALF[dtype] + FP32) * np.abs(ref) + TINY[dtype]
    (a,), _ = run(b, [t], dtype, {t: dtype})
    within(a, ref, bound, "16-bit output")
    (f,), _ = run(b, [t], dtype)
    np.testing.assert_array_equal(f, a)                  # fp32 output: the stored values
    q = b.rms_norm(t - 1, to8=True)
    b.ops[q]["w"] = b.ops[t]["w"]
    (v,), _ = run(b, [q], dtype)
    check8(v, ref, "8-bit output")


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("c", [72, 130, 256, 1000, 2304])
def test_a_row_is_the_same_among_few_and_many(c, dtype):
    # (pixels are shared out over lanes by their number, the layouts and the type of the output)
    from block_util import builder, given, run, stored
    x = stored(case(1, 1, 2200, c, 5), dtype)

    def outputs(x):
        b = builder(c)
        t = given(b, x, dtype)
        n = b.rms_norm(t)
        s = b.rms_norm(b.add(n, t), to8=True)
        q = b.quantize(n)
        layers = [b.pointwise_fp8(s, 24), b.pointwise_fp8(q, 24)]   # (readers, whose sums have an order of their own)
        return b, [b.rms_norm(t, eps=1e-3), b.rms_norm(b.rms_norm(n), eps=1e-4), s, q] + layers

    rows = [0, 1, 7, 40, 62, 254]
    b, outs = outputs(x[:, :, rows])
    few = run(b, outs, dtype, {t: dtype for t in outs})[0]
    for m in (65, 255, 299, 1023, 1025, 2200):
        some = rows[:5] if m < 255 else rows
        log(f"[case] norm of {m} x {c} type {dtype}")
        b, outs = outputs(x[:, :, :m])
        for y, z in zip(run(b, outs, dtype, {t: dtype for t in outs})[0][:4], few):
            np.testing.assert_array_equal(y[:, :, some], z[:, :, :len(some)])


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("n,h,w,c", CASES[1::2])
@pytest.mark.parametrize("act,to8", [(0, False), (1, True), (2, False), (0, True)])
def test_sum_and_norm_in_one_kernel_or_two(n, h, w, c, dtype, act, to8):
    from block_util import HALF, TINY, builder, given, run, stored, within
    log(f"[case] sum and norm {n}x{h}x{w}x{c} type {dtype} act {act} to8 {to8}")
    b = builder(c)
    x, r = (stored(case(n, h, w, c, s), dtype) for s in (1, 2))
    s = b.add(given(b, x, dtype), given(b, r, dtype))
    b.ops[s]["act"] = act
    t = b.rms_norm(s, to8=to8)
    (hs, y), plan = run(b, [s, t], dtype, {s: dtype} if to8 else {s: dtype, t: dtype})
    assert "add_rms_norm" in [i["kind"] for i in plan.nodes()]
    total = oracle.activation(oracle.add(x, r), act)
    within(hs, total, HALF[dtype] * (1 + FP32) * np.abs(total) + TINY[dtype], "sum")
    ref = oracle.rms_norm(hs, b.ops[t]["w"], b.ops[t]["eps"])
    if to8:
        check8(y, ref, "8-bit norm")
    else:
        within(y, ref, (HALF[dtype] + FP32) * np.abs(ref) + TINY[dtype], "norm")
    # the norm alone an output; no fusion: the same bits
    (again,), _ = run(b, [t], dtype)
    np.testing.assert_array_equal(again, y)
    (h2, y2), plan = run(b, [s, t], dtype, fuse=False)
    assert "rms_norm" in [i["kind"] for i in plan.nodes()]
    np.testing.assert_array_equal(h2, hs)
    np.testing.assert_array_equal(y2, y)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("n,h,w,c", CASES)
def test_quantize_is_exact(n, h, w, c, dtype):
    from block_util import builder, given, run, stored
    log(f"[case] quantize {n}x{h}x{w}x{c} type {dtype}")
    x = stored(case(n, h, w, c, 3, 3.0), dtype)
    x[..., ::5] *= 2.0 ** -9
    x = stored(x, dtype)
    x[..., c // 2:] = 0 if c > 300 else x[..., c // 2:]
    b = builder()
    t = b.quantize(given(b, x, dtype))
    (a,), _ = run(b, [t], dtype)
    np.testing.assert_array_equal(a, oracle.quantize(x))
    (a,), _ = run(b, [t], dtype, materialize_all=True)
    np.testing.assert_array_equal(a, oracle.quantize(x))


def test_quantize_borders():
    # blocks whose largest value is at, just under and just over 448 times a power of two; halves between codes;
    # zeros, subnormals, the largest fp16 and values that are not finite
    from block_util import builder, given, run, stored
    rows = []
    for e in (-20, -8, 0, 5):
        for top in (448, 448.5, 447.5, 256, 224.1, 225):
            row = np.zeros(128)
            row[:30] = np.array([top] + [8.5, 9.5, 10.5, 11.5, 17, 19, 21, 0.015625 * 1.5, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10]
                                + list(np.linspace(-top, top, 18))) * 2.0 ** e
            rows.append(row)
    rows += [np.zeros(128), np.full(128, 2.0 ** -24), np.full(128, 65504.0)]
    odd = np.linspace(-3, 3, 128)
    odd[[3, 50]], odd[7], odd[100] = np.inf, -np.inf, np.nan
    rows += [odd, np.full(128, np.inf)]
    x = stored(np.stack(rows)[None, None], 0)
    b = builder()
    t = b.quantize(given(b, x, 0))
    log("[case] quantize borders")
    (a,), _ = run(b, [t], 0)
    np.testing.assert_array_equal(a, oracle.quantize(x))


@pytest.mark.parametrize("dtype", [0, 1])
def test_rows_of_zeros_and_of_extremes(dtype):
    from block_util import HALF, TINY, builder, given, run, stored, within
    big = 60000.0 if dtype == 0 else 1e18
    x = np.random.default_rng(5).standard_normal((1, 1, 70, 264))
    x[0, 0, 0], x[0, 0, 1] = 0, big
    x[0, 0, 2] *= 1e-6
    x[0, 0, 3, 5] = np.nan
    x[0, 0, 4, 6] = np.inf
    x = stored(x, dtype)
    b = builder()
    t = b.rms_norm(given(b, x, dtype))
    log(f"[case] extremes type {dtype}")
    (y,), _ = run(b, [t], dtype)
    with np.errstate(invalid="ignore"):
        ref = oracle.rms_norm(x, b.ops[t]["w"], b.ops[t]["eps"])
    assert (y[0, 0, 0] == 0).all()
    # the other rows are their own
    fine = [i for i in range(70) if i not in (3, 4)]
    within(y[:, :, fine], ref[:, :, fine], (HALF[dtype] + FP32) * np.abs(ref[:, :, fine]) + TINY[dtype])
    assert np.isnan(y[0, 0, 3]).all() and np.isnan(y[0, 0, 4, 6])


def test_norm_of_tensors_inside_a_network():
    # behind a convolution, from fp32 inputs, into a concatenation and an add
    from block_util import HALF, builder, given, run, stored, within
    b = builder(3)
    x = given(b, stored(case(2, 6, 5, 24), 0), 2)
    c = b.conv(x, 40, 1, act=0)
    t = b.rms_norm(c)
    o = b.concat([b.rms_norm(x), t])
    s = b.add(t, c)
    u = b.rms_norm(s)
    log("[case] norms in a network")
    (cv, tv, ov, sv, uv), _ = run(b, [c, t, o, s, u], 0)
    ref = oracle.rms_norm(cv, b.ops[t]["w"], 1e-6)
    within(tv, ref, (HALF[0] + FP32) * np.abs(ref) + 2.0 ** -25)
    np.testing.assert_array_equal(ov[..., 24:], tv)
    ref = oracle.rms_norm(sv, b.ops[u]["w"], 1e-6)
    within(uv, ref, (HALF[0] + FP32) * np.abs(ref) + 2.0 ** -25)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("act", [0, 1, 2])
@pytest.mark.parametrize("to8", [False, True])
def test_a_sum_leaves_nan_and_infinities_as_they_are(act, to8, dtype):
    # in either operand, and of infinities of both signs: one value of a row, whose norm it reaches
    from block_util import HALF, TINY, builder, given, run, stored, within
    rng = np.random.default_rng(8)
    for m, c in ((9, 40), (1100, 72)):
        x, r = (stored(rng.standard_normal((1, 1, m, c)), dtype) for _ in range(2))
        x[0, 0, 1, 3], r[0, 0, 2, c - 1] = np.nan, np.nan
        x[0, 0, 3, 0], r[0, 0, 4, 5] = np.inf, -np.inf
        x[0, 0, 5, 7], r[0, 0, 5, 7] = np.inf, -np.inf
        b = builder(c)
        s = b.add(given(b, x, dtype), given(b, r, dtype))
        b.ops[s]["act"] = act
        t = b.rms_norm(s, to8=to8)
        log(f"[case] {m} x {c}: a sum with NaN and infinities, type {dtype} act {act} to8 {to8}")
        with np.errstate(invalid="ignore"):
            total = x + r if act == 0 else np.clip(x + r, 0, (np.inf, 6)[act - 1])     # (which keeps NaN)
            assert np.isnan(total[0, 0, [1, 2, 5]]).any(-1).all()
            for kw in ({}, {"fuse": False}, {"materialize_all": True}):
                (hs, y), _ = run(b, [s, t], dtype, **kw)
                within(hs, total, np.where(np.isfinite(total), HALF[dtype] * (1 + FP32) * np.abs(total) + TINY[dtype], 0), f"sum {kw}")
                ref = oracle.rms_norm(hs, b.ops[t]["w"], b.ops[t]["eps"])
                if to8:
                    np.testing.assert_array_equal(np.isnan(y), np.isnan(ref), err_msg=f"norm {kw}")
                else:
                    within(y, ref, np.where(np.isfinite(ref), (HALF[dtype] + FP32) * np.abs(ref) + TINY[dtype], 0), f"norm {kw}")
                (alone,), _ = run(b, [t], dtype, **kw)
                np.testing.assert_array_equal(alone, y)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("to8", [False, True])
def test_rows_of_the_least_and_largest_values_without_eps(to8, dtype):
    # (1 / rms passes fp32's range, or is none of its normal values; the norm is about 1 all the same).  The squares
    # and their root are 64-bit: the factor's rounding and two products, three half steps of fp32, are 2^-22
    from block_util import HALF, TINY, builder, given, run, stored, within
    rng = np.random.default_rng(6)
    least = (2.0 ** -24, 2.0 ** -133)[dtype]
    for m, c in ((7, 72), (1100, 40), (3, 4100)):
        x = rng.standard_normal((1, 1, m, c))
        x[0, 0, 0] = least * rng.integers(-3, 4, c)                     # zeros among the least
        x[0, 0, 1] = least * rng.choice([-1, 1], c)
        x[0, 0, 2] = np.where(rng.random(c) < 0.5, 1, -0.6) * (6e4, 3.3e38)[dtype]
        for i in range(3, m):
            x[0, 0, i] *= 2.0 ** rng.integers((-14, -126)[dtype], (12, 124)[dtype])
        x = stored(x, dtype)
        b = builder(c)
        t = b.rms_norm(given(b, x, dtype), eps=0.0, to8=to8)
        b.ops[t]["w"] = np.exp(rng.standard_normal(c)).astype(np.float32)
        ref = oracle.rms_norm(x, b.ops[t]["w"], 0.0)
        log(f"[case] {m} x {c} of extremes, no eps, type {dtype} to8 {to8}")
        (y,), _ = run(b, [t], dtype)
        assert np.isfinite(ref).all()
        if to8:
            check8(y, ref, "8-bit")
        else:
            within(y, ref, (HALF[dtype] + 2.0 ** -22) * np.abs(ref) + TINY[dtype])


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("n,h,w,c", CASES)
def test_norm_to_three_roundings(n, h, w, c, dtype):
    # (as above: the squares and their root are 64-bit)
    from block_util import HALF, TINY, builder, given, run, stored, within
    log(f"[case] norm {n}x{h}x{w}x{c} type {dtype}, 2^-22")
    x = stored(case(n, h, w, c, 11, 4.0), dtype)
    b = builder(c)
    t = b.rms_norm(given(b, x, dtype), eps=1e-5)
    ref = oracle.rms_norm(x, b.ops[t]["w"], b.ops[t]["eps"])
    (y,), _ = run(b, [t], dtype)
    within(y, ref, (HALF[dtype] + 2.0 ** -22) * np.abs(ref) + TINY[dtype])


@pytest.mark.parametrize("dtype", [0, 1])
def test_a_sum_that_only_its_norm_reads(dtype):
    # (not stored) the same bits as where others read it: one or two of them, an output, a part of a concatenation
    from block_util import builder, given, run, stored
    rng = np.random.default_rng(12)
    x, r = (stored(rng.standard_normal((2, 9, 11, 72)), dtype) for _ in range(2))

    def net(more, to8):
        b = builder(2)
        s = b.add(given(b, x, dtype), given(b, r, dtype))
        t = b.rms_norm(s, to8=to8)
        y = b.pointwise_fp8(t, 40) if to8 else b.dw(t)
        b.ops[t]["w"] = np.linspace(0.5, 1.5, 72).astype(np.float32)
        outs = [y, t]
        if more == "output":
            outs.append(s)
        elif more == "reader":
            outs.append(b.conv(s, 16))
        elif more == "concat":
            outs.append(b.conv(b.concat([s, b.dw(s)]), 16))
        if to8:
            b.ops[y].update(q=np.full((40, 72), 0x38, np.uint8), scales=np.ones((1, 1), np.float32), b=None)
        else:
            b.ops[y].update(w=np.ones((72, 3, 3), np.float32), b=None)
        return b, outs

    for to8 in (False, True):
        first = None
        for more in ("nothing", "output", "reader", "concat"):
            log(f"[case] a sum read by its norm and {more}, type {dtype} to8 {to8}")
            for kw in ({}, {"fuse": False}):
                got, plan = run(*net(more, to8), dtype, **kw)
                assert ("add_rms_norm" in [i["kind"] for i in plan.nodes()]) == (not kw)
                first = first or got[:2]
                for a, c in zip(got, first):
                    np.testing.assert_array_equal(a, c)


@pytest.mark.parametrize("dtype", [0, 1])
def test_values_next_to_the_largest_in_8_bits(dtype):
    # stand for the power of two past the type's range: an infinity in a 16-bit array, in fp32 that of fp16 is there
    from block_util import TORCH, builder, given, run, stored
    import torch
    top = (2.0 ** 15, 2.0 ** 127)[dtype]
    x = np.zeros((1, 1, 6, 130))
    x[0, 0, :, 7] = top * np.array([1.75, 1.875, 1.921875, 1.9375, 1.9921875, -1.9921875])
    x[..., 128:] = 3
    x = stored(x, dtype)
    assert np.isfinite(x).all()
    ref = oracle.quantize(x)
    assert ref[0, 0, 2, 7] == 1.875 * top and ref[0, 0, 3, 7] == 2 * top and ref[0, 0, 5, 7] == -2 * top
    b = builder()
    t = b.quantize(given(b, x, dtype))
    log(f"[case] quantize next to the largest, type {dtype}")
    (wide,), _ = run(b, [t], dtype)
    (narrow,), _ = run(b, [t], dtype, {t: dtype})
    with np.errstate(over="ignore"):
        np.testing.assert_array_equal(wide, ref.astype(np.float32).astype(np.float64))
    np.testing.assert_array_equal(narrow, torch.from_numpy(ref).to(TORCH[dtype]).double().numpy())
    assert np.isinf(narrow[0, 0, 3:, 7]).all() and np.isfinite(narrow[0, 0, :3]).all()


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("n,h,w,c", CASES + [(1, 1, 2500, 264)])
def test_codes_of_a_norm_are_the_exact_norms(n, h, w, c, dtype):
    # (rounded to fp32 once and then to 8 bits: another code only within half a step of 2^-23 of a border between two)
    from block_util import builder, given, run, stored
    x = stored(case(n, h, w, c, 13), dtype)
    b = builder(c)
    t = b.rms_norm(given(b, x, dtype), eps=1e-5, to8=True)
    ref = oracle.rms_norm(x, b.ops[t]["w"], b.ops[t]["eps"])
    log(f"[case] codes of a norm {n}x{h}x{w}x{c} type {dtype}")
    (y,), _ = run(b, [t], dtype)
    near = 2.0 ** -24
    same = [oracle.quantize(ref * a, oracle.block_exponents(ref * e)) for a in (1 - near, 1 + near) for e in (1 - near, 1 + near)]
    lo, hi = np.minimum.reduce(same), np.maximum.reduce(same)
    assert ((y >= lo) & (y <= hi)).all(), int((~((y >= lo) & (y <= hi))).sum())
    assert (lo != hi).mean() < 1e-4 or y.size < 10000


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("c", [640, 16384])
def test_codes_of_a_norm_next_to_borders(c, dtype):
    # weights that bring every channel within a step of fp32 of the middle between two codes: the codes are those of
    # the exact norm rounded to fp32 (two products would cross the middle for a third of them)
    from block_util import builder, given, run, stored
    rng = np.random.default_rng(c)
    x = stored(case(1, 1, 1, c, 14) + 0.1, dtype)
    x[x == 0] = 1
    f = 1 / np.sqrt((x * x).mean() + np.float64(np.float32(1e-5)))
    middle = (8.5 + rng.integers(0, 8, c)) / 8 * 2.0 ** rng.integers(-3, 4, c)
    middle[::128] = 300                                             # (each block's exponent is 0)
    w = (middle / (x.reshape(-1) * f)).astype(np.float32)
    ref = (x * f * w.astype(np.float64)).astype(np.float32).astype(np.float64)
    b = builder(c)
    t = b.rms_norm(given(b, x, dtype), eps=1e-5, to8=True)
    b.ops[t]["w"] = w
    log(f"[case] codes of a norm next to borders, {c} channels, type {dtype}")
    (y,), _ = run(b, [t], dtype)
    np.testing.assert_array_equal(y, oracle.quantize(ref))
