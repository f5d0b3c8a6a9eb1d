"""The pointwise layer in 8 bits against the oracle (64 bits).

Products of codes are exact and so are powers of two.  The matrix instruction adds
the products of eight neighbouring inputs at a time as fixed-point numbers whose last
bit is 2^-13 of the leading one of the largest (measured: of a product 2^-13 times
that of its neighbour the leading bit is left, of a smaller one nothing, of one in
another eight all): up to seven of them lose less than 2^-13 of the largest each.
The sums of eight are added in fp32 in an order of the instruction's own, 16 to a
block; the blocks' sums follow one another, then the bias: with a whole step of
2^-23 for each,
    |error| <= 7 2^-13 sum over eights of the largest |w x| + (16 + K / 128 + 8) 2^-23 sum |w x|,
and half a step of the storage type.
"""
import numpy as np
import pytest

import oracle
from gpu_util import log

pytestmark = pytest.mark.gpu

CASES = [(1, 1, 1), (1, 128, 16), (1, 130, 17), (3, 64, 40), (1, 4096, 256), (5, 1000, 333), (16, 512, 128), (17, 640, 144),
         (33, 256, 1000), (64, 384, 264), (65, 129, 129), (130, 2048, 64), (300, 72, 520), (1, 8192, 24), (2, 16384, 16),
         (257, 1024, 513), (1000, 136, 8)]


def layer(m, cin, cout, dtype, act=0, seed=0, shape=None):
    from block_util import builder, given, stored
    rng = np.random.default_rng([seed, m, cin, cout])
    x = stored(rng.standard_normal(shape or (1, 1, m, cin)) * np.exp(rng.standard_normal((1, 1, 1, cin))), dtype)
    b = builder(m + cin + cout)
    t = b.pointwise_fp8(b.quantize(given(b, x, dtype)), cout, act)
    return b, t, x


def expect(b, t, x, dtype):
    from block_util import HALF, TINY
    op = b.ops[t]
    q = oracle.quantize(x)
    ref = oracle.activation(oracle.pointwise_fp8(q, op["q"], op["scales"], op["b"], op["cout"]), op["act"])
    w = np.abs(oracle.pointwise_fp8_weights(op["q"], op["scales"], op["cout"], x.shape[-1]))
    return ref, HALF[dtype] * np.abs(ref) + TINY[dtype] + sums(q, w, op["b"]) * (1 + HALF[dtype])


def sums(q, w, bias):
    """What the products and their sums may be off by."""
    k = w.shape[1]
    total = np.abs(q) @ w.T + np.abs(bias)
    most = np.zeros_like(total)
    for i in range(0, k, 8):
        some = [np.abs(q[..., j:j + 1]) * w[:, j] for j in range(i, min(i + 8, k))]
        most += np.max(some, axis=0)
    return 7 * 2.0 ** -13 * most + (16 + k / 128 + 8) * 2.0 ** -23 * total


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("m,cin,cout", CASES)
def test_layer(m, cin, cout, dtype):
    from block_util import run, within
    log(f"[case] pointwise_fp8 {m}x{cin}x{cout} type {dtype}")
    b, t, x = layer(m, cin, cout, dtype)
    ref, bound = expect(b, t, x, dtype)
    (y,), _ = run(b, [t], dtype, {t: dtype})
    within(y, ref, bound)
    (f,), _ = run(b, [t], dtype)
    np.testing.assert_array_equal(f, y)
    (f,), _ = run(b, [t], dtype, materialize_all=True, fuse=False)
    np.testing.assert_array_equal(f, y)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("m,cin,cout", [(2000, 200, 2110), (2900, 300, 2900), (16500, 136, 1000), (4200, 1300, 4100), (300, 4000, 500), (150, 2048, 1024)])
def test_tiles(m, cin, cout, dtype):
    # every tile form; some of the rows against the oracle
    from block_util import run, within
    log(f"[case] pointwise_fp8 {m}x{cin}x{cout} type {dtype}")
    b, t, x = layer(m, cin, cout, dtype)
    (y,), _ = run(b, [t], dtype, {t: dtype})
    some = sorted(set(list(range(0, m, m // 40)) + [m - 1, m - 2]))
    ref, bound = expect(b, t, x[:, :, some], dtype)
    within(y[:, :, some], ref, bound)


def test_few_pixels_in_8_bits_by_the_layer_itself_or_before():
    # the same bits with the 8-bit tensor an output, which keeps it
    from block_util import run
    for m, cin, cout in ((1, 4096, 256), (7, 1000, 130), (16, 136, 40)):
        for dtype in (0, 1):
            log(f"[case] pointwise_fp8 {m}x{cin}x{cout} type {dtype}, in one kernel and two")
            b, t, _ = layer(m, cin, cout, dtype, seed=3)
            (y,), plan = run(b, [t], dtype)
            assert [i["kind"] for i in plan.nodes() if "fp8" in i["kind"] or i["kind"] == "quantize"] == ["quantize_pointwise_fp8"]
            (z, _), plan = run(b, [t, t - 1], dtype)
            assert "quantize" in [i["kind"] for i in plan.nodes()]
            np.testing.assert_array_equal(y, z)


@pytest.mark.parametrize("dtype", [0, 1])
def test_extreme_blocks_in_one_kernel_and_two(dtype):
    # blocks of zeros, of the least and the largest values, of subnormals among others, with infinities and NaN
    from block_util import builder, given, run, stored, within
    rng = np.random.default_rng(9)
    x = rng.standard_normal((1, 1, 13, 1024))
    least, most = (2.0 ** -24, 65504.0) if dtype == 0 else (2.0 ** -133, 3.3e38)
    x[0, 0, :, 128:256] = 0
    x[0, 0, :, 256:384] = np.where(rng.random((13, 128)) < 0.5, least, -3 * least)
    x[0, 0, :, 384:512] *= least * 100
    x[0, 0, :, 512:640] = np.where(rng.random((13, 128)) < 0.3, most, -most / 3)
    x[0, 0, :, 640:768] *= 2.0 ** rng.integers(-14, 14, (13, 128))
    x[0, 0, 3, 700], x[0, 0, 5, 900], x[0, 0, 6, 1000] = np.nan, np.inf, -np.inf
    x = stored(x, dtype)
    b = builder(3)
    q = b.quantize(given(b, x, dtype))
    # (a product of the largest values passes fp32's range before the block's scale brings it back)
    t = b.pointwise_fp8(q, 48)
    b.ops[t]["scales"][:, 4] *= 1e-5 if dtype == 0 else 1e-38
    log(f"[case] extreme blocks, type {dtype}")
    (y,), plan = run(b, [t], dtype)
    assert "quantize_pointwise_fp8" in [i["kind"] for i in plan.nodes()]
    (z, v), _ = run(b, [t, q], dtype)
    np.testing.assert_array_equal(y, z)
    with np.errstate(over="ignore"):
        np.testing.assert_array_equal(v, oracle.quantize(x).astype(np.float32))
    bad = [3, 5, 6]
    assert np.isnan(y[0, 0, bad]).all()
    good = [i for i in range(13) if i not in bad]
    ref, bound = expect(b, t, x[:, :, good], dtype)
    within(y[:, :, good], ref, bound)


@pytest.mark.parametrize("act", [1, 2])
def test_activation_and_images(act):
    from block_util import run, within
    log(f"[case] pointwise_fp8 act {act}")
    b, t, x = layer(0, 72, 56, 0, act, shape=(3, 7, 5, 72))
    ref, bound = expect(b, t, x, 0)
    (y,), _ = run(b, [t], 0)
    within(y, ref, bound)


@pytest.mark.parametrize("m", [1, 70])
def test_exponents_far_apart(m):
    # blocks and pixels of very different sizes, scales of both signs, zero among them
    from block_util import builder, given, run, stored, within
    rng = np.random.default_rng(m)
    x = rng.standard_normal((1, 1, m, 1280)) * 2.0 ** np.repeat(rng.integers(-30, 30, (1, 1, m, 10)), 128, -1)
    x[..., 256:384] = 0
    x = stored(x, 1)
    b = builder(7)
    t = b.pointwise_fp8(b.quantize(given(b, x, 1)), 200)
    s = b.ops[t]["scales"]
    s *= 2.0 ** rng.integers(-30, 30, s.shape)
    s[0, 1], s[1, 3] = 0, -s[1, 3]
    log(f"[case] exponents far apart, {m} rows")
    ref, bound = expect(b, t, x, 1)
    (y,), _ = run(b, [t], 1)
    within(y, ref, bound)


def test_a_row_with_nan_is_its_own():
    from block_util import run, within
    b, t, x = layer(20, 300, 60, 0)
    x[0, 0, 7, 299] = np.nan
    x[0, 0, 9, 0] = np.inf
    b.ops[0]["data"] = x
    log("[case] rows with NaN")
    (y,), _ = run(b, [t], 0)
    assert np.isnan(y[0, 0, [7, 9]]).all()
    fine = [i for i in range(20) if i not in (7, 9)]
    x[0, 0, [7, 9]] = 0
    ref, bound = expect(b, t, x, 0)
    within(y[:, :, fine], ref[:, :, fine], bound[:, :, fine])


@pytest.mark.parametrize("dtype", [0, 1])
def test_norm_and_two_layers_share_one_8_bit_tensor(dtype):
    from block_util import HALF, TINY, builder, given, run, stored, within
    rng = np.random.default_rng(4)
    x = stored(rng.standard_normal((2, 5, 9, 200)), dtype)
    b = builder(9)
    n = b.rms_norm(given(b, x, dtype), to8=True)
    p, q = b.pointwise_fp8(n, 96), b.pointwise_fp8(n, 30, 2)
    log(f"[case] two layers of one norm, type {dtype}")
    (nv, pv, qv), plan = run(b, [n, p, q], dtype)
    # (the codes are the kernel's own: test_gpu_norm has them)
    for t, v in ((p, pv), (q, qv)):
        op = b.ops[t]
        w = oracle.pointwise_fp8_weights(op["q"], op["scales"], op["cout"], 200)
        y = oracle.activation(nv @ w.T + op["b"], op["act"])
        bound = HALF[dtype] * np.abs(y) + TINY[dtype] + sums(nv, np.abs(w), op["b"]) * 1.01
        within(v, y, bound)
