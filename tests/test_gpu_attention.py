"""Attention against the oracle (64 bits).

A score is a sum of D products in fp32, off by at most (D + 4) 2^-24 times the sum
of the products' magnitudes (a whole step of 2^-23 for each halving is included
below), which changes a weight by that much relative to it, and so do 2^-18 for
the exponential, its argument and the sums.  The weights are rounded to the
storage type: half a step relative to each, or 2^-25 (fp16) where they are its
subnormals.  So, with the sum of weights S and r the largest score error,
    |error| <= (half + 2 r + 2^-18) sum p |v| / S + 2^-25 sum |v| + half |y|.
"""
import numpy as np
import pytest

import oracle
from gpu_util import log

pytestmark = pytest.mark.gpu


def tensors(rng, q, k, heads, kv, dim, dtype, size=1.0):
    from block_util import stored
    return [stored(rng.standard_normal(s + (m * dim,)) * size, dtype) for s, m in ((q, heads), (k, kv), (k, kv))]


def graph(q, k, v, dtype, heads, kv, dim, bounds=None, k_bounds=None, **kw):
    from block_util import builder, given
    b = builder()
    ids = [given(b, t, dtype) for t in (q, k, v)]
    for name, values in (("bounds", bounds), ("k_bounds", k_bounds)):
        if values is not None:
            kw[name] = b.index_input(np.asarray(values).reshape(1, 1, 1, -1))
    return b, b.attention(*ids, heads, kv, dim, **kw)


def check(q, k, v, dtype, heads, kv, dim, got, bounds=None, k_bounds=None, causal=False, scale=0.0, what=""):
    from block_util import HALF, within
    ref, size = oracle.attention(q, k, v, heads, kv, dim, causal, scale, bounds, k_bounds, weight_of=np.abs)
    s = abs(scale or dim ** -0.5)
    norm = [np.sqrt(np.square(np.where(np.isfinite(t), t, 0).reshape(-1, dim)).sum(1)).max() for t in (q, k)]
    worst = norm[0] * norm[1]                     # (no sum of |q_i k_i| is larger)
    r = (dim + 4) * 2.0 ** -24 * s * worst
    total = np.abs(np.where(np.isfinite(v), v, 0)).sum() if dtype == 0 else 0.0
    with np.errstate(invalid="ignore"):
        bound = (HALF[dtype] + 2 * r + 2.0 ** -18) * size + HALF[dtype] * np.abs(ref) + 2.0 ** -25 * (total + 1)
    within(got, ref, np.where(np.isfinite(bound), bound, 0), what)
    return ref


IMAGES = [
    # n, q plane, k plane, heads, kv, dim, causal
    (1, (1, 1), (1, 1), 1, 1, 8, False), (2, (7, 7), (7, 7), 4, 4, 32, False), (3, (5, 9), (5, 9), 8, 1, 64, True),
    (2, (14, 14), (7, 7), 8, 2, 64, False), (1, (1, 1), (1, 300), 8, 2, 128, True), (2, (1, 65), (1, 64), 2, 1, 80, False),
    (1, (1, 130), (1, 200), 3, 1, 16, True), (1, (1, 70), (1, 20), 2, 2, 40, True), (1, (1, 129), (1, 129), 5, 5, 24, True),
    (4, (1, 1), (1, 1), 6, 3, 96, True), (1, (1, 64), (1, 64), 1, 1, 128, False), (1, (3, 11), (1, 1), 4, 2, 72, False),
    (2, (1, 3), (1, 1000), 16, 2, 64, False), (1, (1, 1), (1, 5000), 4, 1, 64, False), (1, (1, 2), (1, 3000), 64, 1, 32, True),
    (1, (1, 40), (1, 2500), 2, 2, 128, True),
]


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("n,q,k,heads,kv,dim,causal", IMAGES)
def test_images(n, q, k, heads, kv, dim, causal, dtype):
    from block_util import run
    log(f"[case] attention {n} x {q} on {k} heads {heads}/{kv} x {dim} causal {causal} type {dtype}")
    t = tensors(np.random.default_rng([n, heads, dim]), (n,) + q, (n,) + k, heads, kv, dim, dtype)
    b, a = graph(*t, dtype, heads, kv, dim, causal=causal)
    (y,), _ = run(b, [a], dtype, {a: dtype})
    check(*t, dtype, heads, kv, dim, y, causal=causal)
    (f,), _ = run(b, [a], dtype, materialize_all=True, fuse=False)     # sliced operands: the same bits
    np.testing.assert_array_equal(f, y)


@pytest.mark.parametrize("dim", range(8, 129, 8))
def test_every_head_size_over_several_tiles(dim):
    from block_util import run
    for q, k in (((1, 140), (1, 333)), ((1, 1), (1, 700))):
        log(f"[case] attention {q} on {k} heads of {dim}")
        t = tensors(np.random.default_rng(dim), (2,) + q, (2,) + k, 2, 1, dim, dim // 8 % 2)
        b, a = graph(*t, dim // 8 % 2, 2, 1, dim, causal=dim % 3 == 0)
        (y,), _ = run(b, [a], dim // 8 % 2, {a: dim // 8 % 2})
        check(*t, dim // 8 % 2, 2, 1, dim, y, causal=dim % 3 == 0)


PACKED = [
    # bounds, k_bounds, pixels, k pixels
    ([0, 5], None, 5, 5), ([0, 64, 128, 129, 129, 300], None, 300, 300), ([3, 10, 10, 200], None, 210, 210),
    ([0, 1, 2, 3, 4, 5, 6, 7], None, 9, 9), ([0, 33, 166], [0, 1, 400], 166, 400), ([0, 100, 150], [0, 0, 50], 150, 64),
    ([0, 70, 30, 90], None, 100, 100), ([-5, 20, 1000], None, 60, 60), ([50, 50, 50], None, 50, 50),
    ([0, 1, 2, 3], [0, 700, 700, 1500], 3, 1500),
]


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("bounds,k_bounds,nq,nk", PACKED)
def test_packed(bounds, k_bounds, nq, nk, causal, dtype):
    from block_util import run
    log(f"[case] attention packed {bounds} {k_bounds} of {nq}, {nk} causal {causal} type {dtype}")
    t = tensors(np.random.default_rng(nq), (1, 1, nq), (1, 1, nk), 4, 2, 64, dtype)
    b, a = graph(*t, dtype, 4, 2, 64, bounds, k_bounds, causal=causal)
    (y,), _ = run(b, [a], dtype)
    check(*t, dtype, 4, 2, 64, y, bounds, k_bounds, causal)


def test_many_sequences():
    from block_util import run
    rng = np.random.default_rng(8)
    bounds = np.concatenate([[0], rng.integers(0, 5, 300).cumsum()])
    rows = int(bounds[-1]) + 7
    t = tensors(rng, (1, 1, rows), (1, 1, rows), 2, 1, 16, 0)
    b, a = graph(*t, 0, 2, 1, 16, bounds, causal=True)
    log("[case] attention of 300 sequences")
    (y,), _ = run(b, [a], 0)
    check(*t, 0, 2, 1, 16, y, bounds, causal=True)
    assert (y[0, 0, -7:] == 0).all()


@pytest.mark.parametrize("scale", [0.3, -0.2, 4.0])
def test_scales(scale):
    from block_util import run
    log(f"[case] attention scale {scale}")
    t = tensors(np.random.default_rng(3), (1, 1, 100), (1, 1, 150), 2, 2, 32, 0)
    b, a = graph(*t, 0, 2, 2, 32, scale=scale)
    (y,), _ = run(b, [a], 0)
    check(*t, 0, 2, 2, 32, y, scale=scale)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("queries", [130, 3])
def test_hidden_keys_and_values_have_no_part(queries, dtype):
    # keys and values that are infinite or NaN, each hidden from the queries before it
    from block_util import run
    n = 300
    rng = np.random.default_rng(6)
    q, k, v = tensors(rng, (1, 1, queries), (1, 1, n), 4, 2, 64, dtype)
    first = n - queries + 1                        # the first key that not every query sees
    k[0, 0, first + 1, 3] = np.nan
    v[0, 0, n - 1, 5] = np.inf                     # seen by the last query only
    v[0, 0, first, 70] = -np.inf
    v[0, 0, first + 1, 100] = np.nan
    b, a = graph(q, k, v, dtype, 4, 2, 64, causal=True)
    log(f"[case] attention hidden infinities, {queries} queries, type {dtype}")
    (y,), _ = run(b, [a], dtype)
    check(q, k, v, dtype, 4, 2, 64, y, causal=True)
    # and behind the end of a sequence, and outside all of them
    bounds = [0, 100, 200]
    q, k, v = tensors(rng, (1, 1, n), (1, 1, n), 4, 2, 64, dtype)
    for t in (k, v):
        t[0, 0, 200:], t[0, 0, 150] = np.nan, np.inf
    b, a = graph(q, k, v, dtype, 4, 2, 64, bounds)
    (y,), _ = run(b, [a], dtype)
    fine = list(range(100)) + list(range(200, n))
    k2, v2 = np.where(np.isfinite(k), k, 0), np.where(np.isfinite(v), v, 0)
    ref, size = oracle.attention(q, k2, v2, 4, 2, 64, bounds=bounds, weight_of=np.abs)
    assert np.isfinite(y[0, 0, fine]).all() and (y[0, 0, 200:] == 0).all()
    np.testing.assert_allclose(y[0, 0, :100], ref[0, 0, :100], atol=0.02)


def test_extreme_scores():
    # one key far above the others; scores that overflow 16 bits; equal keys
    from block_util import run, stored
    rng = np.random.default_rng(2)
    q, k, v = tensors(rng, (1, 1, 40), (1, 1, 200), 1, 1, 64, 0)
    k[0, 0, 77] *= 30
    q[0, 0, 3] *= 100
    k[0, 0, 100:] = k[0, 0, 100]
    q, k = stored(q, 0), stored(k, 0)
    b, a = graph(q, k, v, 0, 1, 1, 64)
    log("[case] attention extreme scores")
    (y,), _ = run(b, [a], 0)
    check(q, k, v, 0, 1, 1, 64, y)


def test_one_tensor_for_queries_keys_and_values():
    from block_util import builder, given, run, stored
    x = stored(np.random.default_rng(9).standard_normal((2, 6, 7, (4 + 2 + 2) * 24 + 8)), 0)
    b = builder()
    t = given(b, x, 0)
    a = b.attention(t, t, t, 4, 2, 24, q_from=8, k_from=8 + 96, v_from=8 + 144)
    log("[case] attention of one tensor")
    (y,), _ = run(b, [a], 0)
    check(x[..., 8:104], x[..., 104:152], x[..., 152:200], 0, 4, 2, 24, y)


def tight(q, k, v, dtype, heads, kv, dim, got, bounds=None, k_bounds=None, causal=False, scale=0.0, what=""):
    """``check`` with a bound of each row and channel's own: fp16 weights are off by half a step of 2^-11, or where
    that is more by half of 2^-31 of the row's largest (they are kept as 2^7 times that and more, in steps of 2^-24):
        |error| <= (half + 2 r + 2^-18) sum p |v| / S + 2^-32 sum |v| + half |y|, the sums over the keys that a row sees
    (S, the weights' sum, is at least the largest's 1)."""
    from block_util import HALF, TINY, within
    args = (heads, kv, dim, causal)
    ref, size = oracle.attention(q, k, v, *args, scale, bounds, k_bounds, weight_of=np.abs)
    # (equal weights give means)
    _, mean = oracle.attention(np.zeros_like(q), k, v, *args, scale, bounds, k_bounds, weight_of=np.abs)
    count = np.zeros(ref.shape[:3]).reshape(-1)
    nq, nk = int(np.prod(q.shape[:3])), int(np.prod(k.shape[:3]))
    for q0, q1, k0, k1 in oracle.attention_spans(nq, nk, q.shape[0], bounds, k_bounds):
        for i in range(q0, q1):
            count[i] = min(max(i - q0 + 1 + (k1 - k0) - (q1 - q0), 0), k1 - k0) if causal else k1 - k0
    norm = [np.sqrt(np.square(t.reshape(-1, dim)).sum(1)).max() for t in (q, k)]
    r = (dim + 4) * 2.0 ** -24 * abs(scale or dim ** -0.5) * norm[0] * norm[1]
    lost = 2.0 ** -32 * mean * count.reshape(ref.shape[:3] + (1,)) if dtype == 0 else 0.0
    within(got, ref, (HALF[dtype] + 2 * r + 2.0 ** -18) * size + lost + HALF[dtype] * np.abs(ref) + TINY[dtype], what)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("queries,heads", [(1, 1), (1024, 64)])
@pytest.mark.parametrize("bits", [12, 20, 25, 27, 30])
def test_many_keys_of_small_weights(bits, queries, heads, dtype):
    # one key far above 50000 others, whose weights are 2^-bits of its own (keys split over workgroups or in one)
    from block_util import run, stored
    rng = np.random.default_rng(bits)
    n, dim, top = 50000, 8, 777
    q = np.zeros((1, 1, queries, heads * dim))
    q[..., ::dim] = 1
    k, v = np.zeros((1, 1, n, dim)), 1 + 0.2 * rng.standard_normal((1, 1, n, dim))
    k[..., 0], v[..., top, :] = -16, 0
    k[0, 0, top, 0] = -16 + bits                                       # (scores in units of log2: scale)
    q, k, v = (stored(t, dtype) for t in (q, k, v))
    scale = float(np.float32(np.log(2)))
    b, a = graph(q, k, v, dtype, heads, 1, dim, scale=scale)
    log(f"[case] attention on 50000 keys of weight 2^-{bits}, {queries} queries of {heads} heads, type {dtype}")
    (y,), _ = run(b, [a], dtype)
    one = y[:, :, :1, :dim]
    tight(q[:, :, :1, :dim], k, v, dtype, 1, 1, dim, one, scale=scale)
    np.testing.assert_array_equal(y.reshape(-1, dim), np.broadcast_to(one[0, 0], (queries * heads, dim)))


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("n,q,k,heads,kv,dim,causal", IMAGES)
def test_images_to_their_own_bounds(n, q, k, heads, kv, dim, causal, dtype):
    from block_util import run
    log(f"[case] attention {n} x {q} on {k} heads {heads}/{kv} x {dim} causal {causal} type {dtype}, own bounds")
    t = tensors(np.random.default_rng([n, heads, dim, 5]), (n,) + q, (n,) + k, heads, kv, dim, dtype, 1.5)
    b, a = graph(*t, dtype, heads, kv, dim, causal=causal)
    (y,), _ = run(b, [a], dtype, {a: dtype})
    tight(*t, dtype, heads, kv, dim, y, causal=causal)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("bounds,k_bounds,nq,nk", PACKED)
def test_packed_to_their_own_bounds(bounds, k_bounds, nq, nk, causal, dtype):
    from block_util import run
    log(f"[case] attention packed {bounds} {k_bounds} of {nq}, {nk} causal {causal} type {dtype}, own bounds")
    t = tensors(np.random.default_rng([nq, 7]), (1, 1, nq), (1, 1, nk), 4, 2, 64, dtype, 1.5)
    b, a = graph(*t, dtype, 4, 2, 64, bounds, k_bounds, causal=causal)
    (y,), _ = run(b, [a], dtype)
    tight(*t, dtype, 4, 2, 64, y, bounds, k_bounds, causal)


ODD = [
    # queries, keys, heads, kv, dim, causal, bounds: tiles that waves share, keys of each wave, both split over workgroups
    (130, 300, 4, 2, 64, False, None), (130, 300, 2, 1, 96, True, None), (3, 300, 4, 2, 64, False, None), (1, 5000, 4, 1, 128, True, None),
    (40, 2500, 2, 2, 32, False, None), (300, 300, 8, 8, 80, False, [0, 100, 101, 290]), (3000, 3000, 1, 1, 40, True, [0, 2900, 2990]),
    (1100, 900, 16, 1, 8, True, None),
]


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("nq,nk,heads,kv,dim,causal,bounds", ODD)
def test_values_that_are_infinite_or_nan_and_seen(nq, nk, heads, kv, dim, causal, bounds, dtype):
    # of keys whose weight is nothing beside later and earlier ones', and of ordinary ones: a result's channel is what
    # its keys have there, wherever the keys are among tiles, waves and workgroups
    from block_util import run
    rng = np.random.default_rng([nq, nk, dim])
    q, k, v = tensors(rng, (1, 1, nq), (1, 1, nk), heads, kv, dim, dtype)
    q[..., ::dim] = 40
    far = rng.random(nk) < 0.5                         # weights of exp(-200) and less
    far[[0, nk // 2, nk - 1]] = True, False, False
    k[..., ::dim] = np.where(far, 0, 5 * dim ** 0.5)[:, None]
    rows = sorted(set(rng.choice(nk, 12)) | {0, nk - 1})
    for i, j in enumerate(rows):
        v[0, 0, j, rng.integers(kv * dim)] = (np.inf, -np.inf, np.nan)[i % 3]
    v[0, 0, rows[1], 1], v[0, 0, rows[-2], 1] = np.inf, -np.inf
    odd = np.where(np.isfinite(v), 0, v)
    fine = np.where(np.isfinite(v), v, 0)
    ref, size = oracle.attention(q, k, fine, heads, kv, dim, causal, 0.0, bounds, weight_of=np.abs)
    ref = ref.reshape(nq, heads, dim)
    seen = np.zeros(ref.shape)
    of = odd.reshape(nk, kv, dim)
    with np.errstate(invalid="ignore"):
        for q0, q1, k0, k1 in oracle.attention_spans(nq, nk, 1, bounds):
            total = np.concatenate([np.zeros((1, kv, dim)), np.cumsum(of[k0:k1], 0)])
            for i in range(q0, q1):
                end = min(max(i - q0 + 1 + (k1 - k0) - (q1 - q0), 0), k1 - k0) if causal else k1 - k0
                seen[i] = np.repeat(total[end], heads // kv, 0)
        ref = np.where(seen != 0, seen, ref).reshape(1, 1, nq, heads * dim)
    assert np.isposinf(ref).any() and np.isneginf(ref).any() and np.isnan(ref).any() and np.isfinite(ref).any()
    b, a = graph(q, k, v, dtype, heads, kv, dim, bounds, causal=causal)
    log(f"[case] attention, infinities that are seen, {nq} on {nk}, {heads}/{kv} x {dim} causal {causal} {bounds} type {dtype}")
    (y,), _ = run(b, [a], dtype, {a: dtype})
    from block_util import HALF, within
    r = (dim + 4) * 2.0 ** -24 * dim ** -0.5 * np.sqrt(np.square(q.reshape(-1, dim)).sum(1)).max() * np.sqrt(np.square(k.reshape(-1, dim)).sum(1)).max()
    bound = (HALF[dtype] + 2 * r + 2.0 ** -18) * size + HALF[dtype] * np.where(np.isfinite(ref), np.abs(ref), 0) + 2.0 ** -32 * np.abs(fine).sum()
    within(y, ref, bound)
    (f,), _ = run(b, [a], dtype, materialize_all=True, fuse=False)     # sliced operands: the same bits
    np.testing.assert_array_equal(f, y)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("nq,nk,heads,kv,dim,causal,bounds", ODD)
@pytest.mark.parametrize("left", [0.3, 0.01, 0.0])
def test_keys_whose_scores_are_minus_infinity(left, nq, nk, heads, kv, dim, causal, bounds, dtype):
    # weigh nothing, in whole tiles, waves and workgroups too; a row with no others gives zeros, and NaN in q or in a
    # key that is seen makes the row NaN
    from block_util import run
    rng = np.random.default_rng([nq, nk, dim, 1])
    q, k, v = tensors(rng, (1, 1, nq), (1, 1, nk), heads, kv, dim, dtype)
    q[..., ::dim] = 1
    k[0, 0, rng.random(nk) >= left, ::dim] = -np.inf
    if nq > 20:
        q[0, 0, nq // 2, 3] = np.nan
    ref, size = oracle.attention(q, k, v, heads, kv, dim, causal, 0.0, bounds, weight_of=np.abs)
    b, a = graph(q, k, v, dtype, heads, kv, dim, bounds, causal=causal)
    log(f"[case] attention, scores of -inf but for {left}, {nq} on {nk}, {heads}/{kv} x {dim} causal {causal} {bounds} type {dtype}")
    (y,), _ = run(b, [a], dtype, {a: dtype})
    check(q, k, v, dtype, heads, kv, dim, y, bounds, causal=causal)
    assert left or (y[np.isfinite(y)] == 0).all()


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("q,k", [((2, 1, 150), (2, 1, 210)), ((2, 1, 2), (2, 1, 600)), ((1, 1, 1), (1, 1, 3000))])
def test_operands_in_mixed_layouts(q, k, dtype):
    # graph inputs read in place beside sliced tensors, views of a concatenation among them: the same bits
    from block_util import builder, given, run
    t = tensors(np.random.default_rng(q[2]), q, k, 6, 2, 72, dtype)
    first = None
    for sliced in range(8):
        for joined in (False, True):
            b = builder()
            ids = []
            for i, x in enumerate(t):
                x = given(b, x, dtype)
                if sliced >> i & 1:
                    x = b.add(x, given(b, np.zeros_like(t[i]), dtype))
                ids.append(x)
            a = b.attention(*ids, 6, 2, 72)
            outs = [a]
            if joined and sliced & 6 == 6:
                outs.append(b.conv(b.concat(ids[1:]), 8))
            log(f"[case] attention {q} on {k}, sliced {sliced:03b} joined {joined} type {dtype}")
            y = run(b, outs, dtype, {a: dtype})[0][0]
            first = y if first is None else first
            np.testing.assert_array_equal(y, first)
