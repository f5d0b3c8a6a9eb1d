"""Rotary positions against the oracle (64 bits).

An angle is a fraction of a turn: the frequency is within 2^-65 of a turn, times a
32-bit position within 2^-34, and rounded to a float within 2^-26; that is 2^-23 of
a radian.  The hardware's sine and cosine are taken as within 2^-18.  So
    |error| <= (2^-18 + 2^-22) (|a| + |b|) + half a step of the storage type.
"""
import numpy as np
import pytest

import oracle
from gpu_util import log

pytestmark = pytest.mark.gpu

TURN = 2.0 ** -18 + 2.0 ** -22


def series(pairs, axes):
    of = [i * axes // max(1, pairs) for i in range(pairs)]
    return of, [10000.0 ** (-i / max(1, pairs)) for i in range(pairs)]


def check(b, t, x, positions, dtype, got, what=""):
    from block_util import HALF, TINY, within
    op = b.ops[t]
    args = (op["heads"], op["head_dim"], op["axes"], op["freqs"], positions, op["from"], op["adjacent"])
    ref = oracle.rotary(x, *args)
    # |a| + |b| of each pair: turn (|a|, |b|) by zero and add the partner
    half = len(op["axes"])
    a = np.abs(x[..., op["from"]:op["from"] + op["heads"] * op["head_dim"]]).reshape(x.shape[:3] + (op["heads"], op["head_dim"]))
    size = np.zeros_like(a)
    for i in range(half):
        p, q = (2 * i, 2 * i + 1) if op["adjacent"] else (i, i + half)
        size[..., p] = size[..., q] = a[..., p] + a[..., q]
    within(got, ref, HALF[dtype] * np.abs(ref) + TINY[dtype] + TURN * size.reshape(ref.shape), what)
    # the other channels are copies
    rest = size.reshape(ref.shape) == 0
    np.testing.assert_array_equal(got[rest], ref[rest])


CASES = [
    # n, h, w, heads, dim, pairs, adjacent, first, more channels
    (1, 1, 1, 1, 8, 4, True, 0, 0), (1, 14, 14, 12, 64, 32, False, 0, 0), (2, 7, 5, 3, 32, 16, True, 8, 16),
    (1, 9, 9, 4, 80, 40, False, 16, 0), (1, 3, 33, 2, 128, 64, False, 0, 128), (1, 1, 70, 32, 128, 64, True, 0, 0),
    (1, 5, 5, 2, 72, 36, False, 0, 8), (1, 5, 5, 2, 72, 33, True, 8, 0), (1, 4, 4, 3, 64, 16, False, 0, 0),
    (1, 4, 4, 3, 64, 8, True, 0, 0), (1, 2, 3, 2, 24, 0, False, 0, 0), (1, 2, 2, 1, 1024, 512, True, 0, 0),
    (3, 1, 1, 5, 16, 8, False, 0, 4), (1, 1, 9, 7, 40, 1, False, 0, 1),
]


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("n,h,w,heads,dim,pairs,adjacent,first,more", CASES)
def test_rotary(n, h, w, heads, dim, pairs, adjacent, first, more, dtype):
    from block_util import builder, given, run, stored
    log(f"[case] rotary {n}x{h}x{w} heads {heads}x{dim} pairs {pairs} adjacent {adjacent} from {first} type {dtype}")
    rng = np.random.default_rng([n, h, w, heads, dim])
    x = stored(rng.standard_normal((n, h, w, first + heads * dim + more)), dtype)
    b = builder()
    xi = given(b, x, dtype)
    axes, freqs = series(pairs, 3)
    t = b.rotary(xi, heads, dim, axes, freqs, first=first, adjacent=adjacent)
    (y,), _ = run(b, [t], dtype, {t: dtype})
    check(b, t, x, None, dtype, y, "grid")
    (f,), _ = run(b, [t], dtype, materialize_all=True, fuse=False)
    np.testing.assert_array_equal(f, y)
    # given positions, of one axis and of five, far ones and negative ones
    for count in (1, 5):
        pos = rng.integers(-2 ** 31, 2 ** 31, (n, h, w, count))
        pos[0, 0, 0] = -2 ** 31
        pos[-1, -1, -1] = 2 ** 31 - 1
        p = b.index_input(pos)
        axes, freqs = series(pairs, count)
        t = b.rotary(xi, heads, dim, axes, freqs, positions=p, first=first, adjacent=adjacent)
        # (frequencies of whole parts of a turn, whose products with far positions 64 bits hold)
        b.ops[t]["freqs"] = [-2 * np.pi * (i + 1) / 1024 for i in range(pairs)]
        (y,), _ = run(b, [t], dtype)
        small = pos % 1024                     # the same angles, near zero
        check(b, t, x, small, dtype, y, f"{count} axes")
        b.ops.pop()
        b.ops.pop()
        b._hwc[len(b.ops):] = []


def test_one_token_at_each_position_is_the_row():
    # a row of tokens at positions given, and each token by itself: the same bits
    from block_util import builder, given, run, stored
    rng = np.random.default_rng(1)
    x = stored(rng.standard_normal((1, 1, 6, 128)), 1)
    pos = rng.integers(0, 10 ** 6, (1, 1, 6, 3))
    axes, freqs = series(32, 3)

    def turned(x, pos):
        b = builder()
        xi = given(b, x, 1)
        t = b.rotary(xi, 2, 64, axes, freqs, positions=b.index_input(pos))
        return run(b, [t], 1)[0][0]

    log("[case] one token at a time")
    y = turned(x, pos)
    for i in range(6):
        np.testing.assert_array_equal(turned(x[:, :, i:i + 1], pos[:, :, i:i + 1]), y[:, :, i:i + 1])


def test_high_frequencies_at_far_positions():
    # the angles' fractions of a turn by 60 digits; within 2^-25 of a turn, the sine and its products as above
    from decimal import Decimal, getcontext
    from block_util import HALF, builder, given, run, stored, within
    getcontext().prec = 60
    turn = 2 * Decimal("3.14159265358979323846264338327950288419716939937510582097494")
    freqs = [0.5, 7.3, 511.9, -123.456, 1.0, 2.0 ** -40, 300.0000001, -0.75]
    pos = np.array([0, 1, -1, 12345, 2 ** 31 - 1, -2 ** 31, 2 ** 30 + 7, -1999999999], np.int64)
    x = stored(np.random.default_rng(3).standard_normal((1, 1, len(pos), 16)), 0)
    b = builder()
    t = b.rotary(given(b, x, 0), 1, 16, [0] * 8, freqs, positions=b.index_input(pos.reshape(1, 1, -1, 1)))
    log("[case] rotary, high frequencies at far positions")
    (y,), _ = run(b, [t], 0, {t: 0})
    angle = np.array([[float(Decimal(int(p)) * Decimal(f) % turn) for f in freqs] for p in pos])
    lo, hi = x[0, 0, :, :8], x[0, 0, :, 8:]
    ref = np.concatenate([lo * np.cos(angle) - hi * np.sin(angle), lo * np.sin(angle) + hi * np.cos(angle)], 1)
    size = np.tile(np.abs(lo) + np.abs(hi), (1, 2))
    within(y[0, 0], ref, HALF[0] * np.abs(ref) + 2.0 ** -25 + (2.0 ** -18 + 2 * np.pi * 2.0 ** -25) * size)
