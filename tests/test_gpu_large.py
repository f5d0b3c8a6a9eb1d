"""The attention block's operators on tensors of more than 4 GiB: byte offsets and
counts that pass 32 bits.  What a row gives does not depend on the rows before it, so
the last rows are compared with the same rows in a small tensor."""
import pytest

from gpu_util import log

pytestmark = pytest.mark.gpu


def plan(ops, outputs, dtype):
    from paper_1907_01989_amd import engine
    return engine.Plan({"ops": ops, "outputs": outputs, "output_dtypes": {t: dtype for t in outputs}}, dtype=dtype)


def run(ops, outputs, dtype, xs):
    import torch
    p = plan(ops, outputs, dtype)
    ys = p.run(xs)
    torch.cuda.synchronize()
    return ys


def noise(rows, c, seed):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.empty((1, 1, rows, c), dtype=torch.float16, device="cuda")
    for part in x.view(-1, c).split(1 << 18):
        part.copy_(torch.randn(part.shape, generator=g, device="cuda"))
    return x


@pytest.mark.parametrize("c", [1024, 1023])
def test_rows_past_4_gib(c):
    # (1023 channels: no whole slices, by conversions; 1024: read and written in place)
    import torch
    import numpy as np
    rows, last = (1 << 21) + 5077, 3000
    x = noise(rows, c, 1)
    assert x.numel() * 2 > 2 ** 32
    rng = np.random.default_rng(0)
    codes, scales = rng.integers(0, 0x7f, (24, c)).astype(np.uint8), np.full((1, -(-c // 128)), 0.001, np.float32)

    def ops(m):
        return [{"op": "input", "shape": (1, 1, m, c), "dtype": 0}, {"op": "add", "a": 0, "b": 0, "act": 0}, {"op": "rms_norm", "in": 1},
                {"op": "quantize", "in": 0}, {"op": "pointwise_fp8", "in": 3, "cout": 24, "q": codes, "scales": scales},
                {"op": "rotary", "in": 0, "heads": 7, "head_dim": 128, "axes": [2] * 64, "freqs": [0.0] * 64, "from": 8}]

    small = run(ops(last), [1, 2, 4, 5], 0, [x[:, :, -last:].contiguous()])
    for t, ref in zip((1, 2, 4, 5), small):
        log(f"[case] tensor {t} of {rows} x {c}")
        y, = run(ops(rows), [t], 0, [x])
        # (the layer's sums have another order where pixels are few)
        if t == 4:
            torch.testing.assert_close(y[:, :, -last:], ref, rtol=2 ** -9, atol=2 ** -9)
        else:
            assert torch.equal(y[:, :, -last:], ref), t
        del y


def test_keys_past_4_gib():
    # equal weights: means of the values, of which all but the last are zeros; a single query, and a packed
    # sequence that begins behind 4 GiB
    import torch
    n, d = (1 << 25) + 100, 64
    k = torch.zeros((1, 1, n, d), dtype=torch.float16, device="cuda")
    v = torch.zeros_like(k)
    assert k.numel() * 2 > 2 ** 32
    v[0, 0, -1] = torch.arange(d, device="cuda") * 512.0
    v[0, 0, 0] = 1024.0
    q = noise(1, d, 2)
    attn = {"op": "attention", "q": 0, "k": 1, "v": 2, "heads": 1, "kv_heads": 1, "head_dim": d}
    ops = [{"op": "input", "shape": (1, 1, 1, d), "dtype": 0}] + [{"op": "input", "shape": (1, 1, n, d), "dtype": 0}] * 2
    log(f"[case] a query on {n} keys")
    from paper_1907_01989_amd import engine
    p = engine.Plan({"ops": ops + [attn], "outputs": [3]}, dtype=0)
    y = p.run([q, k, v])[0].double()
    ref = (v[0, 0, -1].double() + 1024) / n
    # (the sum of weights is exact up to fp32's roundings; one rounding to fp16, of subnormals)
    assert (y.reshape(-1) - ref).abs().max() <= 2.0 ** -25 + 2.0 ** -10 * ref.max()
    bounds = [0, 0, n - 90, n]
    k[0, 0, -90:] = noise(90, d, 3)[0, 0]
    v[0, 0, -90:] = noise(90, d, 4)[0, 0]
    ops += [{"op": "index_input", "shape": (1, 1, 1, 4)}] * 2 + [{**attn, "bounds": 3, "k_bounds": 4}]
    qs = noise(5, d, 5)
    ops[0] = {"op": "input", "shape": (1, 1, 5, d), "dtype": 0}
    log("[case] a packed sequence behind 4 GiB")
    ix = [torch.tensor(b, dtype=torch.int32, device="cuda").reshape(1, 1, 1, 4) for b in ([0, 0, 0, 5], bounds)]
    y, = run(ops, [5], 0, [qs, k, v] + ix)
    small = [{"op": "input", "shape": (1, 1, m, d), "dtype": 0} for m in (5, 90, 90)] + [attn]
    ref, = run(small, [3], 0, [qs, k[:, :, -90:].contiguous(), v[:, :, -90:].contiguous()])
    torch.testing.assert_close(y, ref, rtol=2 ** -9, atol=2 ** -9)
