"""Performance cases of an attention block's operators: root-mean-square norm (of a sum with a residual, with an output
in 8 bits), the pointwise layer in 8-bit floating point with a scale for each block of 128 (``pointwise_fp8``), rotary
positions with several axes (``rotary``) and attention over images or packed sequences (``attention``).

A case is one graph given to ``engine.Plan`` and run with ``Plan.run``.  Tensors are in the plan's 16-bit storage type,
inputs and outputs too.  Sizes are those of blocks behind convolutional trunks (grids of 7 x 7 to 37 x 37 pixels), and
of blocks with up to some ten thousand tokens.

Keys of a case:
  kind     norm | linear | rotary | attn
  store    storage type, fp16 or bf16
norm       rows, c; residual: the norm of a sum, which is an output too; to8: the norm's output in 8 bits
linear     rows, cin, cout; act: an activation (0 none, 2 ReLU6)
rotary     n, h, w pixels; heads, dim; axes: 2 (rows and columns of an image) or 3 (times, rows and columns, given for
           each pixel); adjacent: channels 2i and 2i + 1 are a pair (else i and i + dim / 2)
attn       heads, kv (heads of keys and values), dim, causal;
           n images of h x w queries and kh x kw keys each, or (n = 0) packed sequences: rows of queries and keys, of
           which the first are sequences of the lengths in the text lens, the others none's
"""
import math

import torch

own = False

BASE = {"store": "fp16"}


def _norm(rows, c, residual=True, to8=True, **kw):
    return {**BASE, "kind": "norm", "rows": rows, "c": c, "residual": residual, "to8": to8, **kw}


def _linear(rows, cin, cout, act=0, **kw):
    return {**BASE, "kind": "linear", "rows": rows, "cin": cin, "cout": cout, "act": act, **kw}


def _rotary(n, h, w, heads, dim, axes=2, adjacent=False, **kw):
    return {**BASE, "kind": "rotary", "n": n, "h": h, "w": w, "heads": heads, "dim": dim, "axes": axes, "adjacent": adjacent, **kw}


def _images(n, h, w, kh, kw_, heads, kv, dim, causal=False, **kw):
    return {**BASE, "kind": "attn", "n": n, "h": h, "w": w, "kh": kh, "kw": kw_, "heads": heads, "kv": kv, "dim": dim, "causal": causal, "rows": 0, "lens": "", **kw}


def _packed(rows, lens, heads, kv, dim, causal=True, **kw):
    return {**BASE, "kind": "attn", "n": 0, "h": 0, "w": 0, "kh": 0, "kw": 0, "heads": heads, "kv": kv, "dim": dim, "causal": causal, "rows": rows, "lens": lens, **kw}


def listed():
    return [
        # one token's residual and norm, 8 bits for the layer behind it: the smallest call, where latency counts
        _norm(name="norm_1x4096", rows=1, c=4096),
        # a 37 x 37 image's tokens, a width that is no whole number of blocks, 16-bit output
        _norm(name="norm_1369x1000_plain", rows=1369, c=1000, residual=False, to8=False),
        # a long prompt: bound by bytes
        _norm(name="norm_16384x2048_bf16", rows=16384, c=2048, store="bf16"),
        # one token through a square layer: bound by weight bytes and latency
        _linear(name="linear_1x4096x4096_bf16", rows=1, cin=4096, cout=4096, store="bf16"),
        # a 14 x 14 image's tokens and one more, odd widths, ReLU6
        _linear(name="linear_197x1000x3992", rows=197, cin=1000, cout=3992, act=2),
        # a long prompt: bound by the products, the most work of the layers
        _linear(name="linear_8192x4096x4096_bf16", rows=8192, cin=4096, cout=4096, store="bf16"),
        # an image's queries and keys behind a trunk of stride 16
        _rotary(name="rotary_14x14x12x64", n=1, h=14, w=14, heads=12, dim=64),
        # a video's: 16 frames of 36 x 52, times, rows and columns given
        _rotary(name="rotary_29952x32x128_bf16", n=1, h=1, w=29952, heads=32, dim=128, axes=3, adjacent=True, store="bf16"),
        # a batch of small planes, many query heads on one head of keys and values from a plane of half the size
        _images(name="attn_b16_14x14_7x7_8h1", n=16, h=14, w=14, kh=7, kw_=7, heads=8, kv=1, dim=64),
        # one token's query against a long row of keys: bound by their bytes, one reader would leave the GPU idle
        _images(name="attn_b1_1x32768_32h8_bf16", n=1, h=1, w=1, kh=1, kw_=32768, heads=32, kv=8, dim=128, causal=True, store="bf16"),
        # images of different sizes packed into one row, an empty one and single tokens among them, unused rows at the end
        _packed(name="attn_packed5003_16h_80", rows=5003, lens="1369,196,1,0,729,64,49,1024,333,1,577,256,400", heads=16, kv=16, dim=80, causal=False),
        # one long causal prompt with grouped heads: bound by the products, the most work
        _packed(name="attn_causal8192_32h8_bf16", rows=8192, lens="8192", heads=32, kv=8, dim=128, store="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width, mostly in whole steps of 64 or 8 channels."""
    c = _log(rng, lo, hi)
    step = rng.choice([64, 64, 8, 8, 1])
    return max(step, c // step * step)


def draw(rng):
    while True:
        kind = rng.choice(["norm", "norm", "linear", "linear", "rotary", "attn", "attn", "attn"])
        store = {"store": rng.choice(["fp16", "bf16"])}
        if kind == "norm":
            c = _norm(_log(rng, 1, 16384), _width(rng, 48, 8192), rng.random() < 0.7, rng.random() < 0.6, **store)
            if c["rows"] * c["c"] <= 16384 * 2048:
                return c
        elif kind == "linear":
            c = _linear(_log(rng, 1, 8192), _width(rng, 64, 8192), _width(rng, 64, 16384), rng.choice([0, 0, 2]), **store)
            if c["rows"] * c["cin"] * c["cout"] <= 8192 * 4096 * 4096 and c["cin"] * c["cout"] <= 8192 * 8192:
                return c
        elif kind == "rotary":
            axes, side = rng.choice([2, 3]), _log(rng, 1, 40)
            shape = (rng.choice([1, 1, 2, 8]), side, _log(rng, 1, 40)) if axes == 2 else (1, 1, _log(rng, 1, 30000))
            c = _rotary(*shape, rng.choice([1, 4, 8, 12, 16, 32]), rng.choice([32, 64, 64, 80, 96, 128]), axes, rng.random() < 0.5, **store)
            if c["n"] * c["h"] * c["w"] * c["heads"] * c["dim"] <= 29952 * 4096:
                return c
        else:
            kv = rng.choice([1, 1, 2, 4, 8])
            heads, dim = kv * rng.choice([1, 2, 4, 8]), rng.choice([16, 32, 64, 64, 80, 96, 128, 128])
            form = rng.choice(["images", "single", "packed", "packed"])
            if form == "images":
                h, w, part = _log(rng, 1, 40), _log(rng, 1, 40), rng.choice([1, 1, 2])
                c = _images(_log(rng, 1, 64), h, w, -(-h // part), -(-w // part), heads, kv, dim, part == 1 and rng.random() < 0.3, **store)
                pairs = c["n"] * h * w * c["kh"] * c["kw"]
            elif form == "single":
                c = _images(rng.choice([1, 1, 2, 8, 32]), 1, 1, 1, _log(rng, 1, 65536), heads, kv, dim, True, **store)
                pairs = 1024 * c["n"] * c["kw"]          # (their bytes, not their products)
            else:
                lens = [rng.choice([0, 1, _log(rng, 1, 1000), _log(rng, 1, 8192)]) for _ in range(rng.choice([1, 2, 5, 16]))]
                lens[0] = max(1, lens[0])
                c = _packed(sum(lens) + rng.choice([0, 0, 1, 100]), ",".join(map(str, lens)), heads, kv, dim, rng.random() < 0.6, **store)
                pairs = c["rows"] ** 2
            if 0 < pairs * heads <= 8192 * 8192 * 32 // 2 and pairs * heads * dim <= 8192 * 8192 * 4096 // 2:
                return c


def _lens(case):
    return [int(t) for t in case["lens"].split(",")]


def _tokens(case):
    """Queries and keys of a case."""
    return (case["rows"], case["rows"]) if case["n"] == 0 else (case["n"] * case["h"] * case["w"], case["n"] * case["kh"] * case["kw"])


def work(case):
    if case["kind"] == "norm":
        values = case["rows"] * case["c"]
        return {"bytes": values * (8 if case["residual"] else 4) + 4 * case["c"], "flops": 4 * values}
    if case["kind"] == "linear":
        rows, cin, cout = case["rows"], case["cin"], case["cout"]
        scales = 4 * -(-cin // 128) * -(-cout // 128)
        return {"bytes": 2 * rows * (cin + cout) + cin * cout + scales + 4 * cout, "flops": 2 * rows * cin * cout}
    if case["kind"] == "rotary":
        pixels = case["n"] * case["h"] * case["w"]
        values = pixels * case["heads"] * case["dim"]
        return {"bytes": 4 * values + (12 * pixels if case["axes"] == 3 else 0), "flops": 3 * values}
    q, k = _tokens(case)
    if case["n"] == 0:
        pairs = sum(t * (t + 1) // 2 if case["causal"] else t * t for t in _lens(case))
    else:
        a, b = q // case["n"], k // case["n"]
        seen = sum(max(0, i + 1 + b - a) for i in range(a)) if case["causal"] else a * b
        pairs = case["n"] * seen
    index = 4 * (len(_lens(case)) + 1) if case["n"] == 0 else 0
    return {"bytes": 2 * case["dim"] * (2 * q * case["heads"] + 2 * k * case["kv"]) + index, "flops": 4 * pairs * case["heads"] * case["dim"]}


# ------------------------------------------------------------------- inputs
def _shape(n, h, w, c):
    """As the engine hands tensors out: (n, c) where an image is one pixel."""
    return (n, c) if h == 1 and w == 1 else (n, h, w, c)


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    store = torch.bfloat16 if case["store"] == "bf16" else torch.float16

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    s = {}
    if case["kind"] == "norm":
        # tokens of a residual stream: a spread of its own for each, some channels larger than the others
        size = normal(1, 1, 1, case["c"]).mul_(0.5).exp_() * normal(1, 1, case["rows"], 1).mul_(0.3).exp_()
        s["x"] = (normal(1, 1, case["rows"], case["c"]) * size).to(store)
        if case["residual"]:
            s["r"] = (normal(1, 1, case["rows"], case["c"]) * 0.5).to(store)
        s["weight"] = 1 + 0.2 * normal(case["c"])
    elif case["kind"] == "linear":
        rows, cin, cout = case["rows"], case["cin"], case["cout"]
        s["x"] = (normal(1, 1, rows, cin) * normal(1, 1, 1, cin).mul_(0.5).exp_()).to(store)
        s["codes"] = (normal(cout, cin) * 100).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
        s["scales"] = normal(-(-cout // 128), -(-cin // 128)).mul_(0.2).exp_() * (0.01 / math.sqrt(cin))
        s["bias"] = 0.1 * normal(cout)
    elif case["kind"] == "rotary":
        pixels = (case["n"], case["h"], case["w"])
        s["x"] = normal(*pixels, case["heads"] * case["dim"]).to(store)
        if case["axes"] == 3:
            # frames of 36 x 52 that begin somewhere in a long video
            at = torch.arange(case["w"], device="cuda")
            start = int(torch.randint(0, 100000, (1,), generator=g, device="cuda"))
            s["positions"] = torch.stack([start + at // (36 * 52), at // 52 % 36, at % 52], 1).to(torch.int32).reshape(*pixels, 3)
    else:
        q, k = ((1, 1, case["rows"]),) * 2 if case["n"] == 0 else ((case["n"], case["h"], case["w"]), (case["n"], case["kh"], case["kw"]))
        s["q"] = normal(*q, case["heads"] * case["dim"]).to(store)
        s["k"] = normal(*k, case["kv"] * case["dim"]).to(store)
        s["v"] = normal(*k, case["kv"] * case["dim"]).to(store)
        if case["n"] == 0:
            ends = torch.tensor([0] + _lens(case)).cumsum(0)
            s["bounds"] = ends.to(device="cuda", dtype=torch.int32).reshape(1, 1, 1, -1)
    return s


def _frequencies(case):
    """Each pair's axis (0 times, 1 rows, 2 columns) and angle per position: the pairs are shared out among the axes,
    and each axis has a falling series of its own."""
    pairs, first = case["dim"] // 2, 3 - case["axes"]
    axes = [first + i * case["axes"] // pairs for i in range(pairs)]
    of = [axes.count(a) for a in axes]
    return axes, [10000.0 ** (-(i - axes.index(a)) / m) for i, (a, m) in enumerate(zip(axes, of))]


def _plan(case, s):
    """The plan that a program keeps for these weights, and the tensors it runs on."""
    from paper_1907_01989_amd import _binding as B, engine
    store = B.DTYPE_BF16 if case["store"] == "bf16" else B.DTYPE_FP16
    ops, inputs = [], []

    def given(name):
        if s[name].dtype == torch.int32:
            ops.append({"op": "index_input", "shape": tuple(s[name].shape)})
        else:
            ops.append({"op": "input", "shape": tuple(s[name].shape), "dtype": store})
        inputs.append(s[name])
        return len(ops) - 1

    def op(**kw):
        ops.append(kw)
        return len(ops) - 1

    host = {k: s[k].cpu().numpy() for k in ("weight", "codes", "scales", "bias") if k in s}
    if case["kind"] == "norm":
        x, outputs = given("x"), []
        if case["residual"]:
            x = op(op="add", a=x, b=given("r"), act=0)
            outputs.append(x)
        outputs.append(op(op="rms_norm", w=host["weight"], eps=1e-6, to8=case["to8"], **{"in": x}))
    elif case["kind"] == "linear":
        x = op(op="quantize", **{"in": given("x")})
        outputs = [op(op="pointwise_fp8", cout=case["cout"], act=case["act"], q=host["codes"], scales=host["scales"], b=host["bias"], **{"in": x})]
    elif case["kind"] == "rotary":
        axes, freqs = _frequencies(case)
        x = given("x")
        positions = given("positions") if case["axes"] == 3 else -1
        outputs = [op(op="rotary", heads=case["heads"], head_dim=case["dim"], adjacent=case["adjacent"], axes=axes, freqs=freqs, positions=positions, **{"in": x})]
    else:
        q, k, v = given("q"), given("k"), given("v")
        bounds = given("bounds") if case["n"] == 0 else -1
        outputs = [op(op="attention", q=q, k=k, v=v, heads=case["heads"], kv_heads=case["kv"], head_dim=case["dim"], causal=case["causal"], bounds=bounds)]
    plan = engine.Plan({"ops": ops, "outputs": outputs, "output_dtypes": {t: store for t in outputs}}, dtype=store)
    return plan, inputs, plan.alloc_outputs()


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if case["kind"] == "rotary":
        axes, freqs = _frequencies(case)
        s["axes"], s["freqs"] = torch.tensor(axes, device="cuda"), torch.tensor(freqs, device="cuda", dtype=torch.float64)
    if own:
        s["plan"], s["inputs"], s["outputs"] = _plan(case, s)
    return s


# ------------------------------------------------------------------- plain form
def _blocks(x):
    """Channels in blocks of 128, zeros behind the last."""
    c = x.shape[-1]
    return torch.nn.functional.pad(x, (0, -c % 128)).unflatten(-1, (-1, 128))


def _in_8_bits(x):
    """The values that 8 bits (e4m3) and a power of two for each block of 128 channels stand for: the smallest that
    brings the block's largest magnitude to at most 448."""
    b = _blocks(x)
    m, e = torch.frexp(b.abs().amax(-1, keepdim=True))
    e = (e - 9 + (m > 0.875).to(e.dtype)).clamp_min(-126)
    q = torch.ldexp(b, -e).float().to(torch.float8_e4m3fn).to(x.dtype)
    return torch.ldexp(q, e).flatten(-2)[..., : x.shape[-1]]


def _plain_norm(case, s):
    # (in 64 bits: values next to a border between two 8-bit ones)
    h = s["x"]
    out = []
    if case["residual"]:
        h = (h.float() + s["r"].float()).to(h.dtype)
        out.append(h)
    wide = torch.float64 if case["to8"] else torch.float32
    x = h.to(wide)
    y = x * (x.square().mean(-1, keepdim=True) + 1e-6).rsqrt() * s["weight"].to(wide)
    if case["to8"]:
        y = _in_8_bits(y)
    return out + [y.to(h.dtype)]


def _plain_linear(case, s):
    cin, cout = case["cin"], case["cout"]
    w = s["codes"].view(torch.float8_e4m3fn).float()
    w = w * s["scales"].repeat_interleave(128, 0)[:cout].repeat_interleave(128, 1)[:, :cin]
    y = _in_8_bits(s["x"].float()).reshape(-1, cin) @ w.t() + s["bias"]
    if case["act"] == 2:
        y = y.clamp(0, 6)
    return [y.to(s["x"].dtype).reshape(1, 1, -1, cout)]


def _plain_rotary(case, s):
    # (angles in 64 bits: those of far positions)
    n, h, w = case["n"], case["h"], case["w"]
    if case["axes"] == 3:
        at = s["positions"].double()
    else:
        at = torch.stack(torch.meshgrid(*(torch.arange(m, device="cuda", dtype=torch.float64) for m in (n, h, w)), indexing="ij"), -1)
    angle = (at[..., s["axes"]] * s["freqs"]).unsqueeze(-2)
    cos, sin = angle.cos().float(), angle.sin().float()
    x = s["x"].float().unflatten(-1, (case["heads"], case["dim"]))
    a, b = (x[..., 0::2], x[..., 1::2]) if case["adjacent"] else x.chunk(2, -1)
    a, b = a * cos - b * sin, a * sin + b * cos
    y = torch.stack([a, b], -1).flatten(-2) if case["adjacent"] else torch.cat([a, b], -1)
    return [y.flatten(-2).to(s["x"].dtype)]


def _seen(case, s, tq, tk):
    """Which keys each query sees."""
    i, j = torch.arange(tq, device="cuda").unsqueeze(1), torch.arange(tk, device="cuda").unsqueeze(0)
    if case["n"] == 0:
        ends = s["bounds"].reshape(-1)[1:].contiguous()
        of = torch.searchsorted(ends, i, right=True)
        m = (of == torch.searchsorted(ends, j.t().contiguous(), right=True).t()) & (of < ends.numel())
        return m & (j <= i) if case["causal"] else m
    return j <= i + (tk - tq) if case["causal"] else None


def _plain_attn(case, s):
    d, n = case["dim"], max(1, case["n"])

    def heads(x, count):
        return x.float().reshape(n, -1, count, d).transpose(1, 2)

    q = heads(s["q"], case["heads"])
    k, v = (heads(s[t], case["kv"]).repeat_interleave(case["heads"] // case["kv"], 1).contiguous() for t in ("k", "v"))
    e = q @ k.transpose(2, 3).contiguous()
    e *= 1 / math.sqrt(d)
    seen = _seen(case, s, e.shape[2], e.shape[3])
    if seen is not None:
        e.masked_fill_(~seen, -math.inf)
    e -= e.amax(-1, keepdim=True).clamp_min_(torch.finfo(torch.float32).min)
    e.exp_()
    total = e.sum(-1, keepdim=True)
    y = e @ v
    y = torch.where(total > 0, y / total, 0.0)
    return [y.transpose(1, 2).reshape(s["q"].shape).to(s["q"].dtype)]


def run(s):
    case = s["case"]
    if own:
        return s["plan"].run(s["inputs"], s["outputs"])
    out = {"norm": _plain_norm, "linear": _plain_linear, "rotary": _plain_rotary, "attn": _plain_attn}[case["kind"]](case, s)
    return [y.reshape(_shape(*y.shape)) for y in out]


# ------------------------------------------------------------------- the definition, in 64 bits
def _rounded(x):
    """To three bits behind the leading one, ties to even, and in steps of 2^-9 below 2^-6."""
    exponent = torch.floor(torch.log2(x.abs().clamp_min(2.0 ** -40))).clamp_min(-6)
    step = torch.exp2(exponent - 3)
    return torch.round(x / step) * step


def _quantized(x):
    out = torch.empty_like(x)
    whole = x.shape[-1] // 128 * 128
    for part, to in ((x[..., :whole].unflatten(-1, (whole // 128, 128)), out[..., :whole]), (x[..., whole:].unsqueeze(-2), out[..., whole:])):
        if part.numel() == 0:
            continue
        top = part.abs().amax(-1, keepdim=True)
        e = torch.ceil(torch.log2(top.clamp_min(1e-300) / 448))
        # (the logarithm may be off by its last bit at a power of two)
        e = torch.where(top > 448 * torch.exp2(e), e + 1, e)
        e = torch.where(top <= 448 * torch.exp2(e - 1), e - 1, e).clamp_min(-126)
        to.copy_((_rounded(part / torch.exp2(e)) * torch.exp2(e)).flatten(-2))
    return out


def _exact_norm(case, s):
    x = s["x"].double()
    out = []
    if case["residual"]:
        out.append(x + s["r"].double())
        x = (s["x"].float() + s["r"].float()).to(s["x"].dtype).double()    # (the norm is of the stored sum)
    y = s["weight"].double() * x / torch.sqrt((x * x).sum(-1, keepdim=True) / case["c"] + 1e-6)
    return out + [_quantized(y) if case["to8"] else y]


def _exact_linear(case, s):
    cout, cin = case["cout"], case["cin"]
    code = s["codes"].long()
    exponent, mantissa = code >> 3 & 15, code & 7
    w = torch.where(exponent > 0, (8 + mantissa).double() * torch.exp2((exponent - 10).double()), mantissa.double() * 2.0 ** -9)
    w = torch.where(code > 127, -w, w)
    rows, cols = torch.arange(cout, device="cuda") // 128, torch.arange(cin, device="cuda") // 128
    w *= s["scales"].double()[rows][:, cols]
    y = torch.mm(_quantized(s["x"].double()).reshape(-1, cin), w.T.contiguous()) + s["bias"].double()
    return [torch.clamp(y, 0, 6) if case["act"] == 2 else y]


def _exact_rotary(case, s):
    axes, freqs = _frequencies(case)
    n, h, w = case["n"], case["h"], case["w"]
    half = case["dim"] // 2
    x = s["x"].double().reshape(n, h, w, case["heads"], case["dim"])
    y = torch.empty_like(x)
    lines = [torch.arange(m, device="cuda", dtype=torch.float64) for m in (n, h, w)]
    grid = [lines[0].reshape(n, 1, 1, 1), lines[1].reshape(1, h, 1, 1), lines[2].reshape(1, 1, w, 1)]
    for i in range(half):
        t = s["positions"][..., axes[i]].double().unsqueeze(-1) if case["axes"] == 3 else grid[axes[i]]
        turn = torch.polar(torch.ones_like(t), t * freqs[i])
        p, q = (2 * i, 2 * i + 1) if case["adjacent"] else (i, i + half)
        z = torch.complex(x[..., p], x[..., q]) * turn
        y[..., p], y[..., q] = z.real, z.imag
    return [y]


def _exact_attn(case, s):
    d, group, n = case["dim"], case["heads"] // case["kv"], case["n"]
    q, k, v = (s[t].double().reshape(-1, count, d) for t, count in (("q", case["heads"]), ("k", case["kv"]), ("v", case["kv"])))
    out = torch.zeros_like(q)
    if n == 0:
        ends = torch.tensor(_lens(case)).cumsum(0).tolist()
        spans = [(b - t, b, b - t, b) for t, b in zip(_lens(case), ends)]
    else:
        a, b = q.shape[0] // n, k.shape[0] // n
        spans = [(i * a, i * a + a, i * b, i * b + b) for i in range(n)]
    for q0, q1, k0, k1 in spans:
        if q1 == q0 or k1 == k0:
            continue
        hidden = torch.ones(q1 - q0, k1 - k0, dtype=torch.bool, device="cuda").triu_(1 + (k1 - k0) - (q1 - q0))
        for head in range(case["heads"]):
            z = torch.mm(q[q0:q1, head].contiguous(), k[k0:k1, head // group].T.contiguous()) / math.sqrt(d)
            if case["causal"]:
                z = z.masked_fill(hidden, -math.inf)
            p = torch.nan_to_num(torch.softmax(z, 1), nan=0.0)
            out[q0:q1, head] = torch.mm(p, v[k0:k1, head // group].contiguous())
    return [out]


def exact(case, seed):
    s = _inputs(case, seed)
    return {"norm": _exact_norm, "linear": _exact_linear, "rotary": _exact_rotary, "attn": _exact_attn}[case["kind"]](case, s)
