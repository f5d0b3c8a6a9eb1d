"""Performance cases of the classifier head's operators: the fully connected layer with 4-bit weights (``fc_int4``)
and what is asked of its logits (``topk``, ``log_prob``, ``entropy``).

A case is one graph given to ``engine.Plan`` and run with ``Plan.run``: the layer alone (``fc``), the questions alone
about logits that a program already has (``answers``), or both, which scores given classes (``score``).  Sizes are
those of the MobileNet heads, and of heads with many classes at one to a few hundred rows.

Keys of a case:
  kind     fc | answers | score
  n        rows (batch entries);  cout: classes
  cin      input channels;  group: input channels that share a scale;  zeros: groups have zero points too (else 8)
  store    storage type of activations and scales, fp16 or bf16;  src: element type of the input, fp16 or fp32
  k        top classes per row;  t: given classes per row
  masked   nine in ten classes are ruled out (-inf) in each row, and the first row rules out all
"""
import math

import torch

own = False

BASE = {"cin": 0, "group": 32, "zeros": False, "store": "fp16", "src": "fp16", "k": 0, "t": 0, "masked": False}


def _case(**kw):
    return {**BASE, **kw}


def listed():
    return [
        # v2's classifier on one image: the smallest call, where latency counts
        _case(name="fc_b1_1280x1000", kind="fc", n=1, cin=1280, cout=1000),
        # v1's classifier at the serving batch, with zero points
        _case(name="fc_b64_1024x1000", kind="fc", n=64, cin=1024, cout=1000, zeros=True),
        # one row through a square layer with coarse groups: bound by latency and weight bytes
        _case(name="fc_b1_4096x4096", kind="fc", n=1, cin=4096, cout=4096, group=128),
        # one row of bf16 features to many classes: bound by weight bytes, the largest weights
        _case(name="fc_b1_4096x32000_bf16", kind="fc", n=1, cin=4096, cout=32000, group=64, zeros=True, store="bf16", src="fp32"),
        # odd sizes throughout: a ragged last group, an odd number of channels and classes, a few rows
        _case(name="fc_b7_2001x5003", kind="fc", n=7, cin=2001, cout=5003, group=96, zeros=True, src="fp32"),
        # a small batch through a large square layer
        _case(name="fc_b16_8192x8192", kind="fc", n=16, cin=8192, cout=8192, group=128),
        # a large batch: bound by the products, the most work
        _case(name="fc_b256_4096x4096_bf16", kind="fc", n=256, cin=4096, cout=4096, group=64, store="bf16", src="fp32"),
        # the five best answers of a batch of images, the given labels' log probabilities and the entropy
        _case(name="answers_b64_1000", kind="answers", n=64, cout=1000, k=5, t=1, src="fp32"),
        # one row of many classes: one reader of a long row leaves the GPU idle
        _case(name="answers_b1_131072", kind="answers", n=1, cout=131072, k=20, t=1, src="fp32"),
        # an evaluation over many rows: bound by the logits' bytes, the largest input
        _case(name="answers_b4096_32000", kind="answers", n=4096, cout=32000, k=10, t=4, src="fp32"),
        # rows with most classes ruled out, an odd number of fp16 logits
        _case(name="answers_b33_49999_masked", kind="answers", n=33, cout=49999, k=50, t=8, masked=True),
        # scoring of given classes from features, logits never handed out
        _case(name="score_b8_2048x32000", kind="score", n=8, cin=2048, cout=32000, t=2, group=128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(["fc", "fc", "fc", "answers", "answers", "score"])
        if kind == "answers":
            c = _case(kind=kind, n=_log(rng, 1, 4096), cout=_log(rng, 10, 262144), t=rng.choice([1, 1, 2, 4, 8]),
                      src=rng.choice(["fp32", "fp32", "fp16"]), masked=rng.random() < 0.25)
            c["k"] = min(rng.choice([1, 3, 5, 5, 10, 20, 50, 64]), c["cout"])
            if c["n"] * c["cout"] <= 4096 * 32000:
                return c
            continue
        c = _case(kind=kind, n=_log(rng, 1, 256 if kind == "fc" else 64), cin=_log(rng, 64, 8192), cout=_log(rng, 16, 65536),
                  group=rng.choice([32, 32, 64, 64, 96, 128, 128, 256]), zeros=rng.random() < 0.5,
                  store=rng.choice(["fp16", "fp16", "bf16"]))
        if rng.random() < 0.6:
            c["cin"] = (c["cin"] + 31) // 32 * 32
            c["cout"] = (c["cout"] + 7) // 8 * 8
        c["src"] = "fp32" if c["store"] == "bf16" else rng.choice(["fp16", "fp16", "fp32"])
        if kind == "score":
            c["t"] = rng.choice([1, 1, 2, 5])
        if c["cin"] * c["cout"] <= 4096 * 32000 and c["n"] * c["cin"] * c["cout"] <= 256 * 4096 * 4096:
            return c


def work(case):
    n, cin, cout = case["n"], case["cin"], case["cout"]
    groups = -(-cin // case["group"])
    src = 2 if case["src"] == "fp16" else 4
    asked = 4 * n * (2 * case["k"] + 2 * case["t"] + 1)        # classes and their log probabilities, labels, entropy
    if case["kind"] == "answers":
        return {"bytes": n * cout * src + asked, "flops": 4 * n * cout}
    b = cin * cout // 2 + cout * groups * (3 if case["zeros"] else 2) + 4 * cout + n * cin * src
    b += 4 * n * cout if case["kind"] == "fc" else asked
    return {"bytes": b, "flops": 2 * n * cin * cout + (4 * n * cout if case["kind"] == "score" else 0)}


# ------------------------------------------------------------------- inputs
def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    n, cin, cout = case["n"], case["cin"], case["cout"]
    src = torch.float16 if case["src"] == "fp16" else torch.float32
    store = torch.bfloat16 if case["store"] == "bf16" else torch.float16

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    s = {}
    if case["t"]:
        s["given"] = torch.randint(0, cout, (n, case["t"]), generator=g, device="cuda", dtype=torch.int32)
    if case["kind"] == "answers":
        x = normal(n, cout).mul_(3)
        if case["masked"]:
            x[torch.rand(n, cout, generator=g, device="cuda") < 0.9] = -math.inf
            x[0] = -math.inf
        s["logits"] = x.to(src)
        return s
    groups = -(-cin // case["group"])
    # features that were stored in the plan's type; codes of normal weights, about 2.5 steps to a standard deviation;
    # scales around the ones that give logits a spread of two
    s["x"] = normal(n, cin).to(store).to(src)
    code = torch.randint(6, 11, (cout, groups), generator=g, device="cuda") if case["zeros"] else torch.full((cout, groups), 8, device="cuda")
    zeros = code.to(torch.uint8)
    q = (normal(cout, cin).mul_(2.5) + zeros.repeat_interleave(case["group"], 1)[:, :cin]).round_().clamp_(0, 15).to(torch.uint8)
    if cin % 2:
        q = torch.cat([q, torch.zeros_like(q[:, :1])], 1)
    s["q"] = q[:, 0::2] | q[:, 1::2] << 4                       # two codes to a byte, the even channel in the low half
    s["scales"] = (normal(cout, groups).mul_(0.2).exp_() * (0.8 / math.sqrt(cin))).to(store)
    s["zeros"] = zeros if case["zeros"] else None
    s["bias"] = normal(cout).mul_(0.1)
    return s


def _plan(case, s):
    """The plan that a program keeps for these weights, and the tensors it runs on."""
    from paper_1907_01989_amd import _binding as B, engine
    n, cin, cout = case["n"], case["cin"], case["cout"]
    src = B.DTYPE_FP16 if case["src"] == "fp16" else B.DTYPE_FP32
    ops, outputs, inputs = [], [], []
    if case["kind"] == "answers":
        ops.append({"op": "input", "shape": (n, 1, 1, cout), "dtype": src})
        inputs.append(s["logits"])
    else:
        ops.append({"op": "input", "shape": (n, 1, 1, cin), "dtype": src})
        inputs.append(s["x"])
        host = {k: None if s[k] is None else s[k].float().cpu().numpy() if k in ("scales", "bias") else s[k].cpu().numpy() for k in ("q", "scales", "zeros", "bias")}
        ops.append({"op": "fc_int4", "in": 0, "cout": cout, "group": case["group"], "q": host["q"], "scales": host["scales"], "zeros": host["zeros"], "b": host["bias"]})
        if case["kind"] == "fc":
            outputs.append(1)
    logits = len(ops) - 1
    if case["k"]:
        ops.append({"op": "topk", "in": logits, "k": case["k"]})
        ops.append({"op": "log_prob", "in": logits, "index": len(ops) - 1})
        outputs += [len(ops) - 2, len(ops) - 1]
    if case["t"]:
        ops.append({"op": "index_input", "shape": (n, 1, 1, case["t"])})
        inputs.append(s["given"])
        ops.append({"op": "log_prob", "in": logits, "index": len(ops) - 1})
        ops.append({"op": "entropy", "in": logits})
        outputs += [len(ops) - 2, len(ops) - 1]
    plan = engine.Plan({"ops": ops, "outputs": outputs}, dtype=B.DTYPE_BF16 if case["store"] == "bf16" else B.DTYPE_FP16)
    return plan, inputs, plan.alloc_outputs()


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        s["plan"], s["inputs"], s["outputs"] = _plan(case, s)
    return s


# ------------------------------------------------------------------- plain form, in 32 bits
def _logits(case, s):
    q, cin = s["q"], case["cin"]
    w = torch.stack([q & 15, q >> 4], 2).reshape(case["cout"], -1)[:, :cin].float()
    w -= 8.0 if s["zeros"] is None else s["zeros"].float().repeat_interleave(case["group"], 1)[:, :cin]
    w *= s["scales"].float().repeat_interleave(case["group"], 1)[:, :cin]
    return s["x"].float() @ w.t() + s["bias"]


def _top(x, k):
    """The k largest of each row, ties to the lowest index: keys of the value's order and the index, all different."""
    bits = (x + 0.0).view(torch.int32)
    bits = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
    key = (bits << 32) - torch.arange(x.shape[1], device=x.device)
    return key.topk(k, dim=1).indices


def run(s):
    case = s["case"]
    if own:
        return s["plan"].run(s["inputs"], s["outputs"])
    x = s["logits"].float() if case["kind"] == "answers" else _logits(case, s)
    if case["kind"] == "fc":
        return [x]
    d = x - x.amax(1, keepdim=True).clamp_min(torch.finfo(torch.float32).min)
    e = d.exp()
    total = e.sum(1, keepdim=True)
    logs = total.log()

    def log_prob(i):
        return torch.where(total > 0, d.gather(1, i) - logs, -math.inf)

    out = []
    if case["k"]:
        top = _top(x, case["k"])
        out += [top.to(torch.int32), log_prob(top)]
    out.append(log_prob(s["given"].long()))
    out.append(torch.where(total > 0, logs - (e * d.clamp_min(-1e30)).sum(1, keepdim=True) / total, 0.0))
    return out


# ------------------------------------------------------------------- the definition, in 64 bits
def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "answers":
        z = s["logits"].double()
    else:
        cin = case["cin"]
        group_of = torch.arange(cin, device="cuda") // case["group"]
        codes = torch.empty((case["cout"], cin), dtype=torch.float64, device="cuda")
        codes[:, 0::2] = (s["q"] % 16).double()[:, : (cin + 1) // 2]
        codes[:, 1::2] = (s["q"] // 16).double()[:, : cin // 2]
        codes -= 8 if s["zeros"] is None else s["zeros"].double()[:, group_of]
        codes *= s["scales"].double()[:, group_of]
        z = torch.mm(s["x"].double(), codes.T.contiguous()) + s["bias"].double()
    if case["kind"] == "fc":
        return [z]
    empty = torch.isinf(z).all(1, keepdim=True)
    lp = torch.log_softmax(torch.where(empty, torch.zeros_like(z), z), 1)
    p = lp.exp()
    h = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(1, keepdim=True)
    lp = torch.where(empty, torch.full_like(lp, -math.inf), lp)
    out = []
    if case["k"]:
        top = torch.sort(z, dim=1, descending=True, stable=True).indices[:, : case["k"]]
        out += [top.to(torch.int32), torch.gather(lp, 1, top)]
    return out + [torch.gather(lp, 1, s["given"].long()), torch.where(empty, torch.zeros_like(h), h)]
