"""Performance cases of what lies between the looked-up rows and the next token: layer norm and its gradient, the product of tokens
with weight codes in 8-bit integers, and sampling from the logits.

With ``own`` false an operator runs in its plain form, elementary torch operations in 32 bits (in 64 for the masses that a token is drawn
by); with ``own`` true through the package.  Widths and vocabularies are those of the package's workloads and performance cases.
"""
import math

import numpy as np
import torch

own = False

EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "int32": torch.int32, "int64": torch.int64}
K_X = 6                         # of the 8-bit weight codes that the quantized step emits


def _norm(name, rows, dim, **more):
    c = dict(name=name, op="norm", rows=rows, dim=dim, x="bf16", weight="f32", out="bf16", gap=0)
    c.update(more)
    return c


def _norm_grad(name, rows, dim, **more):
    c = dict(name=name, op="norm_grad", rows=rows, dim=dim, x="bf16", weight="f32", dout="bf16", grad="f32", gap=0, accumulate=False)
    c.update(more)
    return c


def _linear(name, tokens, inputs, outputs, **more):
    c = dict(name=name, op="linear", tokens=tokens, inputs=inputs, outputs=outputs, x="bf16", out="bf16", scales="codes", bias="none", gap=0)
    c.update(more)
    return c


def _sample(name, rows, vocab, **more):
    c = dict(name=name, op="sample", rows=rows, vocab=vocab, logits="f32", ids="int64", temperature=1.0, top_k=0, top_p=1.0, min_p=0.0,
             per_row=False, masked=0.0, gap=0)
    c.update(more)
    return c


def listed():
    return [
        # the norm in front of the head, one token of a decoding loop
        _norm("norm-1", 1, 768),
        # a batch of eight sequences of the large model
        _norm("norm-16k", 16384, 2048),
        # one sequence's gradient, added to what the flat gradient vector holds
        _norm_grad("norm-grad-1k-add", 1024, 768, x="f32", dout="f32", accumulate=True),
        # the large model's batch
        _norm_grad("norm-grad-16k", 16384, 2048),
        # odd width, rows that lie further apart
        _norm_grad("norm-grad-8k-odd", 8191, 1001, x="f16", dout="f16", weight="f16", grad="f16", gap=7),
        # the tied head of the small model for one token, straight from the codes that the step emits
        _linear("linear-1-head", 1, 768, 50257, out="f32"),
        # a layer of the large model for a batch of 64 sequences that decode together
        _linear("linear-64", 64, 2048, 8192, scales="channel", bias="f32"),
        # the same layer for eight prompts
        _linear("linear-16k", 16384, 2048, 8192, scales="channel", bias="f32"),
        # odd sizes: no row of the weights begins where the last one did
        _linear("linear-odd", 129, 1001, 3001, x="f16", out="f16", scales="channel", bias="f16", gap=3),
        # one sequence's next token, by the usual filters
        _sample("sample-1", 1, 50257, temperature=0.8, top_k=50, top_p=0.95),
        # 256 sequences, each with filters of its own
        _sample("sample-256", 256, 50257, logits="bf16", per_row=True),
        # odd vocabulary, a third of it masked, by mass alone
        _sample("sample-33-odd", 33, 32003, logits="f16", top_p=0.9, masked=0.33, gap=5, ids="int32"),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi)))))

    def width(lo, hi):
        n = spread(lo, hi)
        return max(lo, n - n % 16) if rng.random() < 0.6 else n

    kind = lambda: rng.choice(["f32", "bf16", "bf16", "f16"])  # noqa: E731
    gap = rng.choice([0, 0, 8, 3])
    op = rng.choice(["norm", "norm_grad", "linear", "linear", "sample"])
    if op in ("norm", "norm_grad"):
        dim = width(32, 8192)
        rows = spread(1, min(40000, 3.3e7 / dim))
        if op == "norm":
            c = _norm("", rows, dim, x=kind(), weight=kind(), out=kind(), gap=gap)
        else:
            c = _norm_grad("", rows, dim, x=kind(), weight=kind(), dout=kind(), grad=kind(), gap=gap, accumulate=rng.random() < 0.5)
    elif op == "linear":
        inputs, outputs = width(32, 8192), width(32, 60000)
        outputs = min(outputs, int(1.0e8 / inputs))
        tokens = spread(1, min(16384, 2.7e11 / inputs / outputs, 1.3e8 / outputs))
        c = _linear("", tokens, inputs, outputs, x=kind(), out=kind(), scales=rng.choice(["codes", "channel"]),
                    bias=rng.choice(["none", "f32", "bf16"]), gap=gap)
    else:
        vocab = width(500, 130000)
        rows = spread(1, min(1024, 1.28e7 / vocab))
        c = _sample("", rows, vocab, logits=kind(), ids=rng.choice(["int32", "int64"]), temperature=rng.choice([0.3, 0.7, 1.0, 1.5]),
                    top_k=rng.choice([0, 0, 1, 40, 1000]), top_p=rng.choice([1.0, 0.95, 0.9, 0.5]), min_p=rng.choice([0.0, 0.0, 0.05]),
                    per_row=rng.random() < 0.3, masked=rng.choice([0.0, 0.0, 0.5]), gap=gap)
    del c["name"]
    return c


def work(case):
    size = lambda t: {"none": 0, "f32": 4, "bf16": 2, "f16": 2, "int32": 4, "int64": 8}[t]  # noqa: E731
    if case["op"] in ("norm", "norm_grad"):
        n, d = case["rows"] * case["dim"], case["dim"]
        if case["op"] == "norm":
            return {"bytes": n * (size(case["x"]) + size(case["out"])) + 2.0 * d * size(case["weight"]) + 8.0 * case["rows"], "flops": 8.0 * n}
        once = 2.0 if case["accumulate"] else 1.0
        return {"bytes": n * (size(case["x"]) + 2.0 * size(case["dout"])) + d * size(case["weight"]) + 2.0 * once * d * size(case["grad"]) +
                8.0 * case["rows"], "flops": 14.0 * n}
    if case["op"] == "linear":
        T, K, N = case["tokens"], case["inputs"], case["outputs"]
        return {"bytes": T * K * size(case["x"]) + 1.0 * N * K + T * N * size(case["out"]) + N * (4.0 * (case["scales"] == "channel") + size(case["bias"])),
                "flops": 2.0 * T * N * K}
    n = case["rows"] * case["vocab"]
    return {"bytes": n * size(case["logits"]) + case["rows"] * (4.0 + size(case["ids"]) + 16.0 * case["per_row"]), "flops": 4.0 * n}


# ---------------------------------------------------------------------------------------------- inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) % (1 << 62))
    return g


def _wide(gen, rows, dim, gap, dtype, std, offset=None, gain=None):
    """Rows of `dim` values, `gap` more elements between them."""
    whole = torch.empty(rows, dim + gap, device="cuda").normal_(0.0, std, generator=gen)
    if gain is not None:
        whole[:, :dim] *= gain
    if offset is not None:
        whole[:, :dim] += offset
    return whole.to(dtype)[:, :dim]


def prepare(case, seed):
    return {"norm": _prepare_norm, "norm_grad": _prepare_norm, "linear": _prepare_linear, "sample": _prepare_sample}[case["op"]](case, seed)


def _prepare_norm(case, seed):
    gen = _generator(seed)
    rows, dim, op = case["rows"], case["dim"], case["op"]
    # a residual stream: channels of their own mean, a few of them much larger than the others
    offset = torch.empty(dim, device="cuda").normal_(0.0, 0.5, generator=gen)
    gain = torch.where(torch.rand(dim, generator=gen, device="cuda") < 0.01, 20.0, 1.0)
    s = dict(op=op, x=_wide(gen, rows, dim, case["gap"], TYPES[case["x"]], 1.0, offset, gain))
    s["weight"] = torch.empty(dim, device="cuda").normal_(1.0, 0.2, generator=gen).to(TYPES[case["weight"]])
    if op == "norm":
        s["bias"] = torch.empty(dim, device="cuda").normal_(0.0, 0.1, generator=gen).to(TYPES[case["weight"]])
        s["dtype"] = TYPES[case["out"]]
    else:
        s["dout"] = _wide(gen, rows, dim, case["gap"], TYPES[case["dout"]], 1e-2)
        x = s["x"].float()
        s["mean"] = x.mean(1)
        s["rstd"] = 1.0 / ((x - s["mean"][:, None]).square_().mean(1) + EPS).sqrt()
        # slices of the flat gradient vector
        flat = torch.empty(2 * dim, device="cuda").normal_(0.0, 1e-2, generator=gen).to(TYPES[case["grad"]])
        s["dweight"], s["dbias"], s["accumulate"] = flat[:dim], flat[dim:], case["accumulate"]
    if own:
        from paper_2004_14180_amd import LayerNorm
        s["layer"] = LayerNorm(dim, eps=EPS)
        if op == "norm":
            s["out"] = torch.zeros(rows, dim, dtype=s["dtype"], device="cuda")
            s["mean"], s["rstd"] = torch.zeros(rows, device="cuda"), torch.zeros(rows, device="cuda")
        else:
            s["dx"] = torch.zeros(rows, dim, dtype=s["dout"].dtype, device="cuda")
    return s


def _prepare_linear(case, seed):
    gen = _generator(seed)
    T, K, N = case["tokens"], case["inputs"], case["outputs"]
    s = dict(op="linear", x=_wide(gen, T, K, case["gap"], TYPES[case["x"]], 1.0), dtype=TYPES[case["out"]], scales=None, k_x=None, bias=None)
    w = torch.empty(N, K, device="cuda").normal_(0.0, 1.0, generator=gen)
    if case["scales"] == "codes":
        # weights of deviation 0.02 lie on the step's grid of 2^-7; 0.1 here, so that the codes are not mostly zero
        s["k_x"], s["weight"] = K_X, (w * (0.1 * 2.0 ** (K_X + 1))).round_().clamp_(-2.0 ** K_X, 2.0 ** K_X).to(torch.int8)
    else:
        # each channel's largest weight at the largest code
        big = w.abs().amax(1)
        s["weight"] = (w * (127.0 / big)[:, None]).round_().to(torch.int8)
        s["scales"] = big * (0.02 / 127.0)
    if case["bias"] != "none":
        s["bias"] = torch.empty(N, device="cuda").normal_(0.0, 0.1, generator=gen).to(TYPES[case["bias"]])
    if own:
        from paper_2004_14180_amd import Linear8
        s["layer"] = Linear8(N, K, T)
        s["out"] = torch.zeros(T, N, dtype=s["dtype"], device="cuda")
    return s


def _prepare_sample(case, seed):
    gen = _generator(seed)
    rows, vocab = case["rows"], case["vocab"]
    # logits as a language model's: a broad middle and a few tokens far above it
    logits = torch.empty(rows, vocab + case["gap"], device="cuda").normal_(0.0, 2.0, generator=gen)
    for k in range(8):
        at = torch.randint(0, vocab, (rows, 1), generator=gen, device="cuda")
        logits.scatter_add_(1, at, torch.full_like(at, 8.0 - k, dtype=torch.float32))
    if case["masked"] > 0.0:
        logits.masked_fill_(torch.rand(rows, vocab + case["gap"], generator=gen, device="cuda") < case["masked"], -math.inf)
        logits[:, 0] = 0.0              # never all of them
    s = dict(op="sample", logits=logits.to(TYPES[case["logits"]])[:, :vocab], dtype=TYPES[case["ids"]])
    s["u"] = torch.rand(rows, generator=gen, device="cuda")
    for name, values in (("temperature", [0.0, 0.5, 0.8, 1.0, 1.3]), ("top_k", [0, 0, 1, 20, 50, 2000]), ("top_p", [1.0, 0.95, 0.9, 0.5]),
                         ("min_p", [0.0, 0.0, 0.02, 0.1])):
        s[name] = case[name]
        if case["per_row"]:
            pick = torch.randint(0, len(values), (rows,), generator=gen, device="cuda")
            s[name] = torch.tensor(values, dtype=torch.int32 if name == "top_k" else torch.float32, device="cuda")[pick]
    if own:
        from paper_2004_14180_amd import Sampler
        s["sampler"] = Sampler(vocab, rows)
        s["out"] = torch.zeros(rows, dtype=s["dtype"], device="cuda")
    return s


# ---------------------------------------------------------------------------------------------- one pass
def run(s):
    return {"norm": _run_norm, "norm_grad": _run_norm_grad, "linear": _run_linear, "sample": _run_sample}[s["op"]](s)


def _run_norm(s):
    if own:
        s["layer"].forward(s["x"], s["weight"], s["bias"], s["out"], mean=s["mean"], rstd=s["rstd"])
        return {k: s[k] for k in ("out", "mean", "rstd")}
    x = s["x"].float()
    mean = x.mean(1)
    x = x - mean[:, None]
    rstd = 1.0 / (x.square().mean(1) + EPS).sqrt()
    return {"out": (x * rstd[:, None] * s["weight"].float() + s["bias"].float()).to(s["dtype"]), "mean": mean, "rstd": rstd}


def _run_norm_grad(s):
    if own:
        s["layer"].grad(s["dout"], s["x"], s["weight"], s["mean"], s["rstd"], s["dx"], s["dweight"], s["dbias"], accumulate=s["accumulate"])
        return {k: s[k] for k in ("dx", "dweight", "dbias")}
    dy = s["dout"].float()
    x = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
    for name, g in (("dweight", (dy * x).sum(0)), ("dbias", dy.sum(0))):
        s[name].copy_(s[name].float() + g if s["accumulate"] else g)
    g = dy * s["weight"].float()
    dx = (g - g.mean(1, keepdim=True) - x * (g * x).mean(1, keepdim=True)) * s["rstd"][:, None]
    return {"dx": dx.to(s["dout"].dtype), "dweight": s["dweight"], "dbias": s["dbias"]}


def _run_linear(s):
    if own:
        s["layer"].forward(s["x"], s["weight"], s["out"], weight_scales=s["scales"], k_x=s["k_x"], bias=s["bias"])
        return s["out"]
    x = s["x"].float()
    big = x.abs().amax(1, keepdim=True)
    codes = (x * (torch.ones_like(big) / big * 127.0)).round()
    y = None
    for a in range(0, x.shape[1], 1024):        # sums of 1024 products of 8 bits are whole numbers that 32 bits hold
        part = codes[:, a:a + 1024] @ s["weight"][:, a:a + 1024].float().t()
        y = part if y is None else y + part
    y = y * (big * (1.0 / 127.0))
    y = y * (2.0 ** -(s["k_x"] + 1) if s["scales"] is None else s["scales"])
    if s["bias"] is not None:
        y = y + s["bias"].float()
    return y.to(s["dtype"])


def _column(value):
    return value[:, None] if isinstance(value, torch.Tensor) else value


def _run_sample(s):
    if own:
        s["sampler"].sample(s["logits"], s["u"], s["out"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
        return s["out"]
    # tokens in descending order of their logits, the lower index first; every filter keeps the first ones
    x, token = s["logits"].float().sort(dim=1, descending=True, stable=True)
    x = x.double()
    t, k, p, least = (_column(s[n]) for n in ("temperature", "top_k", "top_p", "min_p"))
    t, k, p, least = (v.double() if isinstance(v, torch.Tensor) else torch.full((1, 1), float(np.float32(v)), dtype=torch.float64, device=x.device)
                      for v in (t, k, p, least))
    place = torch.arange(x.shape[1], device=x.device)
    mass = torch.exp((x - x[:, :1]) / torch.where(t > 0, t, torch.ones_like(t)))
    keep = ((k <= 0) | (place < k)) & ((t > 0) | (place < 1))
    total = torch.where(keep, mass, torch.zeros_like(mass)).cumsum(1)
    # the shortest beginning whose mass is p of the whole: a token stays if what is in front of it has less
    ahead = total - torch.where(keep, mass, torch.zeros_like(mass))
    keep = keep & ((ahead < p * total[:, -1:]) | (p >= 1) | (place < 1)) & (mass >= least)
    total = torch.where(keep, mass, torch.zeros_like(mass)).cumsum(1)
    at = (total <= s["u"].double()[:, None] * total[:, -1:]).sum(1, keepdim=True)
    return token.gather(1, at)[:, 0].to(s["dtype"])


# ---------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    global own
    before, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = before
    return {"norm": _exact_norm, "norm_grad": _exact_norm_grad, "linear": _exact_linear, "sample": _exact_sample}[case["op"]](s)


def _exact_norm(s):
    x = s["x"].double()
    var, mean = torch.var_mean(x, dim=1, correction=0)
    rstd = torch.rsqrt(var + EPS)
    y = torch.addcmul(s["bias"].double(), (x - mean.unsqueeze(1)).mul_(rstd.unsqueeze(1)), s["weight"].double())
    return {"out": y, "mean": mean, "rstd": rstd}


def _exact_norm_grad(s):
    # with the mean and the deviation that the call is given
    rows, dim = s["x"].shape
    r = s["rstd"].double().unsqueeze(1)
    h = torch.sub(s["x"].double(), s["mean"].double().unsqueeze(1)).mul_(r)
    dy = s["dout"].double()
    dw, db = torch.mul(dy, h).sum(dim=0), torch.mv(dy.t(), torch.ones(rows, dtype=torch.float64, device="cuda"))
    if s["accumulate"]:
        dw, db = dw + s["dweight"].double(), db + s["dbias"].double()
    g = dy.mul_(s["weight"].double())
    along = torch.mul(g, h).sum(dim=1) / dim
    dx = g.sub_((g.sum(1) / dim).unsqueeze(1)).sub_(h.mul_(along.unsqueeze(1))).mul_(r)
    return {"dx": dx, "dweight": dw, "dbias": db}


def _exact_linear(s):
    # a token's codes are defined by their operations in 32 bits; from there on 64
    x = s["x"].to(torch.float32)
    most = torch.linalg.vector_norm(x, ord=math.inf, dim=1)
    inverse = torch.mul(torch.reciprocal(most), 127.0)
    codes = torch.round(torch.mul(x, inverse.unsqueeze(1))).double()
    unit = s["scales"].double() if s["scales"] is not None else torch.full((s["weight"].shape[0],), 0.5 ** (s["k_x"] + 1), dtype=torch.float64, device="cuda")
    out = torch.zeros(x.shape[0], s["weight"].shape[0], dtype=torch.float64, device="cuda")
    if s["bias"] is not None:
        out += s["bias"].double()
    for a in range(0, out.shape[1], 4096):
        out[:, a:a + 4096] += torch.matmul(codes * (most.double() / 127.0).unsqueeze(1), (s["weight"][a:a + 4096].double() * unit[a:a + 4096, None]).t())
    return out


def _exact_sample(s):
    rows = s["logits"].shape[0]
    filters = [v.cpu().double().numpy() if isinstance(v, torch.Tensor) else np.full(rows, np.float32(v), dtype=np.float64)
               for v in (s["temperature"], s["top_k"], s["top_p"], s["min_p"])]
    u = s["u"].cpu().double().numpy()
    logits = s["logits"].float().cpu().numpy().astype(np.float64)
    out = torch.zeros(rows, dtype=torch.int64)
    for r in range(rows):
        t, k, p, least = (float(f[r]) for f in filters)
        x = logits[r]
        order = np.lexsort((np.arange(x.size), -x))
        if t == 0.0:
            out[r] = int(order[0])
            continue
        mass = np.exp((x[order] - x[order[0]]) / t)
        if k > 0:
            mass = mass[:int(k)]
        end = mass.size
        if p < 1.0:
            end = min(end, 1 + int(np.searchsorted(np.cumsum(mass), p * np.cumsum(mass)[-1], side="left")))
        end = min(end, int(np.count_nonzero(mass >= least)))
        run_of = np.cumsum(mass[:end])
        out[r] = int(order[np.searchsorted(run_of, u[r] * run_of[-1], side="right")])
    return out.to(s["dtype"])
