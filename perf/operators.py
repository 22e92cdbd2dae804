"""Performance cases of the operators beside the quantized step: AdamW over many tensors with states in 32 or 8 bits, the norm of all
gradients with its clipping factor, embedding lookup with scaling, and the embedding's gradient by sorted tokens.

With ``own`` false an operator runs in its plain form, elementary torch operations in 32 bits; with ``own`` true through the package.
Layer lists are those of the package's workloads and performance cases; parameters, gradients and moments are slices of one flat vector
per kind, as the package's step has them.
"""
import math

import torch

own = False

BETA1, BETA2, EPS, LR, DECAY = 0.9, 0.999, 1e-8, 1e-4, 0.1
BLOCK = 256                     # elements of a tensor that share the scales of their 8-bit states
FP8_MAX, FP8_LEAST = 448.0, 2.0 ** -9
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "codes8": torch.int8, "codes16": torch.int16}
K_X = {"codes8": 6, "codes16": 14}


def _adamw(name, layers, **more):
    c = dict(name=name, op="adamw", layers=layers, n=0, blocks=0, d=0, vocab=0, ctx=0, bits=32, grad="f32", copy="none", clip=False)
    c.update(more)
    return c


def _norm(name, layers, **more):
    c = dict(name=name, op="norm", layers=layers, n=0, blocks=0, d=0, vocab=0, ctx=0, grad="f32")
    c.update(more)
    return c


def _lookup(name, rows, dim, tokens, **more):
    c = dict(name=name, op="lookup", rows=rows, dim=dim, tokens=tokens, table="bf16", out="bf16", ids="int64", spread="zipf", pad=0.0)
    c.update(more)
    return c


def _grad(name, rows, dim, tokens, **more):
    c = dict(name=name, op="grad", rows=rows, dim=dim, tokens=tokens, dout="bf16", grad="f32", ids="int64", spread="zipf", pad=0.0,
             gap=0, accumulate=False)
    c.update(more)
    return c


def listed():
    gpt2 = dict(blocks=12, d=768, vocab=50257, ctx=1024)
    gpt1p3b = dict(blocks=24, d=2048, vocab=50257, ctx=2048)
    return [
        # a small model of ragged layers at any offset: launches and host work count
        _adamw("adamw-ragged-51k", "ragged", n=51440),
        # an image model of 62 tensors with 8-bit states, fp32 gradients
        _adamw("adamw8-resnet18", "resnet18", bits=8),
        # mixed-precision training of GPT-2 small: bf16 gradients, clipped, fp32 master weights and the model's bf16 copy
        _adamw("adamw-gpt2-small", "gpt", grad="bf16", copy="bf16", clip=True, **gpt2),
        # the large end: GPT-1.3B, where 8-bit states save 8 GB
        _adamw("adamw8-gpt-1.3b", "gpt", bits=8, grad="bf16", copy="bf16", clip=True, **gpt1p3b),
        # clipping a small model's gradients
        _norm("norm-ragged-51k", "ragged", n=51440),
        # ... and a large one's
        _norm("norm-gpt-1.3b", "gpt", grad="bf16", **gpt1p3b),
        # one token of a decoding loop, from the 8-bit weight codes that the quantized step emits
        _lookup("lookup-1-codes", 50257, 768, 1, table="codes8", out="f16", ids="int32"),
        # one sequence, fp32 weights
        _lookup("lookup-1k-f32", 50257, 768, 1024, table="f32", out="f32"),
        # a batch of eight sequences of the large model
        _lookup("lookup-16k-bf16", 50257, 2048, 16384),
        # one sequence's gradient added to that of the tied output head
        _grad("grad-1k-add", 50257, 768, 1024, dout="f32", accumulate=True),
        # a batch of eight sequences of the large model, the whole gradient matrix written
        _grad("grad-16k", 50257, 2048, 16384),
        # odd sizes, strided rows, padded sequences: one token of eight is the padding
        _grad("grad-8k-odd", 32003, 1001, 8191, dout="f16", gap=7, pad=0.125, ids="int32", accumulate=True),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(math.exp(rng.uniform(math.log(lo), math.log(hi))))

    op = rng.choice(["adamw", "adamw", "norm", "lookup", "grad", "grad"])
    if op in ("adamw", "norm"):
        n = spread(1e3, 3e8)
        layers = rng.choice(["flat", "ragged", "gpt"])
        more = dict(n=n, grad=rng.choice(["f32", "bf16", "f16"]))
        if layers == "gpt":
            d = max(16, spread((n / 400.0) ** 0.5 + 1, (n / 14.0) ** 0.5 + 2))
            more.update(d=d, vocab=max(1, int(n * 0.28 / d)), ctx=max(1, int(n * 0.02 / d)), blocks=max(1, min(40, int(0.7 * n / (12.0 * d * d)))))
        if op == "adamw":
            more.update(bits=rng.choice([8, 32]), copy=rng.choice(["none", "bf16", "f16"]), clip=rng.random() < 0.5)
            c = _adamw("", layers, **more)
        else:
            c = _norm("", layers, **more)
    else:
        rows = spread(1e3, 1.3e5)
        dim = spread(64, min(4096, 1.0e8 / rows))
        dim = max(64, dim - dim % 8) if rng.random() < 0.6 else dim
        if dim == 3072:
            dim = 3071
        tokens = spread(1, min(40000, 3.3e7 / dim))
        more = dict(ids=rng.choice(["int32", "int64"]), spread=rng.choice(["zipf", "zipf", "uniform"]), pad=rng.choice([0.0, 0.0, 0.2]))
        if op == "lookup":
            table = rng.choice(["f32", "bf16", "f16", "codes8", "codes16"])
            c = _lookup("", rows, dim, tokens, table=table, out=rng.choice(["f32", "bf16", "f16"]), **more)
        else:
            c = _grad("", rows, dim, tokens, dout=rng.choice(["f32", "bf16", "f16"]), grad=rng.choice(["f32", "f32", "bf16"]),
                      gap=rng.choice([0, 0, 5, 8]), accumulate=rng.random() < 0.5, **more)
    del c["name"]
    return c


# ---------------------------------------------------------------------------------------------- sizes
def _sizes(case):
    """The tensors' sizes."""
    if case["layers"] == "flat":
        return [case["n"]]
    if case["layers"] == "resnet18":
        sizes = [64 * 3 * 49, 64, 64]
        cin = 64
        for stage, c in enumerate((64, 128, 256, 512)):
            for block in range(2):
                first = block == 0
                sizes += [c * (cin if first else c) * 9, c, c, c * c * 9, c, c]
                if first and stage > 0:
                    sizes += [c * cin, c, c]
            cin = c
        return sizes + [512 * 1000, 1000]
    if case["layers"] == "gpt":
        d = case["d"]
        block = [d, d, d * 3 * d, 3 * d, d * d, d, d, d, d * 4 * d, 4 * d, 4 * d * d, d]
        return [case["vocab"] * d, case["ctx"] * d] + block * case["blocks"] + [d, d]
    # matrices and the short vectors between them, of every size and alignment, n elements in all
    n, sizes, k = case["n"], [], 0
    while n > 0:
        big = max(1, n * (3 + k % 4) // 8)
        for s in (big, 1 + (big * 7 + k) % 251):
            if n > 0:
                sizes.append(min(s, n))
                n -= sizes[-1]
        k += 1
    return sizes


def _places(case):
    """(begin of each tensor in the flat vectors, their length).  With 8-bit states a tensor begins at a block of its own; otherwise one
    follows the other."""
    at, out = 0, []
    for s in _sizes(case):
        out.append(at)
        at += -(-s // BLOCK) * BLOCK if case.get("bits") == 8 else s
    return out, at


def _zipf_edge(rows):
    return math.log((rows + 2.7) / 2.7)


def _distinct(case):
    """How many rows the tokens touch, on average."""
    rows, n = case["rows"], case["tokens"] * (1.0 - case["pad"])
    if case["spread"] == "uniform":
        return rows * -math.expm1(n * math.log1p(-1.0 / rows))
    r = torch.arange(rows, dtype=torch.float64)
    p = torch.log((r + 3.7) / (r + 2.7)) / _zipf_edge(rows)
    return float((-torch.expm1(n * torch.log1p(-p))).sum())


def work(case):
    size = lambda t: {"none": 0, "f32": 4, "bf16": 2, "f16": 2, "codes8": 1, "codes16": 2, "int32": 4, "int64": 8}[t]  # noqa: E731
    if case["op"] in ("adamw", "norm"):
        P = sum(_sizes(case))
        if case["op"] == "norm":
            return {"bytes": P * size(case["grad"]) + 8.0, "flops": 2.0 * P}
        state = 16.0 if case["bits"] == 32 else 4.0 + 16.0 / BLOCK
        return {"bytes": P * (8.0 + state + size(case["grad"]) + size(case["copy"])), "flops": 16.0 * P}
    T, D, ids = case["tokens"], case["dim"], case["tokens"] * size(case["ids"])
    if case["op"] == "lookup":
        return {"bytes": ids + _distinct(case) * D * size(case["table"]) + T * D * size(case["out"]), "flops": 1.0 * T * D}
    out = 2.0 * _distinct(case) if case["accumulate"] else 1.0 * case["rows"]
    real = T * (1.0 - case["pad"])
    return {"bytes": ids + real * D * size(case["dout"]) + out * D * size(case["grad"]), "flops": 2.0 * real * D}


# ---------------------------------------------------------------------------------------------- inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) % (1 << 62))
    return g


def _layered(case, at, length, gen, rel, dtype=torch.float32):
    """Values around zero of another size in every tensor, 1e-4 to 1e-1; zeros between the tensors."""
    out = torch.zeros(length, dtype=dtype, device="cuda")
    sizes = _sizes(case)
    pick = torch.Generator().manual_seed(len(sizes) + length % 1009)
    std = (10.0 ** (-4.0 + 3.0 * torch.rand(len(sizes), generator=pick, dtype=torch.float64))).tolist()
    for a, n, s in zip(at, sizes, std):
        if n:
            out[a:a + n].normal_(0.0, s * rel, generator=gen)
    return out


def _unseen(case, at, gen, tensors):
    """The embedding's rows that no token has had yet: gradient and moments are zero there."""
    if case["layers"] == "gpt":
        rows = torch.rand(case["vocab"], generator=gen, device="cuda") < 0.3
        n = case["vocab"] * case["d"]
        for t in tensors:
            t[at[0]:at[0] + n].view(case["vocab"], case["d"]).masked_fill_(rows[:, None], 0.0)


def _to_fp8(x, positive):
    """Blocks of x as (what is stored, scale): the block's largest at FP8_MAX; with `positive` nothing above zero becomes zero."""
    big = x.abs().amax(1, keepdim=True)
    big = torch.where(big < 2.0 ** -116, torch.zeros_like(big), big)
    q = x * torch.where(big > 0, FP8_MAX / big, torch.zeros_like(big))
    if positive:
        q = torch.where((x > 0) & (big > 0), q.clamp_min(FP8_LEAST), q)
    return q.to(torch.float8_e4m3fn), big / FP8_MAX


def _tokens(case, gen):
    rows, T = case["rows"], case["tokens"]
    u = torch.rand(T, generator=gen, device="cuda", dtype=torch.float64)
    if case["spread"] == "uniform":
        tok = (u * rows).long()
    else:
        tok = (torch.exp(u * _zipf_edge(rows)) * 2.7 - 2.7).long()
    tok.clamp_(0, rows - 1)
    if case["pad"] > 0.0:
        # sequences of 1024 tokens, padded at their ends with the last row's token
        i = torch.arange(T, device="cuda") % 1024
        tok = torch.where(i >= 1024 * (1.0 - case["pad"]), rows - 1, tok)
    return tok.to(torch.int32 if case["ids"] == "int32" else torch.int64)


def prepare(case, seed):
    return {"adamw": _prepare_adamw, "norm": _prepare_norm, "lookup": _prepare_lookup, "grad": _prepare_grad}[case["op"]](case, seed)


def _views(flat, at, sizes):
    return [flat[a:a + n] for a, n in zip(at, sizes)]


def _prepare_adamw(case, seed):
    gen = _generator(seed)
    sizes = _sizes(case)
    at, length = _places(case)
    s = dict(op="adamw", step=100, clip=None, copy=None, bits=case["bits"])
    s["p"] = torch.zeros(length, device="cuda")
    for a, n in zip(at, sizes):
        s["p"][a:a + n].normal_(0.0, 0.02, generator=gen)
    s["grad"] = _layered(case, at, length, gen, 1.0, TYPES[case["grad"]])
    m, v = _layered(case, at, length, gen, 0.3), _layered(case, at, length, gen, 1.0).square_()
    _unseen(case, at, gen, (s["grad"], m, v))
    if case["bits"] == 8:
        (s["m"], s["m_scales"]), (s["v"], s["v_scales"]) = _to_fp8(m.view(-1, BLOCK), False), _to_fp8(v.sqrt_().view(-1, BLOCK), True)
        for k in ("m", "v", "m_scales", "v_scales"):
            s[k] = s[k].reshape(-1)
    else:
        s["m"], s["v"] = m, v
    del m, v
    if case["copy"] != "none":
        s["copy"] = torch.zeros(length, dtype=TYPES[case["copy"]], device="cuda")
    if case["clip"]:
        s["clip"] = 0.1 + 0.9 * torch.rand(1, generator=gen, device="cuda")
    # vectors (biases, gains) have no decay, matrices do
    decays = [DECAY if n > 8192 else 0.0 for n in sizes]
    if own:
        from paper_2004_14180_amd import AdamW, AdamWConfig
        blocks = [-(-n // BLOCK) for n in sizes]
        first = [a // BLOCK for a in at]
        state8 = dict(m_scales=_views(s["m_scales"], first, blocks), v_scales=_views(s["v_scales"], first, blocks)) if case["bits"] == 8 else {}
        s["opt"] = AdamW(AdamWConfig(beta1=BETA1, beta2=BETA2, eps=EPS, state_bits=case["bits"]), _views(s["p"], at, sizes),
                         _views(s["m"], at, sizes), _views(s["v"], at, sizes), weight_decay=decays, grad_dtype=TYPES[case["grad"]],
                         copies=None if s["copy"] is None else _views(s["copy"], at, sizes), **state8)
        s["grads"] = _views(s["grad"], at, sizes)
    else:
        s["decayed"] = torch.zeros(length, dtype=torch.bool, device="cuda")
        for a, n, w in zip(at, sizes, decays):
            s["decayed"][a:a + n] = w > 0.0
    return s


def _prepare_norm(case, seed):
    gen = _generator(seed)
    sizes = _sizes(case)
    at, length = _places(case)
    s = dict(op="norm", max_norm=1.0, grad=_layered(case, at, length, gen, 1.0, TYPES[case["grad"]]))
    if own:
        from paper_2004_14180_amd import GradNorm
        s["norm"] = GradNorm(sizes, TYPES[case["grad"]])
        s["grads"] = _views(s["grad"], at, sizes)
        s["out"] = torch.zeros(2, device="cuda")
    return s


def _prepare_lookup(case, seed):
    gen = _generator(seed)
    rows, dim, table = case["rows"], case["dim"], case["table"]
    w = torch.empty(rows, dim, device="cuda").normal_(0.0, 0.02, generator=gen)
    if table in K_X:
        # weights on the grid of the quantized step
        k = K_X[table]
        w = (w * 2.0 ** (k + 1)).round_().clamp_(-2.0 ** k, 2.0 ** k)
    s = dict(op="lookup", weight=w.to(TYPES[table]), tokens=_tokens(case, gen), scale=math.sqrt(dim), k_x=K_X.get(table),
             padding=rows - 1 if case["pad"] > 0.0 else None, dtype=TYPES[case["out"]])
    if own:
        from paper_2004_14180_amd import Embedding
        s["emb"] = Embedding(rows, dim, case["tokens"])
        s["out"] = torch.zeros(case["tokens"], dim, dtype=s["dtype"], device="cuda")
    return s


def _prepare_grad(case, seed):
    gen = _generator(seed)
    rows, dim, T = case["rows"], case["dim"], case["tokens"]
    s = dict(op="grad", tokens=_tokens(case, gen), scale=math.sqrt(dim), padding=rows - 1 if case["pad"] > 0.0 else None,
             accumulate=case["accumulate"])
    whole = torch.empty(T, dim + case["gap"], dtype=TYPES[case["dout"]], device="cuda").normal_(0.0, 1e-2, generator=gen)
    s["dout"] = whole[:, :dim]
    s["grad"] = torch.zeros(rows, dim, dtype=TYPES[case["grad"]], device="cuda")
    if case["accumulate"]:
        s["grad"].normal_(0.0, 1e-2, generator=gen)
    if own:
        from paper_2004_14180_amd import Embedding
        s["emb"] = Embedding(rows, dim, T)
    return s


# ---------------------------------------------------------------------------------------------- one pass
def run(s):
    if s["op"] == "adamw":
        s["step"] += 1
        if own:
            s["opt"].step(s["step"], LR, s["grads"], grad_scale=s["clip"])
        else:
            _plain_adamw(s)
        return {k: s[k] for k in ("p", "m", "v", "m_scales", "v_scales", "copy") if s.get(k) is not None}
    if s["op"] == "norm":
        if own:
            s["norm"].grad_norm(s["grads"], s["max_norm"], s["out"])
            return s["out"]
        n = s["grad"].float().square().sum().sqrt()
        return torch.stack([n, torch.where(n > s["max_norm"], s["max_norm"] / n, torch.ones_like(n))])
    if s["op"] == "lookup":
        if own:
            s["emb"].lookup(s["weight"], s["tokens"], s["out"], scale=s["scale"], k_x=s["k_x"], padding_idx=s["padding"])
            return s["out"]
        x = s["weight"][s["tokens"]].float()
        if s["k_x"] is not None:
            x = x * 2.0 ** -(s["k_x"] + 1)
        x = x * s["scale"]
        if s["padding"] is not None:
            x = torch.where((s["tokens"] == s["padding"])[:, None], torch.zeros_like(x), x)
        return x.to(s["dtype"])
    if own:
        s["emb"].grad(s["tokens"], s["dout"], s["grad"], scale=s["scale"], padding_idx=s["padding"], accumulate=s["accumulate"])
        return s["grad"]
    x = s["dout"].float() * s["scale"]
    if s["padding"] is not None:
        x = torch.where((s["tokens"] == s["padding"])[:, None], torch.zeros_like(x), x)
    g = s["grad"].float() if s["accumulate"] else torch.zeros(s["grad"].shape, device="cuda")
    g.index_add_(0, s["tokens"], x)
    return s["grad"].copy_(g)


def _plain_adamw(s):
    t = s["step"]
    g = s["grad"].float()
    if s["clip"] is not None:
        g = g * s["clip"]
    m, v = s["m"], s["v"]
    if s["bits"] == 8:
        m = (m.float().view(-1, BLOCK) * s["m_scales"][:, None]).view(-1)
        v = (v.float().view(-1, BLOCK) * s["v_scales"][:, None]).square().view(-1)
    m = m * BETA1 + g * (1.0 - BETA1)
    v = v * BETA2 + g * g * (1.0 - BETA2)
    r = v.sqrt()
    p = torch.where(s["decayed"], s["p"] - s["p"] * (LR * DECAY), s["p"])
    p = p - m * (LR / (1.0 - BETA1 ** t)) / (r * (1.0 / math.sqrt(1.0 - BETA2 ** t)) + EPS)
    s["p"].copy_(p)
    if s["copy"] is not None:
        s["copy"].copy_(p)
    if s["bits"] == 8:
        for name, x, positive in (("m", m, False), ("v", r, True)):
            q, scale = _to_fp8(x.view(-1, BLOCK), positive)
            s[name].copy_(q.view(-1))
            s[name + "_scales"].copy_(scale.view(-1))
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)


# ---------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    global own
    before, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = before
    return {"adamw": _exact_adamw, "norm": _exact_norm, "lookup": _exact_lookup, "grad": _exact_grad}[case["op"]](s)


def _exact_adamw(s):
    b1, b2, t, n = 0.9, 0.999, s["step"] + 1, s["p"].numel()
    whole = s["bits"] == 32
    out = {k: torch.zeros(n, dtype=torch.float64, device="cuda") for k in ("p", "m", "v")}
    if s["copy"] is not None:
        out["copy"] = out["p"]
    if not whole:
        out["m_scales"], out["v_scales"] = (torch.zeros(n // BLOCK, dtype=torch.float64, device="cuda") for _ in range(2))
    c = 1.0 if s["clip"] is None else s["clip"].double()
    piece = 1 << 26
    for a in range(0, n, piece):
        at = slice(a, min(n, a + piece))
        of = slice(at.start // BLOCK, -(-at.stop // BLOCK))
        g = s["grad"][at].double().mul_(c)
        if whole:
            m, v = s["m"][at].double(), s["v"][at].double()
        else:
            m = s["m"][at].float().double() * s["m_scales"][of].double().repeat_interleave(BLOCK)
            v = (s["v"][at].float().double() * s["v_scales"][of].double().repeat_interleave(BLOCK)) ** 2
        m, v = torch.lerp(g, m, b1), torch.lerp(g * g, v, b2)
        p = s["p"][at].double()
        p *= 1.0 - LR * DECAY * s["decayed"][at].double()
        out["p"][at] = p - LR * (m / (1.0 - b1 ** t)) / (torch.sqrt(v / (1.0 - b2 ** t)) + EPS)
        for name, x in (("m", m), ("v", v)):
            if whole:
                out[name][at] = x
                continue
            # what is stored before its rounding to 8 bits
            x = x if name == "m" else torch.sqrt(x)
            unit = x.reshape(-1, BLOCK).abs().amax(1) / FP8_MAX
            out[name + "_scales"][of] = unit
            unit = unit.repeat_interleave(BLOCK)
            out[name][at] = torch.where(unit > 0, x / unit, torch.zeros_like(x))
    return out


def _exact_norm(s):
    n = math.sqrt(sum(float(x.double().square().sum()) for x in s["grad"].split(1 << 27)))
    return torch.tensor([n, min(1.0, s["max_norm"] / n)], dtype=torch.float64)


def _exact_lookup(s):
    unit = s["scale"] * (1.0 if s["k_x"] is None else 0.5 ** (s["k_x"] + 1))
    keep = torch.ones_like(s["tokens"], dtype=torch.float64) if s["padding"] is None else s["tokens"].ne(s["padding"]).double()
    return torch.index_select(s["weight"], 0, s["tokens"]).double() * (unit * keep)[:, None]


def _exact_grad(s):
    # sums of runs of the sorted tokens, as differences of running sums over slices of columns
    tok, order = torch.sort(s["tokens"].long(), stable=True)
    row, count = torch.unique_consecutive(tok, return_counts=True)
    out = s["grad"].double() if s["accumulate"] else torch.zeros(s["grad"].shape, dtype=torch.float64, device="cuda")
    if s["padding"] is not None:
        keep = row != s["padding"]
    else:
        keep = torch.ones_like(row, dtype=torch.bool)
    last = count.cumsum(0) - 1
    for a in range(0, out.shape[1], 256):
        total = s["dout"][order, a:a + 256].double().cumsum(0)[last]
        total[1:] -= total[:-1].clone()
        out[row[keep], a:a + 256] += total[keep] * s["scale"]
    return out
