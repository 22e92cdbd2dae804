"""Layer norm, the product with weight codes and sampling together, as the example uses them: its gradients, and answers from the codes."""
import importlib.util
import math
import os

import pytest
import torch

import layer_util
from paper_2004_14180_amd import Embedding, LayerNorm, Linear8, Sampler

pytestmark = pytest.mark.gpu
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "tied_embedding.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("tied_embedding", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_the_example_runs(example, capsys):
    losses = example.main(["--optimizer", "normed", "--steps", "5"])
    assert len(losses) == 5 and all(math.isfinite(x) for x in losses)
    assert "answered tokens" in capsys.readouterr().out


def test_the_examples_gradients(example):
    """Against autograd in 64 bits.  Every product and sum of the fp32 way is off by less than 2^-24 sqrt(4096) of its terms' norm, 4e-6; there
    are about ten one behind the other, and the norm's rows pass on an error at most twice as large: 1e-4."""
    R, D = example.ROWS, example.DIM
    gen = torch.Generator(device="cuda").manual_seed(3)
    codes = torch.randint(-64, 65, (R, D), generator=gen, device="cuda").to(torch.int8)
    xhat = codes.float() / 128
    gain, bias = torch.randn(D, generator=gen, device="cuda") * 0.2 + 1, torch.randn(D, generator=gen, device="cuda") * 0.1
    tok, nxt = next(example.batches(7))
    dw, dgain, dbias = torch.zeros(R, D, device="cuda"), torch.ones(D, device="cuda"), torch.ones(D, device="cuda")
    model = example.Normed()
    loss = model.gradients(tok, nxt, codes, xhat, gain, bias, dw, dgain, dbias, accumulate=True)

    W, G, B = (t.double().requires_grad_() for t in (xhat, gain, bias))
    keep = (tok != example.PADDING).double()
    h = W[tok] * math.sqrt(D) * keep[:, None]
    c = h - h.mean(1, keepdim=True)
    y = c / (c.square().mean(1, keepdim=True) + float(torch.tensor(1e-5))).sqrt() * G + B
    want = -(torch.log_softmax(y @ W.t(), 1).gather(1, nxt[:, None])[:, 0] * keep).sum() / keep.sum()
    want.backward()
    want = want.detach()
    assert abs(float(loss) - float(want)) <= 1e-4 * float(want)
    # rows of the padding are zeros: their norm's gradient is 1 / sqrt(eps) times what comes in, nothing here
    for name, got, exact in (("weight", dw, W.grad), ("gain", dgain - 1, G.grad), ("bias", dbias - 1, B.grad)):
        assert float((got.double() - exact).norm()) <= 1e-4 * float(exact.norm()) + 2.0 ** -23 * exact.numel() ** 0.5, name


def test_answers_from_the_codes(example):
    """Every replayed token is what the definitions give from the one before: lookup, norm, product and draw on the CPU."""
    R, D, texts, length = example.ROWS, example.DIM, 24, 6
    gen = torch.Generator(device="cuda").manual_seed(4)
    codes = torch.randint(-64, 65, (R, D), generator=gen, device="cuda").to(torch.int8)
    gain, bias = torch.randn(D, generator=gen, device="cuda") * 0.2 + 1, torch.randn(D, generator=gen, device="cuda") * 0.1
    first = torch.randint(1, R, (texts,), generator=gen, device="cuda")
    got = example.answer(codes, gain, bias, first, length, top_k=5, temperature=2.0)
    assert got.shape == (length, texts)
    u = torch.rand(length, texts, generator=torch.Generator(device="cuda").manual_seed(5), device="cuda")
    emb, norm, product = Embedding(R, D, 0), LayerNorm(D), Linear8(R, D, texts)
    tok = first
    for t in range(length):
        # the rows and their norm by the package, which other tests hold against 64 bits; from there on bit for bit
        h, y, logits = (torch.zeros(texts, n, device="cuda") for n in (D, D, R))
        emb.lookup(codes, tok, h, scale=math.sqrt(D), k_x=6)
        norm.forward(h, gain, bias, y)
        q, s = layer_util.token_codes(y)
        logits = layer_util.linear8(q, s, codes, 2.0 ** -7, None, torch.float32)
        want = [layer_util.sample(logits[r], u[t, r].item(), 2.0, 5, 1.0, 0.02) for r in range(texts)]
        assert got[t].tolist() == want, t
        tok = got[t]


def test_two_graphs_of_one_handle_in_turn(example):
    """Recorded calls share a handle's scratch: replayed one after the other on one stream they give what eager calls give."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    w = torch.randint(-128, 128, (700, 300), generator=gen, device="cuda").to(torch.int8)
    product, sampler, norm = Linear8(700, 300, 90), Sampler(700, 90), LayerNorm(300)
    sides = []
    stream = torch.cuda.Stream()
    for n in (90, 7):
        x = torch.randn(n, 300, generator=gen, device="cuda")
        u = torch.rand(n, generator=gen, device="cuda")
        b = dict(x=x, y=torch.zeros_like(x), logits=torch.zeros(n, 700, device="cuda"), u=u, out=torch.zeros(n, dtype=torch.int64, device="cuda"),
                 mean=torch.zeros(n, device="cuda"), rstd=torch.zeros(n, device="cuda"), dx=torch.zeros_like(x), dw=torch.zeros(300, device="cuda"))

        def run(b):
            norm.forward(b["x"], None, None, b["y"], b["mean"], b["rstd"])
            product.forward(b["y"], w, b["logits"], k_x=4)
            sampler.sample(b["logits"], b["u"], b["out"], top_k=3)
            norm.grad(b["y"], b["x"], None, b["mean"], b["rstd"], b["dx"], b["dw"])

        run(b)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            run(b)
        sides.append((graph, b, run))
    for k in range(3):
        for graph, b, run in sides:
            b["x"].mul_(1.5)
            graph.replay()
        torch.cuda.synchronize()
        for graph, b, run in sides:
            got = {n: t.clone() for n, t in b.items()}
            run(b)
            assert all(torch.equal(got[n], b[n]) for n in b), k
