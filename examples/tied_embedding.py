"""Next-token model of one tied embedding matrix, trained with the package's operators together.

    python examples/tied_embedding.py [--optimizer adamw|qadam|normed] [--steps 300]

h = scale W[token], logits = h W^T, cross-entropy with the next token of a synthetic first-order chain.  The products and the loss are
torch's; the rest of a step is the package's:

  adamw   lookup -> (loss) -> the embedding's gradient added to the head's -> norm of all gradients and clipping factor -> AdamW with
          8-bit states, weights in fp32 and their bfloat16 copy, which the model computes with; nothing waits for the GPU;
  qadam   two workers look up their tokens straight in the 8-bit weight codes that the quantized step emitted, write their gradients
          into the flat vectors that it reads, and the step makes the next codes;
  normed  as qadam, with a layer norm between the rows and the head: its weights lie around one, which the codes' grid does not reach, and
          are trained by AdamW.  Then the model answers from the codes alone: lookup -> layer norm -> product with the codes in 8-bit
          integers -> a sampled token, recorded into a graph that is replayed for every token.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2004_14180_amd import (AdamW, AdamWConfig, Embedding, GradNorm, LayerNorm, Linear8, QAdam, QAdamConfig, Sampler,  # noqa: E402
                                  adamw_state)

ROWS, DIM, TOKENS, PADDING = 1000, 64, 4096, 0


def followers():
    """The four tokens that can follow each."""
    return torch.randint(1, ROWS, (ROWS, 4), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")


def batches(seed):
    """Endless (tokens, next tokens) of a chain in which four tokens can follow each; the first row is the padding of short texts."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    follow = followers()
    while True:
        tok = torch.randint(1, ROWS, (TOKENS,), generator=gen, device="cuda")
        pick = torch.randint(0, 4, (TOKENS,), generator=gen, device="cuda")
        nxt = follow[tok, pick]
        tok[-TOKENS // 16:] = PADDING
        yield tok, nxt


def head(h, weight, nxt, tok):
    """(loss, gradient of h, gradient of the tied weight) of the output head; padded tokens have no loss."""
    keep = (tok != PADDING).float()
    p = torch.softmax(h.float() @ weight.float().t(), 1)
    loss = -(p.gather(1, nxt[:, None]).clamp_min(1e-30).log()[:, 0] * keep).sum() / keep.sum()
    p.scatter_add_(1, nxt[:, None], torch.full_like(nxt[:, None], -1.0, dtype=torch.float32))
    p *= (keep / keep.sum())[:, None]
    return loss, p @ weight.float(), p.t() @ h.float()


def train_adamw(steps):
    weight = torch.randn(ROWS, DIM, generator=torch.Generator(device="cuda").manual_seed(0), device="cuda") * 0.1
    bias = torch.zeros(DIM, device="cuda")                      # a second tensor: added to the looked-up rows, without decay
    params = [weight, bias]
    copies = [weight.bfloat16(), None]
    cfg = AdamWConfig(beta1=0.9, beta2=0.99, state_bits=8)
    opt = AdamW(cfg, params, copies=copies, weight_decay=[0.01, 0.0], **adamw_state(cfg, params))
    norm, clip = GradNorm([p.numel() for p in params]), torch.zeros(2, device="cuda")
    emb = Embedding(ROWS, DIM, TOKENS)
    h = torch.empty(TOKENS, DIM, dtype=torch.bfloat16, device="cuda")
    losses, data, scale = [], batches(2), math.sqrt(DIM)
    for t in range(1, steps + 1):
        tok, nxt = next(data)
        emb.lookup(copies[0], tok, h, scale=scale, padding_idx=PADDING)
        loss, dh, dw = head(h.float() + bias, copies[0], nxt, tok)
        emb.grad(tok, dh, dw, scale=scale, padding_idx=PADDING, accumulate=True)
        grads = [dw, dh.sum(0)]
        norm.grad_norm(grads, 1.0, clip)
        opt.step(t, 1e-2 * min(1.0, 2.0 * (1.0 - t / (steps + 1))), grads, grad_scale=clip[1:])
        losses.append(loss)
    assert emb.get_status() == 0
    return [float(x) for x in losses]


def train_qadam(steps, workers=2):
    P = ROWS * DIM
    q = QAdam(QAdamConfig(k_g=2, k_x=6, weight_ef=0, beta1=0.9), [0, P], workers)
    x = torch.randn(P, generator=torch.Generator(device="cuda").manual_seed(0), device="cuda") * 0.1
    m, v, werr, xhat = (torch.zeros(P, device="cuda") for _ in range(4))
    errs = [torch.zeros(P, device="cuda") for _ in range(workers)]
    grads = [torch.zeros(P, device="cuda") for _ in range(workers)]
    codes = [torch.zeros(q.grad_code_bytes() // 4, dtype=torch.int32, device="cuda") for _ in range(workers)]
    scales = [torch.zeros(1, device="cuda") for _ in range(workers)]
    wcodes = torch.zeros(P, dtype=torch.int8, device="cuda")
    q.weight_quantize(1, x, werr, wcodes)
    emb = Embedding(ROWS, DIM, TOKENS)
    h = torch.empty(TOKENS, DIM, device="cuda")
    losses, data, scale = [], [batches(2 + i) for i in range(workers)], math.sqrt(DIM)
    for t in range(1, steps + 1):
        q.weight_dequantize(wcodes, xhat)                       # the head multiplies with the whole matrix
        total = 0.0
        for i in range(workers):
            tok, nxt = next(data[i])
            emb.lookup(wcodes.view(ROWS, DIM), tok, h, scale=scale, k_x=6, padding_idx=PADDING)
            loss, dh, dw = head(h, xhat.view(ROWS, DIM), nxt, tok)
            grads[i].copy_(dw.view(-1))
            emb.grad(tok, dh, grads[i].view(ROWS, DIM), scale=scale, padding_idx=PADDING, accumulate=True)
            total = total + loss / workers
        q.step_fused(t, 1e-2 * min(1.0, 2.0 * (1.0 - t / (steps + 1))), 0.99, grads, errs, codes, scales, x, m, v, werr, wcodes)
        losses.append(total)
    assert q.get_status() == 0 and emb.get_status() == 0
    return [float(x) for x in losses]


class Normed:
    """rows -> layer norm -> tied head, with the buffers of one batch."""

    def __init__(self, tokens=TOKENS):
        self.emb, self.norm = Embedding(ROWS, DIM, tokens), LayerNorm(DIM)
        self.h, self.y, self.dh = (torch.empty(tokens, DIM, device="cuda") for _ in range(3))
        self.mean, self.rstd = torch.empty(tokens, device="cuda"), torch.empty(tokens, device="cuda")

    def gradients(self, tok, nxt, codes, xhat, gain, bias, dw, dgain, dbias, accumulate):
        """The loss; the gradient of the tied weight into dw, those of the norm into dgain and dbias (with `accumulate` added to)."""
        scale = math.sqrt(DIM)
        self.emb.lookup(codes, tok, self.h, scale=scale, k_x=6, padding_idx=PADDING)
        self.norm.forward(self.h, gain, bias, self.y, self.mean, self.rstd)
        loss, dy, dhead = head(self.y, xhat, nxt, tok)
        self.norm.grad(dy, self.h, gain, self.mean, self.rstd, self.dh, dgain, dbias, accumulate=accumulate)
        dw.copy_(dhead)
        self.emb.grad(tok, self.dh, dw, scale=scale, padding_idx=PADDING, accumulate=True)
        return loss


def train_normed(steps, workers=2):
    P = ROWS * DIM
    q = QAdam(QAdamConfig(k_g=2, k_x=6, weight_ef=0, beta1=0.9), [0, P], workers)
    x = torch.randn(P, generator=torch.Generator(device="cuda").manual_seed(0), device="cuda") * 0.1
    m, v, werr, xhat = (torch.zeros(P, device="cuda") for _ in range(4))
    errs, grads = ([torch.zeros(P, device="cuda") for _ in range(workers)] for _ in range(2))
    codes = [torch.zeros(q.grad_code_bytes() // 4, dtype=torch.int32, device="cuda") for _ in range(workers)]
    scales = [torch.zeros(1, device="cuda") for _ in range(workers)]
    wcodes = torch.zeros(P, dtype=torch.int8, device="cuda")
    q.weight_quantize(1, x, werr, wcodes)
    gain, bias = torch.ones(DIM, device="cuda"), torch.zeros(DIM, device="cuda")
    dgain, dbias = torch.zeros(DIM, device="cuda"), torch.zeros(DIM, device="cuda")
    cfg = AdamWConfig(beta1=0.9, beta2=0.99)
    opt = AdamW(cfg, [gain, bias], **adamw_state(cfg, [gain, bias]))
    model, losses, data = Normed(), [], [batches(2 + i) for i in range(workers)]
    for t in range(1, steps + 1):
        q.weight_dequantize(wcodes, xhat)
        total, lr = 0.0, 1e-2 * min(1.0, 2.0 * (1.0 - t / (steps + 1)))
        for i in range(workers):
            tok, nxt = next(data[i])
            loss = model.gradients(tok, nxt, wcodes.view(ROWS, DIM), xhat.view(ROWS, DIM), gain, bias, grads[i].view(ROWS, DIM), dgain, dbias,
                                   accumulate=i > 0)
            total = total + loss / workers
        opt.step(t, lr, [dgain / workers, dbias / workers])
        q.step_fused(t, lr, 0.99, grads, errs, codes, scales, x, m, v, werr, wcodes)
        losses.append(total)
    assert q.get_status() == 0 and model.emb.get_status() == 0
    return [float(x) for x in losses], wcodes.view(ROWS, DIM), gain, bias


def answer(codes, gain, bias, first, length, top_k=8, temperature=1.0, seed=5):
    """`length` tokens behind each of `first`, from the weight codes alone: (length, texts)."""
    texts = first.numel()
    emb, norm, product, sampler = Embedding(ROWS, DIM, 0), LayerNorm(DIM), Linear8(ROWS, DIM, texts), Sampler(ROWS, texts)
    tok, h, logits = first.clone(), torch.empty(texts, DIM, device="cuda"), torch.empty(texts, ROWS, device="cuda")
    u = torch.rand(length, texts, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")
    now = u[0].clone()

    def step():
        emb.lookup(codes, tok, h, scale=math.sqrt(DIM), k_x=6)
        norm.forward(h, gain, bias, h)
        product.forward(h, codes, logits, k_x=6)
        sampler.sample(logits, now, tok, temperature=temperature, top_k=top_k, min_p=0.02)

    step()
    tok.copy_(first)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        step()
    out = []
    for t in range(length):
        now.copy_(u[t])
        graph.replay()
        out.append(tok.clone())
    assert emb.get_status() == 0 and sampler.get_status() == 0
    return torch.stack(out)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--optimizer", choices=["adamw", "qadam", "normed"], default="adamw")
    ap.add_argument("--steps", type=int, default=300)
    args = ap.parse_args(argv)
    if args.optimizer == "normed":
        losses, codes, gain, bias = train_normed(args.steps)
        first = torch.arange(1, 65, device="cuda")
        said = answer(codes, gain, bias, first, 32)
        before = torch.cat([first[None], said[:-1]])
        print("normed: %.0f %% of %d answered tokens can follow the one before" %
              (100.0 * (followers()[before] == said[..., None]).any(-1).float().mean(), said.numel()))
    else:
        losses = train_adamw(args.steps) if args.optimizer == "adamw" else train_qadam(args.steps)
    print("%s: loss %.3f -> %.3f in %d steps (uniform %.3f, the chain's own %.3f)" %
          (args.optimizer, losses[0], losses[-1], args.steps, math.log(ROWS), math.log(4)))
    return losses


if __name__ == "__main__":
    main()
