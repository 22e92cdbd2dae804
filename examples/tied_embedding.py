"""Next-token model of one tied embedding matrix, trained with the package's operators together.

    python examples/tied_embedding.py [--optimizer adamw|qadam] [--steps 300]

h = scale W[token], logits = h W^T, cross-entropy with the next token of a synthetic first-order chain.  The products and the loss are
torch's; the rest of a step is the package's:

  adamw   lookup -> (loss) -> the embedding's gradient added to the head's -> norm of all gradients and clipping factor -> AdamW with
          8-bit states, weights in fp32 and their bfloat16 copy, which the model computes with; nothing waits for the GPU;
  qadam   two workers look up their tokens straight in the 8-bit weight codes that the quantized step emitted, write their gradients
          into the flat vectors that it reads, and the step makes the next codes.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2004_14180_amd import AdamW, AdamWConfig, Embedding, GradNorm, QAdam, QAdamConfig, adamw_state  # noqa: E402

ROWS, DIM, TOKENS, PADDING = 1000, 64, 4096, 0


def batches(seed):
    """Endless (tokens, next tokens) of a chain in which four tokens can follow each; the first row is the padding of short texts."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    follow = torch.randint(1, ROWS, (ROWS, 4), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
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


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--optimizer", choices=["adamw", "qadam"], default="adamw")
    ap.add_argument("--steps", type=int, default=300)
    args = ap.parse_args(argv)
    losses = train_adamw(args.steps) if args.optimizer == "adamw" else train_qadam(args.steps)
    print("%s: loss %.3f -> %.3f in %d steps (uniform %.3f, the chain's own %.3f)" %
          (args.optimizer, losses[0], losses[-1], args.steps, math.log(ROWS), math.log(4)))
    return losses


if __name__ == "__main__":
    main()
