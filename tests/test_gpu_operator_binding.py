"""The operators' calls through the checks in Python give what the natively checked calls give."""
import pytest
import torch

from paper_2004_14180_amd import AdamW, AdamWConfig, Embedding, GradNorm, adamw_state, binding

pytestmark = pytest.mark.gpu


def _run():
    gen = torch.Generator(device="cuda").manual_seed(1)
    cfg = AdamWConfig(state_bits=8)
    params = [torch.randn(n, generator=gen, device="cuda") for n in (5, 3000)]
    grads = [torch.randn(n, generator=gen, device="cuda").bfloat16() for n in (5, 3000)]
    norm, clip = GradNorm([5, 3000], torch.bfloat16), torch.zeros(2, device="cuda")
    opt = AdamW(cfg, params, weight_decay=[0.0, 0.1], grad_dtype=torch.bfloat16, **adamw_state(cfg, params))
    norm.grad_norm(grads, 1.0, clip)
    opt.step(1, 1e-2, grads, grad_scale=clip[1:])
    opt.step(2, 1e-2, (None, grads[1]))
    emb = Embedding(50, 24, 300)
    tok = torch.randint(0, 50, (3, 100), generator=gen, device="cuda")
    codes = torch.randint(-64, 65, (50, 24), generator=gen, device="cuda").to(torch.int8)
    out, grad = torch.zeros(3, 100, 24, device="cuda").half(), torch.ones(50, 24, device="cuda")
    emb.lookup(codes, tok, out, scale=2.0, k_x=6, padding_idx=7)
    emb.grad(tok, out, grad, scale=0.5, padding_idx=7, accumulate=True)
    wide = torch.zeros(3, 100, 30, device="cuda")[..., :24]             # rows that only the checks in Python take
    emb.lookup(codes, tok, wide, k_x=6)
    return params + [clip, out, grad, wide]


def test_both_ways_give_the_same(monkeypatch):
    want = _run()
    assert not isinstance(binding._native, binding._Unavailable)
    monkeypatch.setattr(binding, "_native", binding._Unavailable())
    for a, b in zip(_run(), want):
        assert torch.equal(a, b)
