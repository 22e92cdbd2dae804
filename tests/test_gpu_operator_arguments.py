"""Arguments that the operators' calls refuse, whichever checks a call goes through, and what they take alike."""
import pytest
import torch

from paper_2004_14180_amd import AdamW, AdamWConfig, Embedding, GradNorm, adamw_state, binding

pytestmark = pytest.mark.gpu


@pytest.fixture(params=["native checks", "checks in Python"])
def ways(request, monkeypatch):
    binding.load_library()
    if request.param == "checks in Python":
        monkeypatch.setattr(binding, "_native", binding._Unavailable())


def test_integers_beyond_the_boundary_types(ways):
    codes, tok = torch.ones(4, 8, dtype=torch.int8, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    out, grad = torch.full((3, 8), 7.0, device="cuda"), torch.full((4, 8), 7.0, device="cuda")
    emb = Embedding(4, 8, 3)
    for kw in (dict(k_x=(1 << 32) + 3), dict(k_x=3, padding_idx=1 << 64), dict(k_x=-(1 << 32))):
        with pytest.raises(ValueError, match="does not fit"):
            emb.lookup(codes, tok, out, **kw)
    with pytest.raises(ValueError, match="does not fit"):
        emb.grad(tok, out, grad, padding_idx=(1 << 64) + 2)
    params, cfg = [torch.ones(5, device="cuda")], AdamWConfig()
    with pytest.raises(ValueError, match="does not fit"):
        AdamW(cfg, params, **adamw_state(cfg, params)).step((1 << 64) + 1, 1e-3, [torch.ones(5, device="cuda")])
    assert (out == 7).all() and (grad == 7).all() and (params[0] == 1).all()


@pytest.mark.parametrize("accumulate", [True, 1, 2, -1, "yes", [0], False, 0, None, []])
def test_accumulate_is_a_truth_value(ways, accumulate):
    tok, dout, grad = torch.zeros(3, dtype=torch.int64, device="cuda"), torch.ones(3, 8, device="cuda"), torch.full((4, 8), 2.0, device="cuda")
    Embedding(4, 8, 3).grad(tok, dout, grad, accumulate=accumulate)
    before = 2.0 if accumulate else 0.0
    assert (grad[0] == 3.0 + before).all() and (grad[1:] == before).all()


@pytest.mark.parametrize("other", [None, 1.0, [1.0], "x"])
def test_what_is_no_tensor(ways, other):
    f32, tok = torch.ones(4, 8, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    emb, cfg = Embedding(4, 8, 4), AdamWConfig()
    calls = [lambda: emb.lookup(other, tok, f32), lambda: emb.lookup(f32, other, f32), lambda: emb.lookup(f32, tok, other),
             lambda: emb.grad(other, f32, f32), lambda: emb.grad(tok, other, f32), lambda: emb.grad(tok, f32, other),
             lambda: AdamW(cfg, [other], [f32], [f32]), lambda: AdamW(cfg, [f32], [other], [f32]),
             lambda: GradNorm([32]).grad_norm([f32], 1.0, other)]
    if other is not None:           # None: no copy, no gradient, no factor
        opt = AdamW(cfg, [f32], **adamw_state(cfg, [f32]))
        calls += [lambda: AdamW(cfg, [f32], [f32], [f32], copies=[other]), lambda: opt.step(1, 1e-3, [other]),
                  lambda: opt.step(1, 1e-3, [f32], grad_scale=other), lambda: GradNorm([32]).grad_norm([other], 1.0, torch.zeros(2, device="cuda"))]
    for k, call in enumerate(calls):
        with pytest.raises(ValueError, match="expected a tensor"):
            call()
    assert (f32 == 1).all()
