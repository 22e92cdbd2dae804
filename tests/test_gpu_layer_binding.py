"""Calls of layer norm, the product and sampling through the checks in Python give what the natively checked calls give; what no call takes."""
import pytest
import torch

from paper_2004_14180_amd import LayerNorm, Linear8, Sampler, binding

pytestmark = pytest.mark.gpu


def _run():
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(3, 7, 40, generator=gen, device="cuda").bfloat16()
    w, b = torch.randn(40, generator=gen, device="cuda"), torch.randn(40, generator=gen, device="cuda")
    norm = LayerNorm(40)
    y, mean, rstd = torch.zeros_like(x), torch.zeros(3, 7, device="cuda"), torch.zeros(21, device="cuda")
    norm.forward(x, w, b, y, mean, rstd)
    dx, dw, db = torch.zeros_like(x), torch.ones(40, device="cuda"), torch.ones(40, device="cuda")
    norm.grad(y, x, w, mean, rstd, dx, dw, db, accumulate=True)
    codes = torch.randint(-64, 65, (50, 40), generator=gen, device="cuda").to(torch.int8)
    product = Linear8(50, 40, 21)
    out, out2 = torch.zeros(21, 50, device="cuda"), torch.zeros(3, 7, 50, device="cuda").half()
    product.forward(y, codes, out, k_x=6)
    ints, scales = torch.zeros(21, 40, dtype=torch.int8, device="cuda"), torch.zeros(21, device="cuda")
    product.quantize(y, ints, scales)
    product.forward(ints, codes, out2, weight_scales=torch.rand(50, generator=gen, device="cuda"), x_scales=scales, bias=torch.ones(50, device="cuda").half())
    u = torch.rand(21, generator=gen, device="cuda")
    sampler = Sampler(50, 21)
    t64, t32 = torch.zeros(21, dtype=torch.int64, device="cuda"), torch.zeros(3, 7, dtype=torch.int32, device="cuda")
    sampler.sample(out, u, t64, temperature=2.0, top_k=9, top_p=0.8, min_p=0.01)
    sampler.sample(out2, u, t32, temperature=torch.rand(21, generator=gen, device="cuda"), top_k=torch.full((21,), 4, dtype=torch.int32, device="cuda"))
    return [y, mean, rstd, dx, dw, db, out, out2, ints, scales, t64, t32]


def test_both_ways_give_the_same(monkeypatch):
    want = _run()
    assert not isinstance(binding._native, binding._Unavailable)
    monkeypatch.setattr(binding, "_native", binding._Unavailable())
    for a, b in zip(_run(), want):
        assert torch.equal(a, b)


@pytest.fixture(params=["native checks", "checks in Python"])
def ways(request, monkeypatch):
    binding.load_library()
    if request.param == "checks in Python":
        monkeypatch.setattr(binding, "_native", binding._Unavailable())


@pytest.mark.parametrize("other", [None, 1.0, [1.0], "x"])
def test_what_is_no_tensor(ways, other):
    f, n, v = torch.ones(4, 8, device="cuda"), torch.ones(4, device="cuda"), torch.ones(8, device="cuda")
    c, t = torch.ones(4, 8, dtype=torch.int8, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    out = torch.ones(4, 4, device="cuda")
    norm, product, sampler = LayerNorm(8), Linear8(4, 8, 4), Sampler(8, 4)
    calls = [lambda: norm.forward(other, v, v, f), lambda: norm.forward(f, v, v, other), lambda: norm.grad(other, f, v, n, n, f),
             lambda: norm.grad(f, other, v, n, n, f), lambda: norm.grad(f, f, v, other, n, f), lambda: norm.grad(f, f, v, n, n, other),
             lambda: product.forward(other, c, out, k_x=6), lambda: product.forward(f, other, out, k_x=6), lambda: product.forward(f, c, other, k_x=6),
             lambda: product.quantize(other, c, n), lambda: product.quantize(f, other, n), lambda: product.quantize(f, c, other),
             lambda: sampler.sample(other, n, t), lambda: sampler.sample(f, other, t), lambda: sampler.sample(f, n, other)]
    if other is not None:
        calls += [lambda: norm.forward(f, other, v, f), lambda: norm.forward(f, v, other, f), lambda: norm.forward(f, v, v, f, mean=other),
                  lambda: norm.grad(f, f, v, n, n, f, dweight=other), lambda: product.forward(f, c, out, weight_scales=other),
                  lambda: product.forward(c, c, out, k_x=6, x_scales=other), lambda: product.forward(f, c, out, k_x=6, bias=other)]
    for k, call in enumerate(calls):
        with pytest.raises(ValueError, match="expected a tensor"):
            call()
    assert (f == 1).all() and (c == 1).all() and (out == 1).all()


@pytest.mark.parametrize("accumulate", [True, 1, 2, "yes", False, 0, None, []])
def test_accumulate_is_a_truth_value(ways, accumulate):
    f, n = torch.ones(3, 8, device="cuda"), torch.ones(3, device="cuda")
    dw, db = torch.full((8,), 2.0, device="cuda"), torch.full((8,), 2.0, device="cuda")
    LayerNorm(8).grad(f, f * 2, None, n, n, torch.zeros(3, 8, device="cuda"), dw, db, accumulate=accumulate)
    assert (dw == 3.0 + (2.0 if accumulate else 0.0)).all() and (db == 3.0 + (2.0 if accumulate else 0.0)).all()


def test_filters_that_are_no_numbers(ways):
    f, n, t = torch.ones(4, 8, device="cuda"), torch.ones(4, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    q = Sampler(8, 4)
    for kw in (dict(temperature="x"), dict(temperature=None), dict(top_k="3"), dict(top_k=None), dict(top_k=2.5), dict(top_p=[0.5]), dict(min_p=None),
               dict(top_k=1 << 31), dict(top_k=-(1 << 31) - 1)):
        with pytest.raises((ValueError, TypeError)):
            q.sample(f, n, t, **kw)
    assert (t == 0).all()
