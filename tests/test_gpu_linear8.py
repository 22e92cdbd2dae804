"""The product of tokens with 8-bit integers, bit for bit against its operations one by one."""
import pytest
import torch

from layer_util import linear8, token_codes
from operator_util import BF16, F16, F32
from paper_2004_14180_amd import Linear8, QAdamError, binding

pytestmark = pytest.mark.gpu


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _weights(gen, outputs, inputs, gap=0, offset=0):
    """Integers of all of int8, rows `gap` apart, at an address `offset` bytes behind one of 256."""
    whole = torch.randint(-128, 128, (offset + outputs * (inputs + gap),), generator=gen, device="cuda").to(torch.int8)
    return whole[offset:].view(outputs, inputs + gap)[:, :inputs]


def _same(got, want):
    got, want = got.cpu(), want.cpu()
    same = (got == want) | (got.isnan() & want.isnan())
    assert same.all(), "%d of %d differ, first at %s" % (int((~same).sum()), same.numel(), (~same).nonzero()[0].tolist())


def _check(tokens, inputs, outputs, xt=BF16, ot=BF16, scales=True, bias=None, gap=0, offset=0, out_gap=0):
    gen = _gen(tokens * 7 + inputs)
    x = (torch.randn(tokens, inputs + gap, generator=gen, device="cuda") * 3).to(xt)[:, :inputs]
    w = _weights(gen, outputs, inputs, gap, offset)
    unit = torch.rand(outputs, generator=gen, device="cuda") * 0.01 if scales else 2.0 ** -7
    b = None if bias is None else torch.randn(outputs, generator=gen, device="cuda").to(bias)
    whole = torch.full((tokens, outputs + out_gap), 7.0, device="cuda").to(ot)
    out = whole[:, :outputs]
    codes, s = token_codes(x)
    want = linear8(codes, s, w, unit, b, ot)
    q = Linear8(outputs, inputs, tokens)
    kw = dict(weight_scales=unit) if scales else dict(k_x=6)
    q.forward(x, w, out, bias=b, **kw)
    _same(out, want)
    assert (whole[:, outputs:] == 7).all()
    got_codes, got_s = torch.full((tokens, inputs + 3), 7, dtype=torch.int8, device="cuda"), torch.zeros(tokens, device="cuda")
    q.quantize(x, got_codes[:, :inputs], got_s)
    assert torch.equal(got_codes[:, :inputs].cpu(), codes) and torch.equal(got_s.cpu(), s) and (got_codes[:, inputs:] == 7).all()
    out.fill_(7.0)
    q.forward(got_codes[:, :inputs], w, out, x_scales=got_s, bias=b, **kw)
    _same(out, want)


@pytest.mark.parametrize("tokens", [1, 2, 15, 16, 17, 33, 64, 65, 128, 129, 300])
@pytest.mark.parametrize("inputs,outputs", [(64, 64), (768, 1000), (2048, 513), (1, 1), (15, 17), (127, 129), (128, 128), (1001, 257)])
def test_sizes(tokens, inputs, outputs):
    _check(tokens, inputs, outputs, bias=F32)


@pytest.mark.parametrize("tokens", [1, 20, 200, 700])
@pytest.mark.parametrize("inputs,gap,offset", [(256, 0, 0), (256, 0, 1), (256, 16, 0), (256, 16, 16), (250, 6, 3), (96, 32, 5), (2047, 0, 0), (2064, 0, 0)])
def test_addresses_of_the_weights(tokens, inputs, gap, offset):
    _check(tokens, inputs, 391, gap=gap, offset=offset, out_gap=3)


@pytest.mark.parametrize("xt", [F32, BF16, F16])
@pytest.mark.parametrize("ot", [F32, BF16, F16])
@pytest.mark.parametrize("bias", [None, F32, BF16, F16])
@pytest.mark.parametrize("tokens", [3, 70, 260])
def test_types(xt, ot, bias, tokens):
    _check(tokens, 200, 300, xt, ot, scales=bias is None, bias=bias)


@pytest.mark.parametrize("tokens,inputs,outputs", [(1, 131071, 40), (2, 100_003, 33), (130, 20_000, 300), (2000, 512, 1500), (1, 768, 50257), (4096, 128, 70),
                                                   (9, 8192, 4096), (1100, 1024, 2304)])
def test_large(tokens, inputs, outputs):
    _check(tokens, inputs, outputs, F16, F32)


@pytest.mark.parametrize("tokens,inputs,outputs,gap,offset", [(5003, 272, 5001, 0, 0), (5000, 128, 5120, 0, 0), (4800, 1040, 5300, 48, 32), (5003, 272, 5001, 0, 3),
                                                             (5003, 250, 5001, 6, 0), (12800, 16, 2048, 0, 0), (130, 400, 99_999, 0, 0)])
def test_many_tiles(tokens, inputs, outputs, gap, offset):
    _check(tokens, inputs, outputs, BF16, BF16, bias=F32, gap=gap, offset=offset, out_gap=1)
    _check(tokens, inputs, outputs, BF16, F32, scales=False, gap=gap, offset=offset)


# inputs of a token that several workgroups take: 2 to 16 parts of them, of equal and of different lengths, weights at any address
@pytest.mark.parametrize("tokens,outputs", [(17, 1), (32, 64), (33, 300), (64, 2048), (65, 1000), (130, 1027), (500, 700)])
@pytest.mark.parametrize("inputs,gap,offset", [(1024, 0, 1), (1023, 0, 0), (4096, 0, 0), (4224, 16, 0), (8192, 0, 0), (8191, 2, 7), (33_000, 8, 0)])
def test_inputs_shared_by_workgroups(tokens, outputs, inputs, gap, offset):
    _check(tokens, inputs, outputs, BF16, F32, bias=F16, gap=gap, offset=offset, out_gap=2)


def test_inputs_shared_in_turn():
    """Calls of one handle in which tiles have many, few and no parts, one behind the other without a wait."""
    gen = _gen(11)
    inputs, outputs, most = 8192, 200, 300
    x, w = torch.randn(most, inputs, generator=gen, device="cuda"), _weights(gen, outputs, inputs)
    unaligned = torch.empty(outputs * inputs + 1, dtype=torch.int8, device="cuda")[1:].view(outputs, inputs).copy_(w)
    codes, s = token_codes(x)
    want = linear8(codes, s, w, 2.0 ** -7, None, F32).cuda()
    q, same = Linear8(outputs, inputs, most), Linear8(outputs, inputs, most)
    codes, s = codes.cuda(), s.cuda()
    outs = []
    for repeat in range(20):
        for n in (300, 17, 64, 1, 129, 65):
            out, second, third = (torch.full((n, outputs), 9.0, device="cuda") for _ in range(3))
            q.forward(x[:n], w, out, k_x=6)
            same.forward(x[:n], unaligned, second, k_x=6)
            q.forward(codes[:n], w, third, k_x=6, x_scales=s[:n])
            outs.append((n, out, second, third))
    for n, *got in outs:
        for out in got:
            assert torch.equal(out, want[:n]), n


def test_the_largest_sums():
    """Sums of -128 * -128 over the most inputs: just below 2^31."""
    inputs = (1 << 17) - 1
    for tokens in (1, 40, 150):
        x = torch.full((tokens, inputs), -128, dtype=torch.int8, device="cuda")
        w = torch.full((3, inputs), -128, dtype=torch.int8, device="cuda")
        w[1] = 127
        out = torch.zeros(tokens, 3, device="cuda")
        Linear8(3, inputs, tokens).forward(x, w, out, weight_scales=torch.ones(3, device="cuda"), x_scales=torch.ones(tokens, device="cuda"))
        want = torch.tensor([float(16384 * inputs), -float(16256 * inputs), float(16384 * inputs)])
        assert torch.equal(out.cpu(), want.expand(tokens, 3))


def test_tokens_at_the_ends_of_the_range():
    inputs = 300
    x = torch.randn(9, inputs, generator=_gen(1), device="cuda")
    x[0] = 0.0
    x[1] = 1e-38
    x[2] *= 1e37
    x[3, 7] = float("nan")
    x[4, 8] = float("inf")
    x[5, 9] = -float("inf")
    x[6] = -x[6].abs()
    x[7] = 2.0 ** -116
    x[8] = 2.5                                      # every element its own largest
    codes, s = token_codes(x)
    assert s[3:6].isnan().all() and (codes[3:6] == 0).all() and s[0] == 0 and s[1] == 0 and s[7] > 0 and (codes[8] == 127).all()
    w = _weights(_gen(2), 40, inputs)
    out, got, gs = torch.zeros(9, 40, device="cuda"), torch.zeros(9, inputs, dtype=torch.int8, device="cuda"), torch.zeros(9, device="cuda")
    q = Linear8(40, inputs, 9)
    q.quantize(x, got, gs)
    assert torch.equal(got.cpu(), codes)
    _same(gs, s)
    q.forward(x, w, out, k_x=3)
    _same(out, linear8(codes, s, w, 2.0 ** -4, None, F32))
    assert out[3:6].isnan().all() and out[:2].isfinite().all()      # row 2: 300 products of up to 3e37 * 8 pass fp32's range, and are compared above
    for k in range(9):                              # one at a time, where they are made integers on the way
        one = torch.zeros(1, 40, device="cuda")
        q.forward(x[k:k + 1], w, one, k_x=3)
        _same(one, out[k:k + 1])


def test_ties_and_halves():
    x = torch.arange(-127, 128, device="cuda").float()[None] * 0.5          # halves: to even
    x = torch.cat([x, torch.full((1, 1), 127.0, device="cuda")], 1)
    codes, s = token_codes(x)
    got, gs = torch.zeros(1, 256, dtype=torch.int8, device="cuda"), torch.zeros(1, device="cuda")
    Linear8(1, 256, 1).quantize(x, got, gs)
    assert torch.equal(got.cpu(), codes) and torch.equal(gs.cpu(), s)


def test_layouts_and_no_tokens():
    q = Linear8(24, 40, 30)
    gen = _gen(4)
    x, w = torch.randn(2, 3, 5, 40, generator=gen, device="cuda"), _weights(gen, 24, 40)
    out, want = torch.zeros(2, 15, 24, device="cuda"), torch.zeros(30, 24, device="cuda")
    q.forward(x.view(30, 40), w, want, k_x=6)
    q.forward(x, w, out, k_x=6)
    assert torch.equal(out.view(30, 24), want)
    wide = torch.full((30, 50), 7.0, device="cuda")
    q.forward(x, w, wide.view(2, 15, 50)[..., 3:27], k_x=6)             # a form that only the checks in Python take
    assert torch.equal(wide[:, 3:27], want) and (wide[:, :3] == 7).all() and (wide[:, 27:] == 7).all()
    q.forward(x[0, 0, :1].expand(7, 40), w, out.view(30, 24)[:7], k_x=6)
    assert torch.equal(out.view(30, 24)[:7], want[:1].expand(7, 24))
    q.forward(torch.zeros(0, 40, device="cuda"), w, torch.zeros(0, 24, device="cuda"), k_x=6)


@pytest.mark.parametrize("native", [True, False])
def test_no_tokens_in_integers(native, monkeypatch):
    """An empty batch in integers is as good as one in floats; scales beside floats are refused there too."""
    q, w = Linear8(24, 40, 30), _weights(_gen(6), 24, 40)
    if not native:
        monkeypatch.setattr(binding, "_native", binding._Unavailable())
    x, codes, scales = torch.zeros(0, 40, device="cuda"), torch.zeros(0, 40, dtype=torch.int8, device="cuda"), torch.zeros(0, device="cuda")
    out = torch.zeros(0, 24, device="cuda")
    q.quantize(x, codes, scales)
    q.forward(codes, w, out, k_x=6, x_scales=scales)
    q.forward(codes, w, out, weight_scales=torch.ones(24, device="cuda"), x_scales=scales, bias=torch.ones(24, device="cuda"))
    for kw in (dict(x=x, x_scales=scales), dict(x=codes), dict(x=x, x_scales=torch.ones(1, device="cuda"))):
        with pytest.raises(ValueError):
            q.forward(weight=w, out=out, k_x=6, **kw)
    # at the boundary: no tokens in integers need no scales, one does, and floats never take any
    one, y = torch.zeros(1, 40, device="cuda"), torch.zeros(1, 24, device="cuda")
    call = lambda n, kind, at: q._lib.qadam_linear8_forward(q._h, n, one.data_ptr(), kind, 40, at, w.data_ptr(), 40, None, 6, None, 0,  # noqa: E731
                                                            y.data_ptr(), binding.QADAM_F32, 24, None)
    assert call(0, binding.QADAM_CODES8, None) == 0 and call(0, binding.QADAM_CODES8, one.data_ptr()) == 0
    assert call(1, binding.QADAM_CODES8, None) == -1
    assert call(0, binding.QADAM_F32, one.data_ptr()) == -1 and call(1, binding.QADAM_F32, one.data_ptr()) == -1


@pytest.mark.parametrize("tokens,inputs,outputs", [(1, 768, 3000), (20, 768, 3000), (40, 768, 3000), (300, 768, 3000), (40, 8192, 192), (20, 2047, 500), (2500, 128, 3000), (5000, 128, 5120)])
def test_recorded_calls(tokens, inputs, outputs):
    gen = _gen(5)
    x, w = torch.randn(tokens, inputs, generator=gen, device="cuda"), _weights(gen, outputs, inputs)
    q = Linear8(outputs, inputs, tokens)
    got, want = torch.zeros(tokens, outputs, device="cuda"), torch.zeros(tokens, outputs, device="cuda")
    q.forward(x, w, got, k_x=6)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        q.forward(x, w, got, k_x=6)
    for k in range(4):
        x.mul_(-1.5)
        w.add_(1)
        got.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        q.forward(x, w, want, k_x=6)
        assert torch.equal(got, want), k


@pytest.mark.parametrize("tokens", [1, 30, 5000])
def test_another_stream(tokens):
    gen = _gen(8)
    x, w = torch.randn(tokens, 144, generator=gen, device="cuda"), _weights(gen, 5120, 144)
    q, side = Linear8(5120, 144, tokens), torch.cuda.Stream()
    out, want = torch.zeros(tokens, 5120, device="cuda"), torch.zeros(tokens, 5120, device="cuda")
    q.forward(x, w, want, k_x=6)
    torch.cuda.synchronize()
    q.forward(x, w, out, k_x=6, stream=side)
    side.synchronize()
    assert torch.equal(out, want)


def test_more_than_2_to_31_elements():
    """Results and weights beyond 32-bit offsets."""
    gen = _gen(9)
    tokens, inputs, outputs = 70_000, 16, 33_000
    x, w = torch.randn(tokens, inputs, generator=gen, device="cuda"), _weights(gen, outputs, inputs)
    out = torch.empty(tokens, outputs, dtype=BF16, device="cuda")
    assert out.numel() > 1 << 31
    Linear8(outputs, inputs, tokens).forward(x, w, out, k_x=6)
    for rows in (slice(0, 3), slice(65_070, 65_080), slice(tokens - 3, tokens)):
        codes, s = token_codes(x[rows])
        _same(out[rows], linear8(codes, s, w, 2.0 ** -7, None, BF16))
    del out
    outputs, stride = 40, 60_000_001                    # rows of the weights far apart
    whole = torch.zeros(outputs * stride, dtype=torch.int8, device="cuda")
    w = whole.view(outputs, stride)[:, 1:1 + inputs]
    w.copy_(_weights(gen, outputs, inputs))
    for n in (1, 33, 400):
        codes, s = token_codes(x[:n])
        out = torch.zeros(n, outputs, device="cuda")
        Linear8(outputs, inputs, n).forward(x[:n], w, out, k_x=6)
        _same(out, linear8(codes, s, w, 2.0 ** -7, None, F32))


def test_refusals():
    q = Linear8(8, 16, 4)
    z = lambda *s, **k: torch.zeros(*s, device="cuda", **k)  # noqa: E731
    i8 = dict(dtype=torch.int8)
    good = dict(x=z(4, 16), weight=z(8, 16, **i8), out=z(4, 8), k_x=6)
    q.forward(**good)
    for kw in (dict(x=z(4, 15)), dict(x=z(4, 16).double()), dict(x=z(4, 16, **i8)), dict(weight=z(8, 16)), dict(weight=z(7, 16, **i8)), dict(k_x=None),
               dict(k_x=7), dict(k_x=-1), dict(weight_scales=z(8)), dict(k_x=None, weight_scales=z(7)), dict(k_x=None, weight_scales=z(8).half()),
               dict(out=z(4, 9)), dict(out=z(3, 8)), dict(out=z(4, 8, **i8)), dict(out=z(1, 8).expand(4, 8)), dict(bias=z(9)), dict(bias=z(8, **i8)),
               dict(x=z(5, 16), out=z(5, 8)), dict(x_scales=z(4)), dict(x=z(4, 16, **i8), x_scales=z(3)), dict(weight=z(1, 16, **i8).expand(8, 16)),
               dict(x=None), dict(weight=None), dict(out=None), dict(x=z(4, 16).cpu()), dict(k_x=1 << 33), dict(weight=z(16, 8, **i8).t())):
        with pytest.raises((ValueError, QAdamError)):
            q.forward(**{**good, **kw})
    for args in ((z(4, 16), z(4, 16), z(4)), (z(4, 16), z(4, 16, **i8), z(3)), (z(4, 16, **i8), z(4, 16, **i8), z(4)), (z(4, 16), z(4, 15, **i8), z(4))):
        with pytest.raises((ValueError, QAdamError)):
            q.quantize(*args)
    for bad in [(0, 1, 1), (1, 0, 1), (1, 1, -1), (1, 1 << 17, 1), ((1 << 24) + 1, 1, 1), (1, 1, (1 << 24) + 1), (1, 100_000, 1 << 24)]:
        with pytest.raises(QAdamError):
            Linear8(*bad)
