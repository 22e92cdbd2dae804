"""Sampled tokens against the definition: sorted logits, integer masses, one row at a time."""
import math

import pytest
import torch

import layer_util
from operator_util import BF16, F16, F32
from paper_2004_14180_amd import QAdamError, Sampler
from paper_2004_14180_amd.binding import QADAM_STATUS_NO_TOKEN

pytestmark = pytest.mark.gpu


def _at(v, r):
    return v[r].item() if isinstance(v, torch.Tensor) else v


def _check(logits, u, ids=torch.int64, sampler=None, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    rows, vocab = logits.shape
    q = sampler or Sampler(vocab, rows)
    out = torch.full((rows + 2,), -7, dtype=ids, device="cuda")
    q.sample(logits, u, out[1:-1], temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p)
    want = [layer_util.sample(logits[r], u[r].item(), _at(temperature, r), _at(top_k, r), _at(top_p, r), _at(min_p, r)) for r in range(rows)]
    assert out[1:-1].tolist() == want
    assert out[0] == -7 and out[-1] == -7
    assert q.get_status(clear=True) == (QADAM_STATUS_NO_TOKEN if -1 in want else 0)
    return want


def _logits(rows, vocab, dtype, seed=0, std=3.0, gap=0):
    gen = torch.Generator(device="cuda").manual_seed(seed + vocab)
    x = (torch.randn(rows, vocab + gap, generator=gen, device="cuda") * std).to(dtype)[:, :vocab]
    return x, torch.rand(rows, generator=gen, device="cuda")


@pytest.mark.parametrize("vocab", [1, 2, 3, 7, 8, 9, 17, 63, 64, 65, 1000, 1023, 1024, 1025, 4097, 32003, 50257, 70001])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_sizes_and_types(vocab, dtype):
    x, u = _logits(12, vocab, dtype, gap=3)
    _check(x, u)
    _check(x, u, torch.int32, top_k=40, top_p=0.9, temperature=0.7)
    _check(x, u, min_p=0.05)


@pytest.mark.parametrize("temperature", [0.0, 1e-30, 0.01, 0.3, 1.0, 3.0, 100.0, 1e30])
@pytest.mark.parametrize("top_k", [0, 1, 2, 50, 999, 5000, -3])
def test_filters(temperature, top_k):
    x, u = _logits(8, 3001, F32, seed=top_k)
    for top_p in (1.0, 0.95, 0.5, 1e-6, 0.0, -1.0, 2.0):
        for min_p in (0.0, 0.1, 1.0, 7.0, -1.0):
            _check(x, u, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p)


@pytest.mark.parametrize("min_p", [1e-30, 2.0 ** -41, 2.0 ** -40, 1.5 * 2.0 ** -40, 3e-12, 1e-9, 1e-4, 0.3, 0.9999999])
@pytest.mark.parametrize("top_k", [0, 30, 700])
def test_min_p_beside_the_others(min_p, top_k):
    """From half a unit of the masses on: the tokens that reach it are found in the bins, or in the list of the first ones."""
    for dtype, std, temperature in ((F32, 4.0, 1.0), (BF16, 4.0, 0.6), (F32, 30.0, 1.0), (F32, 0.01, 1.0)):
        x, u = _logits(6, 20011, dtype, seed=top_k, std=std)
        u[0] = 1.0 - 2.0 ** -24
        for top_p in (1.0, 0.999, 0.7):
            _check(x, u, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p)


@pytest.mark.parametrize("vocab", [100, 5000, 60000])
@pytest.mark.parametrize("levels", [1, 2, 5])
def test_equal_logits(vocab, levels):
    """Few different values: the lower index comes first, in whatever part of the row it lies."""
    gen = torch.Generator(device="cuda").manual_seed(vocab + levels)
    x = torch.randint(0, levels, (10, vocab), generator=gen, device="cuda").float()
    u = torch.rand(10, generator=gen, device="cuda")
    for dtype in (F32, BF16):
        for top_k in (0, 1, 7, vocab // 2, vocab - 1, vocab):
            for top_p in (1.0, 0.5, 0.25, 0.1):
                _check(x.to(dtype), u, top_k=top_k, top_p=top_p)


def test_zeros_of_both_signs_are_equal():
    x = torch.tensor([[-0.0, 0.0, -1.0, -0.0], [0.0, -0.0, 0.0, -5.0]], device="cuda")
    for u in (0.0, 0.2, 0.3, 0.5, 0.7, 0.9, 0.999):
        _check(x, torch.full((2,), u, device="cuda"), top_k=2)
        _check(x, torch.full((2,), u, device="cuda"))
        _check(x, torch.full((2,), u, device="cuda"), temperature=0.0)


def test_random_numbers_at_the_ends():
    x, _ = _logits(9, 777, F32)
    u = torch.tensor([0.0, -0.0, 1.0 - 2.0 ** -24, 1.0, 5.0, -3.0, float("nan"), float("inf"), 1e-45], device="cuda")
    for kw in (dict(), dict(top_k=5), dict(top_p=0.3), dict(min_p=0.2), dict(temperature=0.1)):
        _check(x, u, **kw)


@pytest.mark.parametrize("temperature", [1e37, 1.17e37, 1.2e37, 1e38, 3.4028234e38])
@pytest.mark.parametrize("vocab", [5, 300, 2047, 3000])
def test_temperatures_at_the_end_of_the_range(temperature, vocab):
    """Logits as far apart as fp32 has them, all of which have masses at such temperatures."""
    x, _ = _logits(8, vocab, F32)
    x[0, 3] = math.inf
    x[1, 2] = 3.4e38
    x[2, ::2], x[2, 1::2] = 3e38, -3e38
    x[3] = torch.linspace(-3.4e38, 3.4e38, vocab, dtype=torch.float64).float()
    x[4, 0], x[4, 1] = math.inf, -math.inf
    x[5, 1:] = torch.finfo(F32).min
    x[6, 4] = -3.4e38
    for u in (0.0, 0.4, 0.8, 0.97, 1.0 - 2.0 ** -24):
        us = torch.full((8,), u, device="cuda")
        for kw in (dict(), dict(top_k=2), dict(top_k=vocab - 1), dict(top_p=0.9), dict(min_p=0.02), dict(min_p=0.9), dict(top_k=900, top_p=0.99, min_p=0.001)):
            _check(x, us, temperature=temperature, **kw)
            _check(x, us, temperature=torch.full((8,), temperature, device="cuda"), **kw)


def test_masks_and_rows_without_a_token():
    x, u = _logits(12, 2000, F32)
    x[0] = -math.inf                                        # nothing left
    x[1, :-1] = -math.inf                                   # one left
    x[2, ::2] = -math.inf
    x[3, 5] = math.nan
    x[4, 6] = math.inf
    x[5, 100:110] = math.inf                                # ten of them share all mass
    x[6] = torch.finfo(F32).min                             # the type's lowest value everywhere is no mask
    x[7, 3:] = torch.finfo(F32).min
    x[8, :] = -math.inf
    x[8, 7] = math.nan
    x[9] = math.inf
    x[10] = -3e38
    x[10, 1999] = 3e38
    for kw in (dict(), dict(top_k=3), dict(top_p=0.6), dict(min_p=0.3), dict(temperature=0.0), dict(temperature=2.0, top_k=1500, top_p=0.99)):
        want = _check(x, u, **kw)
        assert [r for r, t in enumerate(want) if t < 0] == [0, 3, 8]
    for dtype in (BF16, F16):
        _check(x.clamp(-6e4, 6e4).to(dtype), u, top_p=0.9)
        _check(torch.where(x.abs() < 1e30, x, x.sign() * math.inf).to(dtype), u, top_p=0.9)


def test_filters_of_each_row():
    rows = 300
    x, u = _logits(rows, 1500, BF16)
    gen = torch.Generator(device="cuda").manual_seed(1)
    pick = lambda vs, dtype=F32: torch.tensor(vs, dtype=dtype, device="cuda")[torch.randint(0, len(vs), (rows,), generator=gen, device="cuda")]  # noqa: E731
    t, k = pick([0.0, 0.5, 1.0, 2.0]), pick([0, 1, 3, 100, 1499, 1500, 9999, -1], torch.int32)
    p, m = pick([1.0, 0.9, 0.5, 0.0, 2.0, math.nan]), pick([0.0, 0.1, 1.0, math.nan])
    _check(x, u, temperature=t, top_k=k, top_p=p, min_p=m)
    _check(x, u, temperature=t, top_k=20, top_p=0.9)
    t[5], t[6], t[7] = -1.0, math.nan, math.inf             # such a row has no token
    want = _check(x, u, temperature=t, top_k=k, top_p=p, min_p=m)
    assert want[5:8] == [-1, -1, -1]


def test_many_rows_and_one_row_for_all():
    x, u = _logits(3000, 600, F32)
    _check(x, u, top_k=30)
    _check(x[:1].expand(500, 600), u[:500], top_p=0.8)


def test_the_largest_vocabulary():
    """All masses equal and as large as they can be: their sum is 2^62."""
    x = torch.zeros(1, 1 << 22, device="cuda").half()
    for u in (0.0, 0.3, 1.0 - 2.0 ** -24):
        for kw in (dict(), dict(top_p=0.5), dict(top_k=(1 << 22) - 1), dict(min_p=1.0)):
            _check(x, torch.tensor([u], device="cuda"), **kw)


def test_more_rows_than_a_launch():
    rows = (1 << 21) + 3
    gen = torch.Generator(device="cuda").manual_seed(2)
    x, u = torch.randn(rows, 9, generator=gen, device="cuda").half(), torch.rand(rows, generator=gen, device="cuda")
    out = torch.full((rows,), -7, dtype=torch.int32, device="cuda")
    q = Sampler(9, rows)
    q.sample(x, u, out, temperature=0.0)
    top, first = x.max(1, keepdim=True).values, torch.arange(9, device="cuda")
    assert torch.equal(out.long(), torch.where(x == top, first, 9).min(1).values)
    q.sample(x, u, out, top_p=0.7)
    for r in (0, 1, (1 << 21) - 1, 1 << 21, rows - 1):
        assert out[r].item() == layer_util.sample(x[r], u[r].item(), 1.0, 0, 0.7, 0.0)
    assert q.get_status() == 0


def test_another_stream():
    x, u = _logits(64, 9000, F32)
    q, side = Sampler(9000, 64), torch.cuda.Stream()
    out, want = torch.zeros(64, dtype=torch.int64, device="cuda"), torch.zeros(64, dtype=torch.int64, device="cuda")
    q.sample(x, u, want, top_p=0.9)
    torch.cuda.synchronize()
    q.sample(x, u, out, top_p=0.9, stream=side)
    side.synchronize()
    assert torch.equal(out, want)


def test_a_large_vocabulary():
    x, u = _logits(3, 1 << 20, BF16)
    _check(x, u)
    _check(x, u, top_k=100_000, top_p=0.97, temperature=1.7)
    _check(x[:1] * 0, u[:1])                                # a million equal ones


def test_frequencies_follow_the_masses():
    x = torch.tensor([[2.0, 0.0, 1.0, -1.0]], device="cuda").expand(4096, 4)
    u = (torch.arange(4096, device="cuda") + 0.5) / 4096
    out = torch.zeros(4096, dtype=torch.int32, device="cuda")
    Sampler(4, 4096).sample(x, u, out, temperature=1.0)
    want = torch.softmax(x[0].double(), 0) * 4096
    assert ((torch.bincount(out, minlength=4).double() - want).abs() <= 1).all()


def test_recorded_calls():
    x, u = _logits(40, 5000, F32)
    q = Sampler(5000, 40)
    got, want = torch.zeros(40, dtype=torch.int64, device="cuda"), torch.zeros(40, dtype=torch.int64, device="cuda")
    k = torch.full((40,), 30, dtype=torch.int32, device="cuda")
    q.sample(x, u, got, top_k=k, top_p=0.9)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        q.sample(x, u, got, top_k=k, top_p=0.9)
    for i in range(4):
        x.copy_(x.roll(7, 1))
        u.copy_(u.roll(1))
        got.fill_(-7)
        graph.replay()
        torch.cuda.synchronize()
        q.sample(x, u, want, top_k=k, top_p=0.9)
        assert torch.equal(got, want), i


def test_no_rows_and_refusals():
    q = Sampler(16, 4)
    z = lambda *s, **k: torch.zeros(*s, device="cuda", **k)  # noqa: E731
    i64 = dict(dtype=torch.int64)
    q.sample(z(0, 16), z(0), z(0, **i64))
    good = dict(logits=z(4, 16), u=z(4), out=z(4, **i64))
    q.sample(**good)
    for kw in (dict(logits=z(4, 15)), dict(logits=z(4, 16).double()), dict(logits=z(16)), dict(u=z(3)), dict(u=z(4).half()), dict(out=z(4)), dict(out=z(5, **i64)),
               dict(out=z(8, **i64)[::2]), dict(temperature=-1.0), dict(temperature=math.nan), dict(temperature=math.inf), dict(temperature=z(3)),
               dict(top_k=z(4)), dict(top_k=1 << 40), dict(top_p=z(4).half()), dict(min_p=z(5)), dict(logits=z(5, 16), u=z(5), out=z(5, **i64)),
               dict(logits=None), dict(u=None), dict(out=None), dict(logits=z(4, 16).cpu()), dict(top_p=z(4).cpu())):
        with pytest.raises((ValueError, QAdamError)):
            q.sample(**{**good, **kw})
    for bad in [(0, 1), (1, -1), ((1 << 22) + 1, 1), (1, (1 << 24) + 1)]:
        with pytest.raises(QAdamError):
            Sampler(*bad)
