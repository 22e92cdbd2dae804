"""Embedding lookup and its gradient against plain forms in 64 bits, at the sizes, layouts and tokens where they can go wrong."""
import pytest
import torch

from operator_util import BF16, F16, F32, LEAST, U32, close, embedding_grad64, rounded
from paper_2004_14180_amd import Embedding, QAdam, QAdamConfig, QAdamError

pytestmark = pytest.mark.gpu
STATUS = 4


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _tokens(kind, n, rows, gen, dtype=torch.int64):
    if kind == "uniform":
        t = torch.randint(0, rows, (n,), generator=gen)
    elif kind == "zipf":
        t = (torch.exp(torch.rand(n, generator=gen, dtype=torch.float64) * torch.log(torch.tensor(rows + 1.0))) - 1).long().clamp(0, rows - 1)
    elif kind == "same":
        t = torch.full((n,), rows // 2)
    elif kind == "runs":
        t = (torch.arange(n) // 97 * 31) % rows
    elif kind == "last":
        t = torch.where(torch.rand(n, generator=gen) < 0.5, rows - 1, 0)
    else:                                                           # some are outside
        t = torch.randint(-3, rows + 3, (n,), generator=gen)
    return t.to(dtype)


def _matrix(rows, dim, dtype, gap, gen, offset=0):
    """A matrix on the device whose rows lie `gap` elements apart, `offset` elements into its allocation; and all of it."""
    whole = torch.full((offset + rows * (dim + gap) + 16,), 5.0).to(dtype).cuda()
    m = whole[offset:offset + rows * (dim + gap)].view(rows, dim + gap)[:, :dim]
    m.copy_(torch.randn(rows, dim, generator=gen).to(dtype))
    return m, whole


@pytest.mark.parametrize("table", ["f32", "bf16", "f16", "codes8", "codes16"])
@pytest.mark.parametrize("out_type", [F32, BF16, F16])
@pytest.mark.parametrize("rows,dim,n,gap,offset", [(7, 1, 1, 0, 0), (50, 8, 5, 0, 0), (301, 257, 130, 3, 1), (1000, 768, 64, 0, 1),
                                                   (129, 1000, 33, 8, 3), (64, 2048, 200, 0, 0), (5, 5000, 9, 1, 1)])
def test_lookup(table, out_type, rows, dim, n, gap, offset):
    gen = _gen(rows)
    k_x, dtype = {"f32": (None, F32), "bf16": (None, BF16), "f16": (None, F16), "codes8": (5, torch.int8), "codes16": (13, torch.int16)}[table]
    scale = 1.7
    if k_x is None:
        w, _ = _matrix(rows, dim, dtype, gap, gen, offset)
        w64 = w.double().cpu()
    else:
        whole = torch.randint(-2 ** k_x, 2 ** k_x + 1, (offset + rows * (dim + gap),), generator=gen).to(dtype).cuda()
        w = whole[offset:].view(rows, dim + gap)[:, :dim]
        w64 = w.double().cpu() * 2.0 ** -(k_x + 1)
    emb = Embedding(rows, dim, 0)
    for ids, kind, padding in [(torch.int64, "zipf", None), (torch.int32, "outside", rows // 2)]:
        tok = _tokens(kind, n, rows, gen, ids)
        out, whole = _matrix(n, dim, out_type, gap, gen, offset)
        beside = whole.clone()
        emb.lookup(w, tok.cuda(), out, scale=scale, k_x=k_x, padding_idx=padding)
        keep = (tok >= 0) & (tok < rows) & (tok != (-1 if padding is None else padding))
        want = torch.where(keep[:, None], w64[tok.long().clamp(0, rows - 1)] * scale, torch.zeros(1, dtype=torch.float64))
        close(out, want, rounded(2 * U32 * want.abs() + LEAST[F32], want, out_type))
        assert emb.get_status(clear=True) == (STATUS if ((tok < 0) | (tok >= rows)).any() else 0)
        out.copy_(beside[offset:offset + n * (dim + gap)].view(n, dim + gap)[:, :dim])
        assert torch.equal(whole, beside), "wrote beside its rows"


def test_lookup_of_nothing_and_of_many():
    emb = Embedding(10, 4, 0)
    w = torch.randn(10, 4, device="cuda")
    emb.lookup(w, torch.zeros(0, dtype=torch.int64, device="cuda"), torch.zeros(0, 4, device="cuda"))
    tok = torch.randint(0, 10, (3, 50_000, 2), device="cuda")
    out = torch.zeros(3, 50_000, 2, 4, device="cuda")
    emb.lookup(w, tok, out)
    assert torch.equal(out, w[tok])


def test_lookup_of_the_codes_that_the_step_emits():
    """The layer's part of wcodes, looked up without the vector of weights in between: the decoder's bits, times the scale."""
    rows, dim = 211, 97
    sizes = [33, rows * dim, 1000]
    off = [0, 33, 33 + rows * dim, 33 + rows * dim + 1000]
    for k_x in (6, 14):
        q = QAdam(QAdamConfig(k_x=k_x), off, 1)
        x = torch.randn(sum(sizes), generator=_gen(1)).cuda() * 0.2
        wcodes = torch.zeros(sum(sizes), dtype=torch.int8 if k_x <= 6 else torch.int16, device="cuda")
        werr, xhat = torch.zeros_like(x), torch.zeros_like(x)
        q.weight_quantize(1, x, werr, wcodes)
        q.weight_dequantize(wcodes, xhat)
        tok = torch.randint(0, rows, (500,), generator=_gen(2)).cuda()
        out = torch.zeros(500, dim, device="cuda")
        Embedding(rows, dim, 0).lookup(wcodes[33:33 + rows * dim].view(rows, dim), tok, out, k_x=k_x, scale=8.0)
        assert torch.equal(out, xhat[33:33 + rows * dim].view(rows, dim)[tok] * 8.0)


GRAD_SHAPES = [(7, 1, 1, 0, 0), (50, 8, 3, 0, 0), (301, 257, 130, 3, 1), (1000, 768, 1024, 0, 1), (129, 1000, 333, 8, 3),
               (2000, 64, 5000, 0, 0), (70_000, 40, 9000, 0, 0), (600, 130, 20_011, 2, 1), (64, 2048, 2500, 0, 0), (3, 5000, 700, 1, 1),
               (200_000, 9, 3000, 0, 1), (300_007, 12, 5001, 0, 0), (530_001, 7, 2500, 0, 0), (900, 20, 140_001, 1, 0), (11, 129, 2049, 0, 0), (5, 1025, 2000, 0, 0), (40, 70, 2048, 0, 0), (255, 65, 2100, 2, 1)]


@pytest.mark.parametrize("rows,dim,n,gap,offset", GRAD_SHAPES)
@pytest.mark.parametrize("kind", ["uniform", "zipf", "same", "runs", "last", "outside"])
@pytest.mark.parametrize("accumulate", [False, True])
def test_grad(rows, dim, n, gap, offset, kind, accumulate):
    gen = _gen(n)
    types = [F32, BF16, F16]
    k = (n + len(kind) + accumulate) % 9
    dtype, gtype = types[k % 3], types[k // 3]
    ids = torch.int32 if k % 2 else torch.int64
    tok = _tokens(kind, n, rows, gen, ids)
    padding = rows // 2 if kind in ("zipf", "outside") else None
    dout, _ = _matrix(n, dim, dtype, gap, gen, offset)
    grad, whole = _matrix(rows, dim, gtype, gap, gen, offset)
    before, beside = grad.double().cpu(), whole.clone()
    emb = Embedding(rows, dim, n)
    scale = 0.7
    emb.grad(tok.cuda(), dout, grad, scale=scale, padding_idx=padding, accumulate=accumulate)
    want, bound = embedding_grad64(tok, dout, rows, scale, padding)
    if accumulate:
        want, touched = want + before, bound > 4 * LEAST[F32]
        bound = bound + U32 * want.abs()
        untouched = torch.bincount(tok.long()[(tok >= 0) & (tok < rows) & (tok != (-1 if padding is None else padding))], minlength=rows) == 0
        assert torch.equal(grad.cpu()[untouched].double(), before[untouched])
    close(grad, want, rounded(bound, want, gtype))
    assert emb.get_status() == (STATUS if kind == "outside" and ((tok < 0) | (tok >= rows)).any() else 0)
    first = grad.clone()
    grad.copy_(before.to(gtype))
    emb.grad(tok.cuda(), dout, grad, scale=scale, padding_idx=padding, accumulate=accumulate)
    assert torch.equal(grad, first), "not the same bits on every run"
    grad.copy_(before.to(gtype))
    assert torch.equal(whole, beside), "wrote beside its rows"


def test_grad_of_nothing():
    emb = Embedding(20, 5, 8)
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    g = torch.ones(20, 5, device="cuda")
    emb.grad(none, torch.zeros(0, 5, device="cuda"), g, accumulate=True)
    assert (g == 1).all()
    emb.grad(none, torch.zeros(0, 5, device="cuda"), g)
    assert (g == 0).all()
    for tok in (torch.full((8,), 3), torch.full((8,), -1), torch.full((8,), 1 << 40)):        # all padding, all outside
        g.fill_(1)
        emb.grad(tok.cuda(), torch.ones(8, 5, device="cuda"), g, padding_idx=3)
        assert (g == 0).all()


def test_grad_of_an_expanded_row():
    """Loss = sum of the lookup: one row of ones for every token."""
    tok = _tokens("zipf", 3000, 100, _gen(1))
    g = torch.zeros(100, 24, device="cuda")
    Embedding(100, 24, 3000).grad(tok.view(3, 1000).cuda(), torch.ones(1, 1, 24, device="cuda").expand(3, 1000, 24), g)
    want = torch.bincount(tok, minlength=100).float()
    assert torch.equal(g.cpu(), want[:, None].expand(100, 24))


def test_infinities_and_nans_stay_in_their_rows_and_padding_does_not_spread_them():
    tok = torch.tensor([1, 2, 3, 2, 4] * 300)
    d = torch.ones(1500, 12)
    d[tok == 3] = float("nan")
    d[1] = float("inf")
    for n in (5, 1500):
        g = torch.zeros(6, 12, device="cuda")
        Embedding(6, 12, n).grad(tok[:n].cuda(), d[:n].cuda(), g, padding_idx=3)
        assert (g[3] == 0).all() and (g[2] == float("inf")).all() and (g[1] == n / 5).all() and (g[4] == n / 5).all()


def test_gradient_against_differences():
    """The lookup is linear: central differences of sum(out * dout) in its weights are the gradient but for rounding."""
    rows, dim, n, scale, h = 9, 6, 40, 1.5, 0.25
    gen = _gen(8)
    tok = _tokens("outside", n, rows, gen).cuda()
    w, dout = torch.randn(rows, dim, generator=gen).cuda(), torch.randn(n, dim, generator=gen).cuda()
    emb, out, g = Embedding(rows, dim, n), torch.zeros(n, dim, device="cuda"), torch.zeros(rows, dim, device="cuda")
    emb.grad(tok, dout, g, scale=scale, padding_idx=4)

    def loss(x):
        emb.lookup(x, tok, out, scale=scale, padding_idx=4)
        return float((out.double() * dout.double()).sum())

    for r in range(rows):
        for k in range(dim):
            up, down = w.clone(), w.clone()
            up[r, k] += h
            down[r, k] -= h
            # each of the n values of the lookup that enter is rounded twice, at about |w| + h
            bound = 2 * n * 2 * U32 * scale * 4.0 * float(dout.abs().max()) / (2 * h) + n * U32 * 10
            assert abs((loss(up) - loss(down)) / (2 * h) - float(g[r, k])) <= bound


def test_into_a_slice_of_the_flat_gradient_beyond_32_bits():
    """A matrix of more than 2^31 elements, in the flat gradient behind another layer."""
    rows, dim = 1_050_000, 2051
    flat = torch.zeros(7 + rows * dim, dtype=BF16, device="cuda")
    g = flat[7:].view(rows, dim)
    tok = torch.tensor([0, rows - 1, rows // 2, rows - 1], device="cuda")
    d = torch.randn(4, dim, generator=_gen(3)).cuda()
    emb = Embedding(rows, dim, 4)
    emb.grad(tok, d, g, accumulate=True)
    assert torch.equal(g[0], d[0].to(BF16)) and torch.equal(g[rows - 1], (d[1] + d[3]).to(BF16)) and torch.equal(g[rows // 2], d[2].to(BF16))
    assert (flat[:7] == 0).all() and int((flat != 0).sum()) <= 3 * dim
    out = torch.zeros(4, dim, dtype=BF16, device="cuda")
    emb.lookup(g, tok, out)
    assert torch.equal(out, g[tok])
    g[rows - 2].fill_(1)
    emb.grad(tok, d, g)
    assert (g[rows - 2] == 0).all() and torch.equal(g[rows - 1], (d[1] + d[3]).to(BF16))


def test_recorded_calls():
    rows, dim, n = 3000, 100, 5000
    gen = _gen(4)
    tok, d = _tokens("zipf", n, rows, gen).cuda(), torch.randn(n, dim, generator=gen).cuda()
    w, out, g = torch.randn(rows, dim, device="cuda"), torch.zeros(n, dim, device="cuda"), torch.zeros(rows, dim, device="cuda")
    emb = Embedding(rows, dim, n)
    emb.grad(tok, d, g)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        emb.lookup(w, tok, out)
        emb.grad(tok, d, g)
    for k in range(4):
        tok.copy_(tok.roll(17) if k % 2 else (tok + 1) % rows)
        w.add_(1.0)
        g.fill_(9.0)
        graph.replay()
        torch.cuda.synchronize()
        got = g.clone()
        emb.grad(tok, d, g)
        assert torch.equal(out, w[tok]) and torch.equal(got, g), k


def test_refusals():
    for bad in [(0, 4, 4), (4, 0, 4), (4, 4, -1), ((1 << 28) + 1, 4, 4), (4, (1 << 20) + 1, 4)]:
        with pytest.raises(QAdamError):
            Embedding(*bad)
    emb = Embedding(10, 4, 6)
    z = lambda *s, dtype=F32: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
    w, tok, out = z(10, 4), z(6, dtype=torch.int64), z(6, 4)
    for kw in [dict(weight=z(9, 4)), dict(weight=z(10, 4).cpu()), dict(weight=z(4, 10).t()), dict(weight=z(10, 4, dtype=torch.float64)),
               dict(weight=z(10, 4, dtype=torch.int8)), dict(k_x=6), dict(tokens=z(6)), dict(tokens=z(12, dtype=torch.int64)[::2]),
               dict(out=z(5, 4)), dict(out=z(6, 4, dtype=torch.int32)), dict(tokens=tok.cpu()), dict(out=z(6, 8)[:, ::2])]:
        with pytest.raises(ValueError):
            emb.lookup(**{**dict(weight=w, tokens=tok, out=out), **kw})
    for k_x, dtype in [(7, torch.int8), (6, torch.int16), (15, torch.int16), (-1, torch.int8)]:
        with pytest.raises(QAdamError) as e:
            emb.lookup(z(10, 4, dtype=dtype), tok, out, k_x=k_x)
        assert e.value.code == -1
    with pytest.raises(QAdamError) as e:                            # rows of the output on top of each other
        emb.lookup(w, tok, z(1, 4).expand(6, 4))
    assert e.value.code == -1
    with pytest.raises(QAdamError) as e:
        emb.grad(z(7, dtype=torch.int64), z(7, 4), w)
    assert e.value.code == -3
    for kw in [dict(dout=z(5, 4)), dict(grad=z(10, 5)), dict(dout=z(6, 4, dtype=torch.float64)), dict(grad=z(10, 4, dtype=torch.int32)),
               dict(dout=z(6, 8)[:, ::2])]:
        with pytest.raises(ValueError):
            emb.grad(**{**dict(tokens=tok, dout=out, grad=w), **kw})
    with pytest.raises(QAdamError) as e:
        emb.grad(tok, out, z(1, 4).expand(10, 4))
    assert e.value.code == -1
