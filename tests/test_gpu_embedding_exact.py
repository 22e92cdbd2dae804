"""The embedding's gradient where every sum is exact: rows of small integers that differ from token to token, so that a token that is
lost, repeated or added to another row shows whatever the length of its run."""
import pytest
import torch

from paper_2004_14180_amd import Embedding
from test_gpu_embedding import GRAD_SHAPES, _gen, _tokens

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def _integers(n, dim, gap, offset, seed, dtype):
    """n rows of dim integers in -8..8, none of them zero, on the device, `gap` elements apart."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randint(1, 9, (offset + n * (dim + gap),), generator=gen, device="cuda")
    x = x * (torch.randint(0, 2, x.shape, generator=gen, device="cuda") * 2 - 1)
    return x.to(dtype)[offset:].view(n, dim + gap)[:, :dim]


def _sums(tok, dout, rows, padding):
    """int64 sums of the rows' tokens; their magnitudes stay below 2^24 in any order."""
    tok = tok.reshape(-1).cuda().long()
    assert tok.numel() * 8 < 1 << 24
    keep = (tok >= 0) & (tok < rows) & (tok != (-1 if padding is None else padding))
    return torch.zeros(rows, dout.shape[1], dtype=torch.int64, device="cuda").index_add_(0, tok[keep], dout[keep].long())


def _check(emb, tok, dout, rows, dim, padding, accumulate, gap=0, offset=0):
    grad = _integers(rows, dim, gap, offset, rows, F32)
    want = _sums(tok, dout, rows, padding) + (2 * grad.long() if accumulate else 0)
    emb.grad(tok.cuda(), dout, grad, scale=0.5, padding_idx=padding, accumulate=accumulate)
    assert torch.equal((grad * 2).long(), want) and torch.equal((grad * 2).long().float(), grad * 2)


# ... and lists that are not sorted, of more than one workgroup of column slices per token: several slices past the last one, pieces of
# frequent rows joined in each
DIRECT = [(64, 2048, 1024, 0, 0), (5, 2049, 600, 0, 1), (9, 4096, 500, 2, 0), (4, 1300, 1000, 0, 3), (700, 1025, 1024, 0, 0), (6, 8000, 250, 1, 0)]


@pytest.mark.parametrize("rows,dim,n,gap,offset", GRAD_SHAPES + DIRECT)
@pytest.mark.parametrize("kind", ["uniform", "zipf", "same", "runs", "last", "outside"])
def test_every_token_is_added_once(rows, dim, n, gap, offset, kind):
    tok = _tokens(kind, n, rows, _gen(n), torch.int32 if (n + len(kind)) % 2 else torch.int64)
    padding = rows // 2 if kind in ("zipf", "outside") else None
    dout = _integers(n, dim, gap, offset, n, [F32, BF16, F16][(n + dim) % 3])
    emb = Embedding(rows, dim, n)
    for accumulate in (False, True):
        _check(emb, tok, dout, rows, dim, padding, accumulate, gap, offset)


@pytest.mark.parametrize("rows,dim", [(900, 20), (600_000, 9), (30, 1040)])
def test_one_handle_for_lists_of_every_length(rows, dim):
    """Short, grouped and digit-sorted lists share their handle's scratch."""
    most = 140_001 if dim < 1000 else 9000
    emb = Embedding(rows, dim, most)
    dout = _integers(most, dim, 0, 0, 1, BF16)
    lengths = [5, most, 1500, 2049, 1, most - 1, 2048, 9000, 0, 700, 131_072, 64, 131_073, 2048, 4097, 1024]
    for k, n in enumerate(n for n in lengths if n <= most):
        for kind in ("same", "zipf") if k % 2 else ("last", "same"):
            _check(emb, _tokens(kind, n, rows, _gen(k)), dout[:n], rows, dim, None, bool(k & 2))


@pytest.mark.parametrize("n", [(1 << 20) + 77, 1_900_003])
@pytest.mark.parametrize("kind", ["same", "last", "runs"])
def test_long_runs(n, kind):
    """Runs of up to 47 500 pieces."""
    rows, dim = 211, 6
    tok = torch.arange(n) // 9973 % rows if kind == "runs" else _tokens(kind, n, rows, _gen(n))
    _check(Embedding(rows, dim, n), tok, _integers(n, dim, 0, 0, n, F16), rows, dim, None, kind == "last")


@pytest.mark.parametrize("rows", [1 << 28, (1 << 27) + 3])
def test_as_many_rows_as_a_handle_takes(rows):
    """Written whole: more rows than wavefronts of a launch."""
    n = 4099
    tok = torch.randint(0, rows, (n,), generator=_gen(1))
    tok[:3] = torch.tensor([0, rows - 1, rows - 1])
    dout = _integers(n, 1, 0, 0, 5, F32)
    grad = torch.ones(rows, 1, dtype=BF16, device="cuda")
    Embedding(rows, 1, n).grad(tok.cuda(), dout, grad)
    got = grad.view(-1).nonzero()[:, 0]
    row, place = tok.unique(return_inverse=True)
    want = torch.zeros(len(row), dtype=torch.int64).index_add_(0, place, dout.cpu().long()[:, 0])
    assert torch.equal(got.cpu(), row[want != 0]) and torch.equal(grad.view(-1)[got].long().cpu(), want[want != 0])


@pytest.mark.parametrize("n", [3000, 131_072, (1 << 20) + 3])
@pytest.mark.parametrize("value", [0.51, 1.1])
@pytest.mark.parametrize("accumulate", [False, True])
def test_equal_rows_add_up(n, value, accumulate):
    """One row for every token, all of them of one row: roundings of equal sums, which all go the same way, must not add up.  A piece of
    up to 64 tokens has 63 roundings; the joined sum, the scale, the product and the addition have one each."""
    dout = torch.full((1, 5), value, device="cuda")
    grad = torch.full((3, 5), 2.0, device="cuda")
    Embedding(3, 5, n).grad(torch.ones(n, dtype=torch.int32, device="cuda"), dout.expand(n, 5), grad, scale=0.3, accumulate=accumulate)
    want = n * float(dout[0, 0]) * 0.3 + (2.0 if accumulate else 0.0)
    assert ((grad[1].double() - want).abs() <= 67 * 2.0 ** -24 * want).all()
    assert (grad[[0, 2]] == (2.0 if accumulate else 0.0)).all()
