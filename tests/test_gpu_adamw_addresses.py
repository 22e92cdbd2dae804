"""AdamW with moments, scales, weights, copies and gradients that each begin at another address: the same bits as from allocations of
their own."""
import pytest
import torch

from operator_util import BF16, F16, F32
from paper_2004_14180_amd import AdamW, AdamWConfig, adamw_state

pytestmark = pytest.mark.gpu
SIZES = [1, 2, 255, 256, 257, 1023, 4096, 5001, 70_003]


def _at(t, offset):
    """A copy of t that begins `offset` elements into its allocation, and the elements beside it."""
    whole = torch.zeros(t.numel() + offset + 70, dtype=t.dtype, device="cuda")
    whole.view(torch.uint8).fill_(0x35)
    out = whole[offset:offset + t.numel()]
    out.copy_(t)
    return out, (whole[:offset].view(torch.uint8), whole[offset + t.numel():].view(torch.uint8))


@pytest.mark.parametrize("bits,ptype,gtype,ctype", [(8, F32, BF16, BF16), (8, BF16, F16, None), (32, F32, F32, F16), (32, F16, BF16, None)])
@pytest.mark.parametrize("first", [1, 2, 3, 5, 31, 64])
def test_every_buffer_at_an_address_of_its_own(bits, ptype, gtype, ctype, first):
    gen = torch.Generator(device="cuda").manual_seed(first)
    cfg = AdamWConfig(state_bits=bits)
    rand = lambda n, dtype: torch.randn(n, generator=gen, device="cuda").to(dtype)  # noqa: E731
    params, grads = [rand(n, ptype) for n in SIZES], [[rand(n, gtype) for n in SIZES] for _ in range(2)]
    state = adamw_state(cfg, params)
    copies = [torch.zeros(n, dtype=ctype, device="cuda") for n in SIZES] if ctype is not None else None
    beside, offset = [], first

    def moved(ts):
        nonlocal offset
        out = []
        for t in ts:
            a, b = _at(t, offset)
            offset = offset * 7 % 67 or 1
            out.append(a)
            beside.extend(b)
        return out

    params2, state2, copies2 = moved(params), {k: moved(ts) for k, ts in state.items()}, None if copies is None else moved(copies)
    grads2 = [moved(g) for g in grads]
    a = AdamW(cfg, params, copies=copies, weight_decay=0.1, grad_dtype=gtype, **state)
    b = AdamW(cfg, params2, copies=copies2, weight_decay=0.1, grad_dtype=gtype, **state2)
    for step in (1, 2):
        a.step(step, 1e-2, grads[step - 1])
        b.step(step, 1e-2, grads2[step - 1])
    lists = [(params, params2)] + [(state[k], state2[k]) for k in state] + ([(copies, copies2)] if copies else [])
    for x, y in lists:
        for i in range(len(SIZES)):
            assert torch.equal(x[i].view(torch.uint8), y[i].view(torch.uint8)), SIZES[i]
    assert all((x == 0x35).all() for x in beside), "wrote beside its buffers"
