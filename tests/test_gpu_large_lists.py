"""Lists of tensors with more elements than one launch takes."""
import pytest
import torch

from operator_util import BF16
from paper_2004_14180_amd import AdamW, AdamWConfig, GradNorm, adamw_state

pytestmark = pytest.mark.gpu
COUNT, N = 17, 1 << 30          # 2^34 elements are one launch's


def test_norm():
    g = torch.randn(N, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1), dtype=BF16)
    want = (COUNT * float(sum(x.double().square().sum() for x in g.split(1 << 26)))) ** 0.5
    out = torch.zeros(2, device="cuda")
    GradNorm([N] * COUNT, BF16).grad_norm([g] * COUNT, 1.0, out)
    assert abs(float(out[0]) - want) <= 2.0 ** -23 * want and abs(float(out[1]) * want - 1) <= 2.0 ** -23


def test_adamw():
    """All tensors begin alike and have one gradient, so they are alike afterwards, and as a tensor of a short list is."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    first = torch.randn(N, device="cuda", generator=gen, dtype=BF16)
    g = torch.randn(N, device="cuda", generator=gen, dtype=BF16)
    cfg = AdamWConfig(state_bits=8)
    params = [first.clone() for _ in range(COUNT)]
    state = adamw_state(cfg, params)
    AdamW(cfg, params, weight_decay=0.1, grad_dtype=BF16, **state).step(1, 1e-2, [g] * COUNT)
    alone = adamw_state(cfg, [first])
    AdamW(cfg, [first], weight_decay=0.1, grad_dtype=BF16, **alone).step(1, 1e-2, [g])
    for i in range(COUNT):
        assert torch.equal(params[i], first), i
        for k in state:
            assert torch.equal(state[k][i].view(torch.uint8), alone[k][0].view(torch.uint8)), (i, k)
