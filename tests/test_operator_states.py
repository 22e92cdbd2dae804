"""How far a second moment in 8 bits goes from its 32-bit value, by the stored format's formulas: the figures that the header states."""
import pytest
import torch

from operator_util import fp8_blocks


@pytest.mark.parametrize("factor,first,second", [(1.0, (0.75, 1.3), (0.75, 1.3)), (0.1, (5.0, 12.0), (0.75, 1.3)), (4.0, (0.75, 1.5), (2.5, 6.0))])
def test_the_root_of_a_second_moment_beside_that_in_64_bits(factor, first, second):
    """A block of normal gradients of different scales; from step 500 on those of its first half are `factor` times as large.  Averages of
    8-bit sqrt(v) over the exact one in both halves after 8000 steps."""
    gen = torch.Generator().manual_seed(1)
    scale = torch.exp(torch.randn(256, generator=gen) * 0.7)
    held, v, beta2 = torch.zeros(256), torch.zeros(256, dtype=torch.float64), 0.999
    for step in range(8000):
        if step == 500:
            scale[:128] *= factor
        g = torch.randn(256, generator=gen) * scale
        v = v * beta2 + g.double().square() * (1 - beta2)
        q, unit = fp8_blocks((held.square() * beta2 + g * g * (1 - beta2)).sqrt(), True)
        held = q.float() * unit
    ratio = held / v.sqrt().float()
    for part, (low, high) in ((ratio[:128], first), (ratio[128:], second)):
        assert low <= float(part.mean()) <= high
