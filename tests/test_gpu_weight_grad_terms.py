"""fp32 rows of the weight gradient keep all of their 24 bits, at every place of the sums."""
import pytest
import torch

import paper_2508_13478_b200 as dhq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t,n,k,g", [(64, 64, 128, 32), (1000, 136, 200, 64), (5000, 1000, 264, 128), (65536, 300, 256, 64), (9000, 2600, 2500, 32)])
def test_one_row_for_each_output_is_exact(t, n, k, g):
    """Each output has one row with a gradient that is not zero: an odd whole number of 24 bits times a power of two, so that its three terms of 8 bits
    are all needed.  Codes are powers of two.  Then every product and every sum is a number of at most 24 bits: nothing is rounded
    anywhere, and the result is dy x^ itself.  The rows lie all over the sum: every stage of the rings, before and after sums are drained, in every part."""
    gen = torch.Generator(device="cuda").manual_seed(t)

    def whole(low, high, *shape):
        return torch.randint(low, high, shape, generator=gen, device="cuda")

    padded = dhq.padded_columns(k, g)
    codes = ((1 << whole(0, 7, t, padded)) * (1 - 2 * whole(0, 2, t, padded))).to(torch.int8)
    exponents = whole(120, 135, t, padded // g).to(torch.uint8)
    rows = torch.arange(n, device="cuda") * (t - 1) // max(1, n - 1)
    value = (whole(1 << 23, 1 << 24, n) | 1).double() * (1 - 2 * whole(0, 2, n)) * 2.0 ** -30
    dy = torch.zeros(t, n, device="cuda")
    dy[rows, torch.arange(n, device="cuda")] = value.float()
    dW = torch.full((n, k), float("nan"), device="cuda")
    dhq.dhq_checkpoint_weight_grad(codes, exponents, dy, dW, group=g)
    power = ((exponents[rows].long() - 127 + 1023) << 52).view(torch.float64)
    want = value[:, None] * (codes[rows].double() * power.repeat_interleave(g, 1))[:, :k]
    assert torch.equal(want, want.float().double()) and torch.equal(dW.double(), want)
