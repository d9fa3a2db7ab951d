"""Weight gradients of fp16 rows from checkpoints whose rotated, or rounded, values are larger than fp16 holds."""
import pytest
import torch

from tests import groups_ref as ref
from tests.test_gpu_checkpoint import ROT, in_group_mean, normal, row_steps, saved
import paper_2508_13478_b200 as dhq

pytestmark = pytest.mark.gpu


def check(x, dy, g, rotate, out):
    """dW against 64 bits.  On the tensor cores q 2^e is an fp16 number times 2^s, s the least power (one for a group's rows, 0 at least) with which the largest
    is finite: 127 2^(e - s) <= 65,504.  So it is rounded to a multiple of 2^(s - 24), by 2^(s - 25) at most, which adds up to
    sum |dy| 2^(s - 25); a rotated result is the mean of G such sums, with signs.  The rest as in assert_sums: half a step of the result, and
    2^-23 of a partial sum for each addition."""
    (t, k), n = x.shape, dy.shape[1]
    codes, exponents = saved(x, g, rotate)
    dW = torch.full((n, k), float("nan"), dtype=ref.NAMES[out], device="cuda")
    dhq.dhq_checkpoint_weight_grad(codes, exponents, dy, dW, group=g, rotation=ROT[rotate])
    d = dy.double()
    want = d.T @ ref.restored64(codes, exponents, g, rotate, k)
    plain = ref.restored64(codes, exponents, g, False, codes.shape[1])
    walk, ends = ((d ** 2).T @ plain ** 2).sqrt(), (d.T @ plain).abs()
    if rotate:
        walk, ends = in_group_mean(walk ** 2, g).div(g).sqrt(), in_group_mean(ends, g)
    assert not (exponents == 255).any()
    s = (exponents.amax(0).int() - 136).clamp(min=0).repeat_interleave(g)[:k].double()
    tol = (ref.half_step(dW.dtype) * want.abs() * 1.01 + torch.finfo(dW.dtype).smallest_normal * ref.half_step(dW.dtype)
           + (row_steps(t, 1) + (g if rotate else 0)) * 2.0 ** -23 * (6 * walk + ends)[:, :k] + d.abs().sum(0)[:, None] * 2.0 ** (s - 25) * 1.01)
    err = (dW.double() - want).abs()
    assert dW.isfinite().all() and (err <= tol).all(), f"{(err / tol).max().item():.2f} times the tolerance"
    return dW


@pytest.mark.parametrize("out", ["fp16", "fp32"])
@pytest.mark.parametrize("rotate", [False, True])
@pytest.mark.parametrize("g", [32, 64, 128])
@pytest.mark.parametrize("value", [520.0, 600.0, 2000.0, 60000.0, 65504.0])
def test_groups_of_one_value(value, g, rotate, out):
    for t, n, k in ((1, 8, 128), (100, 130, 257), (5000, 64, 300)):
        x = torch.full((t, k), value, dtype=torch.float16, device="cuda")
        x[::3] *= -1
        check(x, normal(t, n, seed=n, scale=2.0 ** -10).half(), g, rotate, out)


@pytest.mark.parametrize("t,n,k", [(777, 300, 520), (20000, 64, 64), (3000, 1000, 136)])
@pytest.mark.parametrize("rotate", [False, True])
@pytest.mark.parametrize("g", [32, 128])
def test_rows_of_every_magnitude_together(t, n, k, rotate, g):
    # groups whose rows are all ordinary stand beside groups with a few very large rows
    x = normal(t, k, seed=3)
    x *= 2.0 ** torch.randint(-18, 6, (t, 1), generator=torch.Generator().manual_seed(5)).cuda()
    x[:: 50, k // 2:] = 50000.0
    check(x.half(), normal(t, n, seed=1, scale=2.0 ** -8).half(), g, rotate, "fp32")


@pytest.mark.parametrize("size", [1e6, 1e20, 1e30])
@pytest.mark.parametrize("rotate", [False, True])
def test_checkpoints_of_fp32_values_that_fp16_does_not_have(size, rotate):
    check(normal(500, 200, seed=2, scale=size), normal(500, 70, seed=1).half(), 64, rotate, "fp32")


@pytest.mark.parametrize("rotate", [False, True])
def test_broken_groups_beside_large_ones(rotate):
    x = torch.full((300, 256), 3000.0, dtype=torch.float16, device="cuda")
    x[7, 70] = float("nan")
    codes, exponents = saved(x, 64, rotate)
    dW = torch.empty(40, 256, device="cuda")
    dhq.dhq_checkpoint_weight_grad(codes, exponents, normal(300, 40, seed=1).half(), dW, group=64, rotation=ROT[rotate])
    assert dW[:, 64:128].isnan().all() and dW[:, :64].isfinite().all() and dW[:, 128:].isfinite().all()


@pytest.mark.parametrize("out", ["fp16", "fp32"])
@pytest.mark.parametrize("t,n,k,g", [(65536, 256, 256, 64), (20011, 264, 384, 32), (4096, 1024, 1024, 128), (40, 136, 264, 32)])
def test_large_whole_numbers_are_exact_in_calls_behind_one_another(out, t, n, k, g):
    """Powers 2^13 and 2^14 (2^0 and 2^1 in every third group): a power of two times whole numbers whose sums stay below 2^24, so nothing is
    rounded but the result.  Blocks with and without large groups run side by side, and every call has other codes."""
    many = 6
    gen = torch.Generator(device="cuda").manual_seed(t)
    codes = torch.randint(-127, 128, (many, t, k), generator=gen, device="cuda", dtype=torch.int8)
    padded = dhq.padded_columns(k, g)
    codes = torch.nn.functional.pad(codes, (0, padded - k))
    low = torch.where(torch.arange(padded // g, device="cuda") % 3 == 0, 127, 140)
    exponents = (low + torch.randint(0, 2, (many, t, padded // g), generator=gen, device="cuda")).to(torch.uint8)
    dy = torch.randint(-3, 4, (t, n), generator=gen, device="cuda").half()
    dy *= 2.0 ** -12 if out == "fp16" else 1.0   # (sums of a thousand or so, times 2^14, are within fp16 then)
    want = torch.empty(many, n, k, device="cuda", dtype=torch.float64)
    for i in range(many):
        z = codes[i].double() * (2.0 ** (exponents[i].cpu().double() - 127)).round().cuda().repeat_interleave(g, 1)
        want[i] = (dy.double().T @ z)[:, :k]
    want = want.float().to(ref.NAMES[out])
    dW = torch.zeros_like(want)

    def calls():
        for i in range(many):
            dhq.dhq_checkpoint_weight_grad(codes[i], exponents[i], dy, dW[i], group=g)

    for _ in range(3):
        calls()
    assert torch.equal(dW, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for _ in range(3):
        dW.zero_()
        graph.replay()
        assert torch.equal(dW, want)
