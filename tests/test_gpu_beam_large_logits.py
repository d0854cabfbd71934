"""dasc_beam_select where logits are finite numbers of any size: tokens that are forced, and masks that are no infinities.

A score is off by what bh.same allows: with the largest logit m taken off first, the largest entry's exponential is 1 whatever m is.  In 64 bits m + log(sum) rounds to
a step of m's size, here and in the oracle alike: sums of exponentials are whole numbers in these tests where that step is more than the tolerance."""
import pytest
import torch

import beam_helpers as bh

pytestmark = pytest.mark.gpu
TYPES = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
SIZES = (1e10, 1e12, 1e13, 1e20, 1e30, 2.5e38)


def inputs(seed, R, W, V, dtype):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(R, W, V, generator=gen, device="cuda") * 2.5).to(dtype), torch.randn(R, W, generator=gen, device="cuda") - 10


def held(x, s, n):
    got = bh.call(x, s, n)
    bh.same(got, bh.define(x, s, None, -1, n), x)
    return got


@TYPES
@pytest.mark.parametrize("V, n", [(40, 4), (1000, 8), (70001, 8), (131072, 16)])
def test_forced_tokens(dtype, V, n):
    """One logit far above all others, in the first, a middle and the last place, in one beam, two, or all of them."""
    sizes = (*SIZES, torch.finfo(dtype).max)
    x, s = inputs(1, len(sizes), 4, V, dtype)
    for r, size in enumerate(sizes):
        x[r, 1, (0, V // 2, V - 1)[r % 3]] = size
        if r % 2:
            x[r, 2, V // 3] = size
    x[0, 0, V - 1] = x[0, 2, 5] = x[0, 3, 11] = sizes[0]
    got = held(x, s, n)
    assert bool(torch.isfinite(got[0]).all())


@TYPES
@pytest.mark.parametrize("V", [40, 1000, 70001])
def test_rows_of_one_large_value(dtype, V):
    """Short rows and long ones, low and high, two such beams beside normal ones or in all."""
    values = [*(-v for v in SIZES), *SIZES, torch.finfo(dtype).min, torch.finfo(dtype).max]
    x, s = inputs(2, 2 * len(values), 4, V, dtype)
    for r, value in enumerate(values):
        x[2 * r, 1] = x[2 * r, 3] = value
        x[2 * r + 1] = value
    for n in (4, 16):
        got = held(x, s, n)
        assert bool(torch.isfinite(got[0]).all())


@TYPES
@pytest.mark.parametrize("V", [300, 40000, 131072])
@pytest.mark.parametrize("low", [-1e10, -1e30, "lowest"])
def test_rows_masked_with_a_finite_value(dtype, V, low):
    """Nine tenths of the tokens, here and there, in front, behind; all but a few; all but one of a part of the beams."""
    x, s = inputs(3, 5, 3, V, dtype)
    low = torch.finfo(dtype).min if low == "lowest" else low
    x[0, :, torch.rand(V, generator=torch.Generator().manual_seed(4)).cuda() < 0.9] = low
    x[1, :, : V * 9 // 10] = low
    x[2, :, V // 10:] = low
    x[3, :, 7:] = low
    x[4, 1, : V - 1] = low
    for n in (3, 40):
        held(x, s, n)


@pytest.mark.parametrize("V", [50, 5000, 100003])
def test_logits_around_a_large_number(V):
    """All logits shifted alike: the steps of fp32 between them grow to 2 at 2^24 and 64 at 2^29."""
    x, s = inputs(5, 10, 2, V, torch.float32)
    for r, shift in enumerate((2.0 ** 10, 2.0 ** 20, 2.0 ** 24, 2.0 ** 25, 2.0 ** 29)):
        x[2 * r] = x[2 * r] * max(1.0, shift * 2.0 ** -22) + shift
        x[2 * r + 1] = x[2 * r + 1] * max(1.0, shift * 2.0 ** -22) - shift
    held(x, s, 6)


@TYPES
def test_rows_whose_parts_are_of_different_sizes(dtype):
    """A row's largest logits in one place, everything else lower by orders of magnitude; values over the whole range of the type."""
    V = 60000
    x, s = inputs(6, 4, 3, V, dtype)
    x[0, :, :20000] *= 1e9
    x[1, :, 20000:] -= 1e20
    x[2] *= 1e37
    x[3] = torch.where(torch.arange(V, device="cuda") % 977 == 3, x[3].float() - 1e12, torch.tensor(-float("inf"), device="cuda")).to(dtype)
    held(x, s, 8)
