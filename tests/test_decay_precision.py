"""How far decayed linear attention in chunks is from exact numbers, at bounds that a value with one bf16 part too few does not keep.

A value in n parts of bf16 (rounded to 8 bits, the rest rounded, ...) is off by at most 2^-8n of itself: sums of many terms hide that behind the
roundings of their additions.  So here every state and every output is ONE product, and the bounds are those of
a handful of fp32 operations:
  states   weight e^G from a sum of logarithms below 8 (2^-22) by ex2 (2^-22), times the key (2^-24), in three parts (2^-24), added up from three
           products (3 * 2^-23), carried over a chunk by a factor (2^-22) and a rounding (2^-24): below 2^-19.  In two parts: 2^-17 of a key's power of two.
  outputs  the same weight or state in two parts: 2^-16 covers 2^-17 and the rest.  In one part: 2^-9 of its power of two; bf16 outputs are off by half a step of their own besides.
"""
import pytest
import torch

import paper_2608_30386_b200 as dasc
from decay_helpers import expected, make_case, run

CHUNKED = dasc.ALGO_CHUNKED
STATE, OUTPUT = 2.0 ** -19, 2.0 ** -16


def half_step(x):
    """Half a step of bf16 at x."""
    return torch.where(x == 0, 0.0, torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=1e-300))) - 8))


def in_parts(x, n):
    """x (64 bits) as the sum of n values of bf16, each the last one's remainder, rounded."""
    out = torch.zeros_like(x)
    for _ in range(n):
        out = out + (x - out).float().bfloat16().double()
    return out


def test_the_bounds_tell_the_number_of_parts():
    gen = torch.Generator().manual_seed(7)
    k = torch.randn(128, generator=gen).bfloat16().double() * torch.exp(-torch.rand(128, generator=gen).double())
    v = torch.randn(128, generator=gen).bfloat16().double()
    off = lambda n: (in_parts(k, n) / k - 1).abs().max()  # noqa: E731
    assert off(3) <= 2.0 ** -23 and off(2) > 1.5 * STATE
    assert off(2) <= OUTPUT / 2 and off(1) > 8 * OUTPUT
    exact = k[:, None] * v[None, :]
    for n, holds in ((2, True), (1, False)):
        err = ((in_parts(k, n)[:, None] * v).float().bfloat16().double() - exact).abs()
        assert bool((err <= OUTPUT * exact.abs() + half_step(exact * (1 + OUTPUT))).all()) == holds


def one_term(seed):
    """100 tokens of which one, another for each head, has a key; queries that pick one channel of it; a state of zero before them."""
    case = make_case(seed, [100], H_v=4, H_k=4)
    gen = torch.Generator().manual_seed(seed)
    case.g = -(0.01 + 0.02 * torch.rand(1, 100, 4, generator=gen)).cuda()
    k, q = torch.zeros(1, 100, 4, 128), torch.zeros(1, 100, 4, 128)
    for h, t in enumerate((0, 21, 47, 63)):
        k[0, t, h] = torch.randn(128, generator=gen)
    channel = torch.randint(0, 128, (1, 100, 4, 1), generator=gen)
    q.scatter_(3, channel, torch.randn(1, 100, 4, 1, generator=gen))
    case.q, case.k = q.bfloat16().cuda(), k.bfloat16().cuda()
    return case, expected(case, zero=[1])


@pytest.mark.gpu
def test_states_of_one_term():
    case, (want, _, _, _) = one_term(60)
    for want_o in (True, False):
        state, _ = run(case, algo=CHUNKED, zero=[1], want_o=want_o)
        err = (state.cpu().double() - want).abs()
        assert bool((err <= STATE * want.abs()).all()), float((err / want.abs()).nan_to_num(0.0).max())


@pytest.mark.gpu
@pytest.mark.parametrize("o_dtype", [torch.float32, torch.bfloat16])
def test_outputs_of_one_term(o_dtype):
    """Inside the key's own chunk from its weight, behind it from the state."""
    case, (_, want, _, _) = one_term(61)
    o = run(case, algo=CHUNKED, zero=[1], o_dtype=o_dtype)[1].cpu().double()
    bound = OUTPUT * want.abs() + (half_step(want * (1 + OUTPUT)) if o_dtype == torch.bfloat16 else 0.0)
    err = (o - want).abs()
    assert bool((err <= bound).all()), float((err / want.abs()).nan_to_num(0.0).max())
    for t in (64, 100):  # both kinds are there
        assert bool((want[0, t - 1] != 0).any(-1).all())


@pytest.mark.gpu
def test_prompts_as_a_whole():
    """Root mean squares over 256 tokens.  States: a chunk's twelve products per sum are off by half a step of 2^-23 each, even if all one way
    (7.2e-7), ex2 by 1.2e-7, so 1e-6 holds; keys in two parts would be off by 2^-17 at most and about a third of that in the mean, 2.4e-6.  bf16
    outputs: their own rounding, and errors of 2^-16 that add to it as squares do."""
    case = make_case(62, [256], H_v=4, H_k=2)
    want_state, want, _, _ = expected(case)
    rms = lambda x: float(x.square().mean().sqrt())  # noqa: E731
    req = int(case.req[0])
    state, o = run(case, algo=CHUNKED, o_dtype=torch.bfloat16)
    assert rms(state[req].cpu().double() - want_state[req]) <= 1e-6 * rms(want_state[req])
    rounding = rms(want.float().bfloat16().double() - want)
    assert rms(o.cpu().double() - want) <= 1.05 * rounding
    o = run(case, algo=CHUNKED, o_dtype=torch.float32)[1]
    assert rms(o.cpu().double() - want) <= 2.0 ** -16 * rms(want)
