"""dasc_beam_select and dasc_beam_reorder against their definitions."""
import numpy as np
import pytest
import torch

import beam_helpers as bh
import delta_helpers as dh
import paper_2608_30386_b200 as dasc

pytestmark = pytest.mark.gpu
TYPES = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])


def inputs(seed, R, W, V, dtype, spread=2.5):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(R, W, V, generator=gen, device="cuda") * spread
    return x.to(dtype), torch.randn(R, W, generator=gen, device="cuda") - 10


@TYPES
@pytest.mark.parametrize("R, W, V, n", [(1, 1, 1, 1), (2, 3, 5, 4), (1, 4, 31, 8), (3, 2, 1000, 4), (1, 4, 32000, 4), (2, 5, 50257, 10), (1, 8, 131072, 16),
                                        (1, 32, 16385, 64), (1, 3, 300007, 33), (40, 4, 4099, 8), (80, 4, 20000, 4), (150, 2, 40001, 17), (300, 3, 2003, 6),
                                        (1, 16, 70000, 32), (5, 7, 16384, 7), (2, 1, 40, 64), (150, 32, 501, 64), (3, 32, 40000, 64)])
def test_select(dtype, R, W, V, n):
    x, s = inputs(R + W, R, W, V, dtype)
    bh.same(bh.call(x, s, n), bh.define(x, s, None, -1, n), x)


@TYPES
def test_rows_that_are_strided_or_start_anywhere(dtype):
    big, s = inputs(3, 3, 4, 6007, dtype)
    want = bh.define(big[..., 3:5003], s, None, -1, 8)
    bh.same(bh.call(big[..., 3:5003], s, 8), want, big)
    bh.same(bh.call(big[..., 3:5003].contiguous().view(12, 5000), s, 8), want, big)


@TYPES
@pytest.mark.parametrize("V", [7, 5000, 60000])
def test_ties_go_to_the_lower_beam_and_token(dtype, V):
    """Equal rows of equal scores, rows of one value, and rows of few different values."""
    x, s = inputs(4, 6, 5, V, dtype)
    s[:] = -3.0
    x[0] = 0.0
    x[1] = x[1, :1]
    x[2] = torch.round(x[2])
    x[3, :, ::2] = 8.0
    x[4, 1:] = x[4, :1].flip(-1)
    x[5] = torch.arange(V, device="cuda").div(3, rounding_mode="floor").to(dtype).clamp(max=60000.0)
    for n in (5, 16, 40):
        got, want = bh.call(x, s, n), bh.define(x, s, None, -1, n)
        # Rows 1 .. 4 of request 4 are row 0 backwards.  The sums of their exponentials are equal as numbers and not as sums of rounded terms, which come in
        # another order (the oracle's as well): which of those beams is ahead is not defined, so there each place is held to its total, and the rest to equality.
        totals = s[4].double()[:, None] + torch.log_softmax(x[4].double(), -1)
        picked = (got[1][4].long(), got[2][4].long())
        m = torch.from_numpy(want[1][4] >= 0).cuda()
        assert torch.equal(picked[0] >= 0, m) and len(set(zip(*(p[m].tolist() for p in picked)))) == int(m.sum())
        held = totals[picked[0][m], picked[1][m]]
        assert float((held - torch.from_numpy(want[0][4]).cuda()[m]).abs().max()) <= 2 * 2.0 ** -17
        for k in (0, 1, 2):
            got[k][4] = torch.from_numpy(want[k][4]).cuda()
        bh.same(got, want, x)


@TYPES
def test_masked_logits(dtype):
    """-inf, NaN, +inf and the type's lowest value in places, rows with nothing left, rows with less than is wanted, all in one corner."""
    V = 33000
    x, s = inputs(5, 7, 4, V, dtype)
    inf, low = float("inf"), torch.finfo(dtype).min
    x[0, :, 7:] = -inf
    x[1, 1] = -inf
    x[1, 2] = float("nan")
    x[2] = -inf
    x[3, :, 1::2] = low
    x[3, :, 5] = inf
    x[4, :, :] = low
    x[4, 0, 100:103] = 1.0
    x[5, :, :32500] = -inf
    x[6, 3, :] = -inf
    x[6, 3, 20000] = -5.0
    got, want = bh.call(x, s, 8), bh.define(x, s, None, -1, 8)
    bh.same(got, want, x)
    assert got[1][2].tolist() == [-1] * 8 and got[2][2].tolist() == [-1] * 8 and bool(torch.isneginf(got[0][2]).all())


def test_beams_that_do_not_count_and_beams_that_have_ended():
    x, s = inputs(6, 4, 4, 3001, torch.float32)
    s[0, 1:] = -float("inf")  # the first step
    s[1, 2], s[2, 0] = float("nan"), float("inf")
    s[3] = -float("inf")
    ended = [[0, 0, 0, 0], [1, 0, 1, 0], [1, 1, 1, 1], [1, 0, 0, 0]]
    x[1, 0] = float("nan")  # (not read)
    for n in (3, 4, 9):
        got = bh.call(x, s, n, ended, 17, want_ended=True)
        want = bh.define(x, s, ended, 17, n)
        bh.same(got, want, x)
        over = [[int(p < 0 or ended[r][p] or t == 17) for p, t in zip(want[1][r], want[2][r])] for r in range(4)]
        assert got[3].tolist() == over


def test_scores_and_ended_beams_in_place():
    x, s = inputs(7, 5, 4, 2000, torch.float32)
    ended = torch.tensor([[0, 1, 0, 0]] * 5, dtype=torch.int32, device="cuda")
    want = bh.define(x, s, ended.tolist(), 3, 4)
    parent, token = (torch.empty(5, 4, dtype=torch.int32, device="cuda") for _ in range(2))
    dasc.dasc_beam_select(x, s, s, parent, token, ended=ended, out_ended=ended, end_token=3)
    bh.same((s, parent, token), want, x)
    assert ended.tolist() == [[int(p == 1 or t == 3) for p, t in zip(want[1][r], want[2][r])] for r in range(5)]


def test_scores_of_the_best_are_those_of_log_softmax():
    x, s = inputs(8, 9, 6, 91234, torch.float32, spread=6.0)
    total = (s.double()[..., None] + torch.log_softmax(x.double(), -1)).flatten(1)
    value, at = total.topk(12)
    got = bh.call(x, s, 12)
    assert torch.equal(got[1].long() * 91234 + got[2].long(), at)
    # half a step of fp32, and a sum of exponentials: arguments of up to 16 rounded twice (2^-19), ex2 2^-22, 13 additions in fp32 (2^-20)
    assert float((got[0].double() - value).abs().max()) <= 2.0 ** -18 + float(value.abs().max()) * 2.0 ** -24


@TYPES
@pytest.mark.parametrize("V", [40000, 70001])
def test_good_tokens_side_by_side(dtype, V):
    """A grammar that leaves neighbours only, as -inf and as low values; logits that rise with the token; plateaus higher than what is wanted."""
    x, s = inputs(11, 6, 3, V, dtype)
    low = -1e30
    x[0, :, :9000] = -float("inf")
    x[0, :, 9150:] = -float("inf")
    x[1, :, :9000] = low
    x[1, :, 9150:] = low
    x[2] = torch.arange(V, device="cuda").mul(1e-3).to(dtype)
    x[3] = torch.arange(V, 0, -1, device="cuda").mul(1e-3).to(dtype)
    x[4] = x[4].clamp(min=0.5)
    x[5] = x[5].clamp(max=0.5)
    for n in (4, 64):
        got, want = bh.call(x, s, n), bh.define(x, s, None, -1, n)
        bh.same(got, want, x)


def test_beams_that_have_ended_in_every_place():
    """What is shared out over a request's thread blocks are the rows that count."""
    x, s = inputs(12, 32, 5, 9000, torch.float32)
    ended = [[r >> b & 1 for b in range(5)] for r in range(32)]
    for n in (5, 12):
        bh.same(bh.call(x, s, n, ended, 7), bh.define(x, s, ended, 7, n), x)


def test_equal_calls_give_equal_bits():
    x, s = inputs(9, 20, 8, 30011, torch.bfloat16)
    a, b = bh.call(x, s, 16), bh.call(x, s, 16)
    assert all(torch.equal(p, q) for p, q in zip(a, b))


# ---- reordering --------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kind", [dasc.KDA, dasc.GDN], ids=["kda", "gdn"])
@pytest.mark.parametrize("W, R, d_k, d_v, L", [(1, 3, 32, 32, 1), (2, 1, 128, 128, 3), (4, 9, 64, 64, 2), (5, 7, 32, 4, 4), (32, 3, 16, 12, 2), (3, 40, 128, 128, 1)])
def test_reorder(kind, W, R, d_k, d_v, L):
    gen = torch.Generator().manual_seed(W * R)
    H, n = 2, R * W + 3
    plan = dh.make_plan(kind, L, H, H, d_k, d_v)
    state = torch.randint(-2 ** 31, 2 ** 31 - 1, (n, L, H, d_k, d_v), generator=gen, dtype=torch.int64).to(torch.int32).cuda().view(torch.float32)
    conv = torch.randint(0, 255, (n, 48 * 33), generator=gen, dtype=torch.int16).cuda().view(torch.bfloat16)
    slots = torch.randperm(n, generator=gen)[:R * W].view(R, W)
    parent = torch.randint(-1 if W > 2 else 0, W + (W > 3), (R, W), generator=gen)
    want_state, want_conv = state.clone(), conv.clone()
    want_new, want_src = [], []
    for r in range(R):
        new, src = bh.assign(slots[r].tolist(), parent[r].tolist())
        want_new.append(new)
        want_src.append(src)
        for a, b in zip(new, src):
            if b >= 0 and a != b:
                want_state[a], want_conv[a] = state[b], conv[b]
    req, par = (x.to(torch.int32).cuda() for x in (slots, parent))
    new, src = torch.full_like(req, 77), torch.full_like(req, 77)
    unit = H * d_k * d_v
    dasc.dasc_beam_reorder(plan, state, unit, L * unit, req, par, new, src_idx=src, conv=conv)
    assert new.tolist() == want_new and src.tolist() == want_src
    assert torch.equal(state.view(torch.int32), want_state.view(torch.int32))
    assert torch.equal(conv.view(torch.int16), want_conv.view(torch.int16))
    assert [sorted(x) for x in new.tolist()] == [sorted(x) for x in slots.tolist()]


def test_reorder_leaves_other_layers_gaps_and_padding_alone():
    plan = dh.make_plan(dasc.GDN, 4, 2, 1, 32, 32)
    unit = 2 * 32 * 32
    state = torch.randn(6, 4, unit + 4, device="cuda")
    before = state.clone()
    req = dh.i32([[5, 0, 2], [-1, -1, -1], [1, 3, -1]])
    parent = dh.i32([[1, 1, 1], [0, 0, 0], [1, 1, 1]])
    new, src = torch.empty_like(req), torch.empty_like(req)
    dasc.dasc_beam_reorder(plan, state, unit + 4, 4 * (unit + 4), req, parent, new, src_idx=src, layer_begin=1, layer_end=3)
    assert new.tolist() == [[0, 5, 2], [-1, -1, -1], [3, 1, -1]] and src.tolist() == [[0, 0, 0], [-1, -1, -1], [3, 3, 3]]
    before[5, 1:3, :unit] = before[2, 1:3, :unit] = before[0, 1:3, :unit]
    before[1, 1:3, :unit] = before[3, 1:3, :unit]
    assert torch.equal(state, before)


def test_reorder_of_convolution_states_or_slots_alone():
    plan = dh.make_plan(dasc.KDA, 1, 1, 1, 32, 32)
    conv = torch.arange(4 * 16, dtype=torch.float32, device="cuda").view(4, 16)
    wide = torch.zeros(4, 32, device="cuda")
    wide[:, :16] = conv
    req, parent = dh.i32([[0, 1, 2, 3]]), dh.i32([[2, 2, 0, 2]])
    new = torch.empty_like(req)
    dasc.dasc_beam_reorder(plan, None, 0, 0, req, parent, new, conv=wide[:, :16])
    assert new.tolist() == [[2, 1, 0, 3]]
    conv[1] = conv[3] = conv[2]
    assert torch.equal(wide[:, :16], conv) and bool((wide[:, 16:] == 0).all())
