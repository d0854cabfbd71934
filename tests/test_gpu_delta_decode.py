"""dasc_delta_step and dasc_delta_draft against the recurrence in 64 bits."""
import pytest
import torch

import delta_helpers as dh
import paper_2608_30386_b200 as dasc

pytestmark = pytest.mark.gpu
KINDS = pytest.mark.parametrize("kind", [dasc.KDA, dasc.GDN], ids=["kda", "gdn"])


@KINDS
@pytest.mark.parametrize("d_k, d_v, H_v, H_k, n", [(128, 128, 4, 2, 3), (128, 128, 8, 8, 40), (64, 64, 4, 4, 5), (64, 192, 2, 1, 3), (32, 32, 3, 3, 1),
                                                   (32, 96, 6, 2, 7), (128, 32, 2, 2, 2), (128, 64, 8, 4, 45), (64, 128, 6, 2, 60), (32, 64, 8, 8, 50)])
@pytest.mark.parametrize("dtype, o_dtype", [(torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32), (torch.bfloat16, torch.float32),
                                            (torch.float32, torch.bfloat16)])
def test_step(kind, d_k, d_v, H_v, H_k, n, dtype, o_dtype):
    case = dh.make_case(n, [1] * n, kind=kind, H_v=H_v, H_k=H_k, d_k=d_k, d_v=d_v, dtype=dtype)
    got, want = dh.step(case, o_dtype=o_dtype), dh.expected(case)
    dh.check(case, got, want, o_dtype)
    assert dh.worst(got[0], want[0]) < 1e-5


@KINDS
@pytest.mark.parametrize("d_k, d_v, H_v, H_k, n", [(128, 128, 16, 8, 80), (64, 256, 8, 8, 80), (32, 64, 32, 32, 76), (64, 64, 32, 16, 75)])
def test_step_of_many_states(kind, d_k, d_v, H_v, H_k, n):
    """Enough states for the wider parts."""
    case = dh.make_case(n, [1] * n, kind=kind, H_v=H_v, H_k=H_k, d_k=d_k, d_v=d_v)
    dh.check(case, dh.step(case, o_dtype=torch.bfloat16), dh.expected(case), torch.bfloat16)


@KINDS
@pytest.mark.parametrize("lens", [[1], [5] * 3, [8, 9], [0, 1, 2, 3, 4, 5, 6, 7], [17, 0, 30], [2] * 80, [9] * 40])
@pytest.mark.parametrize("score", [False, True], ids=["advance", "score"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
def test_draft(kind, lens, score, dtype):
    case = dh.make_case(len(lens), lens, kind=kind, H_v=4, H_k=2, dtype=dtype)
    got = dh.run(case, mode=dasc.DRAFT_SCORE if score else dasc.DRAFT_ADVANCE)
    want = dh.expected(case, score=score)
    dh.check(case, got, want)
    assert dh.worst(got[0], want[0]) < 1e-5 and dh.worst(got[1], want[1]) < 1e-5
    if score:
        assert torch.equal(got[0], case.state)


@KINDS
@pytest.mark.parametrize("d_k, d_v", [(64, 64), (32, 32), (32, 160), (64, 32), (128, 64), (128, 256), (64, 128), (32, 128)])
@pytest.mark.parametrize("H_v, R", [(2, 3), (6, 60)])
def test_draft_shapes(kind, d_k, d_v, H_v, R):
    lens = [(3 * i) % 11 for i in range(R)]
    case = dh.make_case(3, lens, kind=kind, H_v=H_v, H_k=2, d_k=d_k, d_v=d_v, dtype=torch.float32)
    dh.check(case, dh.run(case), dh.expected(case))
    dh.check(case, dh.run(case, mode=dasc.DRAFT_SCORE, o_dtype=torch.bfloat16), dh.expected(case, score=True), torch.bfloat16)


@KINDS
def test_advance_over_the_tokens_that_stand_without_outputs(kind):
    lens, used = [5, 5, 9, 12, 0, 4, 3], [1, 5, 8, 20, 3, 0, -2]
    case = dh.make_case(7, lens, kind=kind, H_v=4)
    got = dh.run(case, used=used, want_o=False)
    dh.check(case, got, dh.expected(case, used=used))
    with_o = dh.run(case, used=used)
    dh.check(case, with_o, dh.expected(case, used=used))  # rows behind the tokens that are run stay as they were
    assert torch.equal(with_o[0], got[0])


@KINDS
def test_zero_starts_and_padding(kind):
    lens, zero = [3, 0, 2, 4, 0, 1], [1, 1, 0, 1, 0, 5]
    case = dh.make_case(8, lens, kind=kind)
    req = case.req.tolist()
    req[3] = -1
    case.state[req[0]] = float("nan")  # what is not read may hold anything
    want = dh.expected(case, zero=zero, req=req)
    for i, x in enumerate(want):
        assert not bool(torch.isnan(x).any()), i
    dh.check(case, dh.run(case, zero=zero, req=req), want)


@KINDS
def test_requests_without_any_token(kind):
    """Nothing is read but who starts from zero; nobody does, or states are set to zero."""
    case = dh.make_case(19, [0, 0, 0], kind=kind, L=2)
    req, cu = case.req, torch.zeros(4, dtype=torch.int32, device="cuda")
    for zero in (None, [0, 1, 0]):
        state = case.state.clone()
        dasc.dasc_delta_draft(case.plan, state, *case.strides, req, None, case.k, case.v, case.g, case.beta, cu, 0, 0, from_zero=dh.i32(zero))
        want = case.state.clone()
        if zero:
            want[int(req[1])] = 0
        assert torch.equal(state, want)
    empty = torch.empty(0, dtype=torch.int32, device="cuda")
    dasc.dasc_delta_step(case.plan, state, *case.strides, empty, case.q, case.k, case.v, case.g, case.beta, torch.empty(2, 0, 2, 128, device="cuda"))


@KINDS
def test_padding_in_a_step(kind):
    case = dh.make_case(9, [1] * 6, kind=kind)
    req = case.req.tolist()
    req[1] = req[5] = -1
    dh.check(case, dh.step(case, req=req), dh.expected(case, req=req))


@KINDS
def test_layers_of_a_group_and_both_layouts_of_the_pool(kind):
    case = dh.make_case(10, [2, 7], kind=kind, L=3, H_v=2)
    dh.check(case, dh.run(case, layers=(1, 3)), dh.expected(case, layers=(1, 3)))
    # layer-major, with a gap behind every state
    unit = case.H_v * case.d_k * case.d_v
    slots = case.state.shape[0]
    pool = torch.full((case.L, slots, unit + 8), 3.0, device="cuda")
    pool[:, :, :unit] = case.state.transpose(0, 1).reshape(case.L, slots, unit)
    o = torch.zeros(case.L, case.T, case.H_v, case.d_v, device="cuda")
    dasc.dasc_delta_draft(case.plan, pool, slots * (unit + 8), unit + 8, case.req, case.q, case.k, case.v, case.g, case.beta, case.cu.cuda(), case.T, 7, o=o,
                          q_scale=0.7)
    state, o2 = dh.run(case)
    assert torch.equal(pool[:, :, :unit].reshape(case.L, slots, *case.state.shape[2:]).transpose(0, 1), state) and torch.equal(o, o2)
    assert bool((pool[:, :, unit:] == 3).all())


@KINDS
@pytest.mark.parametrize("pattern", [[0, 0, 0, 0], [3, 3, 1, 1], [2, 0, 2, 2], [1, 2, 3, 0], [-1, 0, 0, 2]])
def test_beams_that_continue_one_state(kind, pattern):
    """Each beam starts from its source and writes its own slot; sources and slots as the reordering gives them."""
    width, groups = 4, 12
    case = dh.make_case(11, [1] * (width * groups), kind=kind, H_v=4)
    slots = case.req.view(groups, width)
    parent = torch.tensor([pattern if g % 3 else pattern[::-1] for g in range(groups)], dtype=torch.int32, device="cuda")
    new, src = torch.empty_like(slots), torch.empty_like(slots)
    dasc.dasc_beam_reorder(case.plan, None, 0, 0, slots, parent, new, src_idx=src)
    got = dh.step(case, req=new.flatten().tolist(), src=src.flatten().tolist(), width=width)
    dh.check(case, got, dh.expected(case, req=new.flatten().tolist(), src=src.flatten().tolist()))
    # and the same bits as states that are copied first
    copied, new2 = case.state.clone(), torch.empty_like(slots)
    dasc.dasc_beam_reorder(case.plan, copied, *case.strides, slots, parent, new2)
    assert torch.equal(new, new2)
    req = torch.where(src < 0, src, new).flatten().tolist()
    again = dh.step(case, req=req, state=copied)
    touched = [s for s in req if s >= 0]
    assert torch.equal(got[0][touched], again[0][touched]) and torch.equal(got[1], again[1])


@KINDS
def test_a_step_is_a_draft_of_one_token(kind):
    case = dh.make_case(12, [1] * 37, kind=kind, H_v=8, dtype=torch.float32)
    (s1, o1), (s2, o2) = dh.step(case), dh.run(case)
    want = dh.expected(case)
    for x in ((s1, o1), (s2, o2)):
        dh.check(case, x, want)


@KINDS
def test_log_decays_at_both_ends(kind):
    """Nothing decays; everything is forgotten (-inf, and far below what fp32 can hold), in single channels or altogether."""
    case = dh.make_case(13, [6, 9, 4], kind=kind, H_v=3, H_k=3, dtype=torch.float32)
    case.g[:, :4] = 0.0
    case.g[:, 7] = float("-inf")
    case.g[:, 9, 1] = -200.0
    case.g[:, 16, 2] = float("-inf")
    for lens in (None, [1] * 19):
        if lens:
            case = dh.make_case(13, lens, kind=kind, H_v=3, H_k=3, dtype=torch.float32)
            case.g[:, 3] = float("-inf")
            case.g[:, 5] = 0.0
            dh.check(case, dh.step(case), dh.expected(case))
        else:
            dh.check(case, dh.run(case), dh.expected(case))


@KINDS
def test_a_value_that_is_none_stays_in_its_column(kind):
    case = dh.make_case(14, [6, 3], kind=kind, dtype=torch.float32)
    plain = dh.run(case)
    case.v[0, 2, 1, 5] = float("nan")
    case.v[0, 7, 0, 9] = float("inf")
    state, o = dh.run(case)
    for r, h, c, first, last in ((0, 1, 5, 2, 6), (1, 0, 9, 7, 9)):
        slot = int(case.req[r])
        assert bool((~torch.isfinite(o[0, first:last, h, c])).all()) and bool((~torch.isfinite(state[slot, 0, h, :, c])).any())
        o[0, first:last, h, c] = plain[1][0, first:last, h, c]
        state[slot, 0, h, :, c] = plain[0][slot, 0, h, :, c]
    assert torch.equal(o, plain[1]) and torch.equal(state, plain[0])


@KINDS
@pytest.mark.parametrize("what", ["k", "g", "beta", "q"])
def test_nothing_runs_backwards(kind, what):
    """Tokens before one that is no number, in their group as well, and other requests keep their bits."""
    case = dh.make_case(20, [7, 2, 11], kind=kind, dtype=torch.float32)
    plain = dh.run(case)
    for t in (4, 9 + 8):  # of the first and the third request
        getattr(case, what)[0, t] = float("nan")
    state, o = dh.run(case)
    kept = [0, 1, 2, 3, 7, 8, *range(9, 17)]
    assert torch.equal(o[0, kept], plain[1][0, kept])
    if what == "q":
        kept = [t for t in range(20) if t not in (4, 17)]
        assert torch.equal(o[0, kept], plain[1][0, kept]) and torch.equal(state, plain[0])
        assert bool(torch.isnan(o[0, [4, 17]]).all())
    else:
        assert bool(torch.isnan(o[0, [5, 6, 18, 19]]).all()) and torch.equal(state[int(case.req[1])], plain[0][int(case.req[1])])


def test_states_that_hardly_decay_keep_their_precision():
    """A constant decay of 1 - 1e-5 rounded to fp32 would be off by 6e-8 in every one of 20,000 tokens, 1.2e-3 of a state in the end."""
    case = dh.make_case(15, [1], kind=dasc.GDN, H_v=2, dtype=torch.float32)
    case.g.fill_(-1.00013e-5)
    case.beta.zero_()
    state = case.state.clone()
    o = torch.empty(1, 1, 2, 128, device="cuda")
    for _ in range(20000):
        dasc.dasc_delta_step(case.plan, state, *case.strides, case.req, case.q, case.k, case.v, case.g, case.beta, o)
    slot = int(case.req[0])
    want = case.state[slot].double() * torch.exp(20000 * case.g[0, 0, 0].double())
    # each token rounds each value once (2^-24, of either sign) and the remainder of its factor (2^-24 of at most 2^-24): 20000 roundings at random
    # stay below 8 sqrt(20000) 2^-24 = 6.8e-5
    assert float(((state[slot].double() - want) / want).abs().max()) < 6.8e-5


@KINDS
def test_equal_calls_give_equal_bits(kind):
    case = dh.make_case(16, [5] * 30 + [13] * 3, kind=kind, H_v=8)
    a, b = dh.run(case), dh.run(case)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_a_slot_behind_two_to_the_31_floats():
    """Addresses beyond 32 bits: the last of 34 slots that are 2^26 floats apart (8.5 GiB)."""
    case = dh.make_case(17, [3, 1], H_v=2)
    far, unit = 33, case.H_v * 128 * 128
    pool = torch.empty((far * 2 ** 26 + unit,), device="cuda")
    for slot in (1, far):
        pool[slot * 2 ** 26:slot * 2 ** 26 + unit] = case.state[int(case.req[0 if slot == far else 1])].flatten()
    o = torch.empty(1, case.T, 2, 128, device="cuda")
    req = dh.i32([far, 1])
    dasc.dasc_delta_draft(case.plan, pool, unit, 2 ** 26, req, case.q, case.k, case.v, case.g, case.beta, case.cu.cuda(), case.T, 3, o=o, q_scale=0.7)
    state, want = dh.run(case)
    assert torch.equal(o, want)
    for slot, r in ((far, 0), (1, 1)):
        assert torch.equal(pool[slot * 2 ** 26:slot * 2 ** 26 + unit], state[int(case.req[r])].flatten())
