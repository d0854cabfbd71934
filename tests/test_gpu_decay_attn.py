"""dasc_decay_attn and dasc_decay_step against the recurrence in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2608_30386_b200 as dasc
from decay_helpers import check, expected, make_case, run

pytestmark = pytest.mark.gpu

SEQ, CHUNKED = dasc.ALGO_SEQUENTIAL, dasc.ALGO_CHUNKED
ALGOS = [pytest.param(SEQ, id="seq"), pytest.param(CHUNKED, id="chunked"), pytest.param(dasc.ALGO_AUTO, id="auto")]
both = pytest.mark.parametrize("algo", ALGOS[:2])
EDGE_LENS = [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 200]


@pytest.mark.parametrize("algo", ALGOS)
@pytest.mark.parametrize("n", EDGE_LENS)
def test_lengths(algo, n):
    case = make_case(n, [n, 3, n + 5], H_v=2, H_k=1)
    check(case, run(case, algo=algo), expected(case), algo != SEQ)


@both
def test_types_of_outputs_and_layers(algo):
    case = make_case(5, [70, 0, 131, 1], L=3, H_v=4, H_k=2)
    want = expected(case, layers=(1, 3))
    for t in (torch.float32, torch.bfloat16):
        check(case, run(case, algo=algo, o_dtype=t, layers=(1, 3)), want, algo != SEQ, t)
    state, _ = run(case, algo=algo, layers=(1, 3), want_o=False)
    check(case, (state, None), want, algo != SEQ)


@both
@pytest.mark.parametrize("mode", [dasc.DECAY_CONTINUE, dasc.DECAY_SCRATCH_MERGE_LOCAL, dasc.DECAY_SCORE])
@pytest.mark.parametrize("decay", ["token", "head"])
def test_modes_with_used_lengths_zero_starts_and_padding(algo, mode, decay):
    case = make_case(11, [9, 80, 0, 64, 130, 5, 66], H_v=4, H_k=2, decay=decay)
    used, zero = [4, 80, 3, 0, 65, 99, -2], [1, 0, 1, 1, 0, 0, 0]
    req = case.req.tolist()
    req[5] = -1
    want = expected(case, mode=mode, used=used, zero=zero, req=req)
    got = run(case, algo=algo, mode=mode, used=used, zero=zero, req=req)
    check(case, got, want, algo != SEQ)
    # what is not written keeps its bits: states that nobody owns, retained heads, rows of o behind the last used token
    same = torch.ones(case.state.shape, dtype=torch.bool)
    for r in range(len(req)):
        runs = min(used[r], case.lens[r]) > 0
        if req[r] >= 0 and mode != dasc.DECAY_SCORE and (runs or zero[r] or mode == dasc.DECAY_SCRATCH_MERGE_LOCAL):
            written = np.ones_like(case.mask[0]) if mode == dasc.DECAY_CONTINUE else 1 - case.mask[0]
            same[req[r], 0, torch.from_numpy(written.astype(bool))] = False
    assert torch.equal(got[0].cpu()[same].view(torch.int32), case.state.cpu()[same].view(torch.int32))
    assert bool((got[1].cpu()[want[3] == 0] == 7.0).all())
    if mode != dasc.DECAY_SCORE:
        check(case, (run(case, algo=algo, mode=mode, used=used, zero=zero, req=req, want_o=False)[0], None), want, algo != SEQ)


@pytest.mark.parametrize("d_k", [32, 64, 128])
@pytest.mark.parametrize("d_v", [32, 64, 96, 128, 256])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_shapes_and_types_token_by_token(d_k, d_v, dtype):
    case = make_case(d_k + d_v, [1, 8, 37], H_v=6, H_k=3, d_k=d_k, d_v=d_v, dtype=dtype)
    check(case, run(case, algo=SEQ), expected(case), False)


@pytest.mark.parametrize("heads", [1, 2, 5, 40, 160])
def test_widths_of_the_column_parts(heads):
    # few heads: narrow parts on many SMs; many: wide ones
    for d in (32, 64, 128):
        case = make_case(heads, [3, 1], H_v=heads, H_k=1, d_k=d, d_v=128)
        check(case, run(case, algo=SEQ), expected(case), False)


@both
def test_strong_and_vanishing_decay(algo):
    """Decay that forgets everything at once (-inf), far more than fp32's exponent holds, none at all (0), next to one another."""
    case = make_case(21, [150, 64], H_v=2)
    g = case.g.cpu()
    g[0, ::7, 0] = 0.0
    g[0, 40, 0] = -float("inf")
    g[0, 41:60, 0] = -1e-3
    g[0, 100, 0] = -3e38
    g[0, :, 1] = -50.0
    g[0, 10:90, 1] = 0.0
    case.g = g.cuda()
    check(case, run(case, algo=algo), expected(case), algo != SEQ)


@both
def test_a_large_drop_does_not_cost_the_tokens_behind_it_precision(algo):
    """Sums of log-decays reach thousands inside a chunk while neighbouring tokens differ by little."""
    case = make_case(22, [128], H_v=1, H_k=1)
    g = torch.full((1, 128, 1), -1e-2)
    g[0, ::16, 0] = -700.0
    case.g = g.cuda()
    check(case, run(case, algo=algo), expected(case), algo != SEQ)


@both
@pytest.mark.parametrize("what", ["nan", "inf", "-inf"])
def test_values_that_are_none_stay_behind_their_token_and_in_their_column(algo, what):
    case = make_case(23, [100, 40], H_v=2, H_k=2)
    clean = run(case, algo=algo)
    case.v[0, 70, 1, 33] = float(what)  # request 0, head 1, column 33
    state, o = run(case, algo=algo)
    bad_o = torch.zeros_like(o, dtype=torch.bool)
    bad_o[0, 70:100, 1, 33] = True
    assert not bool(o[bad_o].isfinite().any())
    assert torch.equal(o[~bad_o], clean[1][~bad_o])
    bad_s = torch.zeros_like(state, dtype=torch.bool)
    bad_s[int(case.req[0]), 0, 1, :, 33] = True
    assert not bool(state[bad_s].isfinite().any())
    assert torch.equal(state[~bad_s], clean[0][~bad_s])


@both
def test_what_lies_behind_a_request_does_not_reach_it(algo):
    """Tokens behind the used ones, or of the next request, hold NaN; a state that is not read holds NaN too."""
    case = make_case(24, [70, 70, 3], H_v=2)
    used = [67, 70, 3]
    clean = run(case, algo=algo, used=used, zero=[0, 1, 0])
    for x in (case.q, case.k, case.v, case.g):
        x[0, 67:70] = float("nan")
    case.state[int(case.req[1])] = float("nan")
    got = run(case, algo=algo, used=used, zero=[0, 1, 0])
    assert torch.equal(got[0], clean[0])
    assert torch.equal(got[1], clean[1])


@both
def test_keys_and_queries_that_are_none(algo):
    """A NaN in q is that token's alone; an infinity in k is in the state from its token on."""
    case = make_case(25, [100], H_v=2, H_k=2)
    clean = run(case, algo=algo)
    case.q[0, 20, 0, 3] = float("nan")
    case.k[0, 50, 1, 9] = float("inf")
    state, o = run(case, algo=algo)
    keep = torch.ones_like(o, dtype=torch.bool)
    keep[0, 20, 0] = False
    keep[0, 50:, 1] = False
    assert torch.equal(o[keep], clean[1][keep])
    assert bool(o[0, 20, 0].isnan().all()) and not bool(o[0, 50:, 1].isfinite().any())
    assert torch.equal(state[int(case.req[0]), 0, 0], clean[0][int(case.req[0]), 0, 0])


@both
def test_equal_calls_give_equal_bits_and_the_bound_on_the_length_is_a_hint(algo):
    case = make_case(26, [300, 5, 64], H_v=4)
    a, b = run(case, algo=algo), run(case, algo=algo)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    want = expected(case)
    for longest in (0, 1, 64, 2 ** 31 - 1):  # too small, or far too large
        check(case, run(case, algo=algo, longest=longest), want, algo != SEQ)


@both
def test_pool_strides(algo):
    """Layer-major pools and gaps between states; what lies between them is not touched."""
    case = make_case(27, [20, 66], L=2, H_v=2)
    want = expected(case)
    n, unit = case.state.shape[0], case.H_v * case.d_k * case.d_v
    for layer_major in (False, True):
        ls, rs = ((n * (unit + 64) + 32, unit + 64) if layer_major else (unit + 96, 2 * (unit + 96) + 128))
        pool = torch.full((2 * n * (unit + 200),), 3.0, device="cuda")
        shape, stride = (n, 2, case.H_v, case.d_k, case.d_v), (rs, ls, case.d_k * case.d_v, case.d_v, 1)
        pool.as_strided(shape, stride).copy_(case.state)
        before = pool.clone()
        o = torch.zeros(2, case.T, 2, 128, device="cuda")
        need = dasc.dasc_decay_workspace_bytes(case.plan, 2, 2, case.T, 66, algo)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
        dasc.dasc_decay_attn(case.plan, pool, ls, rs, case.req, case.q, case.k, case.v, case.g, case.cu.cuda(), case.T, 66, q_scale=0.7, o=o, algo=algo,
                             workspace=ws)
        torch.cuda.synchronize()
        check(case, (pool.as_strided(shape, stride).clone(), o), want, algo != SEQ)
        touched = torch.zeros_like(pool, dtype=torch.bool)
        touched.as_strided(shape, stride).fill_(True)
        assert torch.equal(pool[~touched], before[~touched])


# ---- single tokens ---------------------------------------------------------------------------------------------------------------

def step(case, o_dtype=torch.float32, req=None, stream=None, state=None):
    state = case.state.clone() if state is None else state
    o = torch.full((case.L, case.T, case.H_v, case.d_v), 7.0, device="cuda", dtype=o_dtype)
    dasc.dasc_decay_step(case.plan, state, *case.strides, case.req if req is None else torch.tensor(req, dtype=torch.int32, device="cuda"), case.q, case.k,
                         case.v, case.g, o, decay=dasc.DECAY_PER_HEAD if case.g.dim() == 2 else dasc.DECAY_PER_TOKEN, q_scale=0.7, stream=stream)
    torch.cuda.synchronize()
    return state, o


@pytest.mark.parametrize("n", [1, 2, 7, 80])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d_k,d_v", [(128, 128), (64, 64), (32, 96), (128, 64), (64, 128)])
def test_step(n, dtype, d_k, d_v):
    case = make_case(n, [1] * n, L=2, H_v=4, H_k=2, d_k=d_k, d_v=d_v, dtype=dtype, decay="head" if n % 2 else "token")
    want = expected(case)
    for t in (torch.float32, torch.bfloat16):
        check(case, step(case, t), want, False, t)


def test_step_leaves_padding_alone_and_forgets_at_minus_infinity():
    case = make_case(3, [1] * 6, H_v=4)
    case.g[0, 2] = -float("inf")
    req = case.req.tolist()
    req[1] = req[4] = -1
    got, want = step(case, req=req), expected(case, req=req)
    check(case, got, want, False)
    assert bool((got[1][:, [1, 4]] == 7.0).all())
    owned = [r for r in req if r >= 0]
    rest = [i for i in range(case.state.shape[0]) if i not in owned]
    assert torch.equal(got[0][rest], case.state[rest])


def test_step_of_a_few_heads_equals_the_prompt_form():
    case = make_case(4, [1] * 5, H_v=2)
    a, b = step(case), run(case, algo=SEQ)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
