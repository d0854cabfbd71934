"""dasc_decay_attn, dasc_decay_step and dasc_verify_draft as they are used together, and what a call must not do to another one."""
import numpy as np
import pytest
import torch

import paper_2608_30386_b200 as dasc
from decay_helpers import check, expected, make_case, make_plan, run
from paper_2608_30386_b200 import binding

pytestmark = pytest.mark.gpu

SEQ, CHUNKED = dasc.ALGO_SEQUENTIAL, dasc.ALGO_CHUNKED
CONTINUE, MERGE, SCORE = dasc.DECAY_CONTINUE, dasc.DECAY_SCRATCH_MERGE_LOCAL, dasc.DECAY_SCORE


def workspace(case, longest, algo=dasc.ALGO_AUTO, layers=None):
    need = dasc.dasc_decay_workspace_bytes(case.plan, len(case.lens), layers or case.L, case.T, longest, algo)
    return torch.randint(0, 255, (need,), dtype=torch.uint8, device="cuda") if need else None


# ---- long requests are run in segments ----


@pytest.mark.parametrize("lens", [[2085], [1100, 0, 5, 1500], [1024, 1025], [1023, 64, 2049]])
@pytest.mark.parametrize("decay", ["token", "head"])
def test_long_requests(lens, decay):
    case = make_case(31, lens, H_v=2, H_k=1, decay=decay)
    # split at all: more workspace than the status words
    assert workspace(case, max(lens)).numel() > 128 * 128 * 4
    want = expected(case)
    for t in (torch.float32, torch.bfloat16):
        check(case, run(case, o_dtype=t), want, True, t)
    check(case, (run(case, want_o=False)[0], None), want, True)


@pytest.mark.parametrize("mode", [CONTINUE, MERGE, SCORE])
def test_long_requests_with_used_lengths_zero_starts_and_padding(mode):
    case = make_case(32, [1500, 1100, 1300, 2000, 40], H_v=2, H_k=2)
    used, zero = [1500, 3, 700, 0, 40], [0, 1, 0, 1, 0]
    req = case.req.tolist()
    req[2] = -1
    want = expected(case, mode=mode, used=used, zero=zero, req=req)
    got = run(case, mode=mode, used=used, zero=zero, req=req)
    check(case, got, want, True)
    assert bool((got[1].cpu()[want[3] == 0] == 7.0).all())
    if mode == SCORE:
        assert torch.equal(got[0], case.state)


def test_a_bound_on_the_length_that_is_too_low_or_too_high_limits_nothing():
    case = make_case(33, [1300, 70], H_v=1, H_k=1)
    want = expected(case)
    for longest in (20, 64, 1024, 1300, 100000):
        check(case, run(case, longest=longest), want, True)


@pytest.mark.parametrize("algo", [SEQ, CHUNKED])
@pytest.mark.parametrize("n", [1, 2, 3, 7, 8, 9, 15, 16, 17])
def test_scoring_a_few_tokens(algo, n):
    case = make_case(41, [n, 1, n + 1], H_v=3, H_k=1)
    want = expected(case, mode=SCORE)
    for t in (torch.float32, torch.bfloat16):
        got = run(case, algo=algo, mode=SCORE, o_dtype=t)
        check(case, got, want, algo == CHUNKED, t)
        assert torch.equal(got[0], case.state)


# ---- many requests ----


@pytest.mark.parametrize("algo", [SEQ, CHUNKED])
def test_more_requests_than_are_sorted(algo):
    case = make_case(34, [1 + i % 3 for i in range(598)] + [130, 0], H_v=1, H_k=1)
    check(case, run(case, algo=algo), expected(case), algo == CHUNKED)


@pytest.mark.parametrize("algo", [SEQ, CHUNKED, dasc.ALGO_AUTO])
def test_no_tokens_at_all(algo):
    case = make_case(35, [0, 0, 0], L=2)
    got = run(case, algo=algo, zero=[1, 0, 1])
    check(case, got, expected(case, zero=[1, 0, 1]), False)
    assert torch.equal(run(case, algo=algo)[0], case.state)


# ---- offsets beyond 32 bits ----


@pytest.mark.parametrize("algo", [SEQ, CHUNKED])
def test_states_and_streams_far_into_memory(algo):
    near = make_case(36, [70, 3], H_v=16, H_k=16)
    want = run(near, algo=algo)
    # states 2^31 + 64 elements apart
    far_apart = 2 ** 31 + 64
    pool = torch.empty(far_apart + 16 * 16384, device="cuda")
    req = torch.tensor([1, 0], dtype=torch.int32, device="cuda")
    views = [pool[far_apart * i:far_apart * i + 16 * 16384].view(16, 128, 128) for i in (1, 0)]
    for r in range(2):
        views[r].copy_(near.state[near.req[r], 0])
    # tokens behind 2^20 + 3 others: an offset of 2^31 and more elements
    skip = 2 ** 20 + 3
    def stretch(x):
        y = torch.empty((1, skip + near.T, *x.shape[2:]), dtype=x.dtype, device="cuda")
        y[:, skip:] = x
        return y
    q, k, v, g = (stretch(x) for x in (near.q, near.k, near.v, near.g))
    o = torch.empty(v.shape, device="cuda")
    cu = torch.tensor([0, skip, skip + 70, skip + 73], dtype=torch.int32, device="cuda")
    ws = torch.empty(dasc.dasc_decay_workspace_bytes(near.plan, 3, 1, skip + near.T, 70, algo) or 16, dtype=torch.uint8, device="cuda")
    dasc.dasc_decay_attn(near.plan, pool, 16 * 16384, far_apart, torch.cat([torch.full_like(req[:1], -1), req]), q, k, v, g, cu, skip + near.T, 70, q_scale=0.7,
                         o=o, algo=algo, workspace=ws)
    torch.cuda.synchronize()
    assert torch.equal(o[:, skip:], want[1])
    for r in range(2):
        assert torch.equal(views[r], want[0][near.req[r], 0])


def test_rows_of_probabilities_far_into_memory():
    V, stride = 1000, 2 ** 30 + 8
    gen = torch.Generator().manual_seed(37)
    p, q = (torch.softmax(torch.randn(n, V, generator=gen), -1).bfloat16().cuda() for n in (5, 4))
    memory = torch.empty(4 * stride + V, dtype=torch.bfloat16, device="cuda")
    far = memory.as_strided((5, V), (stride, 1))
    far.copy_(p)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    for u in (0.0, 0.5, 1.0):
        out, kept = torch.zeros(2, 1, 5, dtype=torch.int32, device="cuda"), torch.zeros(2, 1, dtype=torch.int32, device="cuda")
        for i, rows in enumerate((p, far)):
            dasc.dasc_verify_draft(rows, q, i32([1, 5, 7, 999]), i32([0, 4]), torch.full((4,), u, device="cuda"), torch.full((1,), 0.7, device="cuda"), out[i], kept[i])
        assert torch.equal(out[0], out[1]) and torch.equal(kept[0], kept[1])


# ---- refusals ----


def test_workspaces_shapes_and_plans_that_do_not_fit():
    case = make_case(38, [100], H_v=2)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731

    def call(case, ws, algo=dasc.ALGO_AUTO, plan=None):
        dasc.dasc_decay_attn(plan or case.plan, case.state, *case.strides, case.req, case.q, case.k, case.v, case.g, case.cu.cuda(), case.T, case.T, algo=algo, workspace=ws)

    ws = workspace(case, 100)
    before = case.state.clone()
    for bad in (None, ws[:-1], torch.zeros(ws.numel() + 256, dtype=torch.uint8, device="cuda")[16:]):
        with pytest.raises(dasc.DascError) as e:
            call(case, bad)
        assert e.value.status == binding.ERR_WORKSPACE
    for other in (make_case(39, [100], d_k=64, d_v=64), make_case(39, [100], dtype=torch.float32), make_case(39, [100], d_v=64)):
        with pytest.raises(dasc.DascError) as e:
            call(other, ws, CHUNKED)
        assert e.value.status == binding.ERR_SHAPE
        call(other, None)  # and in fp32 it is run, workspace or not
        call(other, ws)
        torch.cuda.synchronize()
        assert dasc.dasc_decay_status(ws) == binding.OK
    z = np.zeros(2 * 128, np.float32)
    kda = dasc.dasc_plan(dasc.KDA, 1, 2, 2, 128, 128, z, z, w_max=16.0)
    with pytest.raises(dasc.DascError) as e:
        call(case, ws, plan=kda)
    assert e.value.status == binding.ERR_UNSUPPORTED
    with pytest.raises(dasc.DascError) as e:
        dasc.dasc_decay_step(kda, case.state, *case.strides, case.req, case.q[:, :1], case.k[:, :1], case.v[:, :1], case.g[:, :1], torch.zeros_like(case.v[:, :1]))
    assert e.value.status == binding.ERR_UNSUPPORTED
    assert torch.equal(case.state, before)
    with pytest.raises((ValueError, TypeError)):  # streams that are not laid out as they have to be, too short, of another type
        dasc.dasc_decay_attn(case.plan, case.state, *case.strides, case.req, case.q.transpose(1, 2), case.k, case.v, case.g, i32([0, 100]), 100, 100, workspace=ws, o=case.v)
    with pytest.raises((ValueError, TypeError)):
        dasc.dasc_decay_attn(case.plan, case.state, *case.strides, case.req, case.q, case.k, case.v, case.g, i32([0, 101]), 101, 101, workspace=ws)
    with pytest.raises((ValueError, TypeError)):
        dasc.dasc_decay_attn(case.plan, case.state, *case.strides, case.req, case.q, case.k, case.v.float(), case.g, i32([0, 100]), 100, 100, workspace=ws)
    with pytest.raises((ValueError, TypeError)):
        dasc.dasc_decay_attn(case.plan, case.state, *case.strides, case.req.long(), case.q, case.k, case.v, case.g, i32([0, 100]), 100, 100, workspace=ws)


@pytest.mark.parametrize("lens", [[100, 40], [2085]])
def test_a_bounded_wait_that_runs_out_is_reported_and_leaves_states_and_context_as_they_were(lens):
    case = make_case(40, lens, H_v=1, H_k=1)
    ws = workspace(case, max(lens), CHUNKED)

    def call():
        state, o = case.state.clone(), torch.zeros(1, case.T, 1, 128, device="cuda")
        dasc.dasc_decay_attn(case.plan, state, *case.strides, case.req, case.q, case.k, case.v, case.g, case.cu.cuda(), case.T, max(lens), o=o, q_scale=0.7,
                             algo=CHUNKED, workspace=ws)
        torch.cuda.synchronize()
        return state, o

    try:
        dasc.dasc_debug_set_refresh_poll_limit(1)
        state, _ = call()
    finally:
        dasc.dasc_debug_set_refresh_poll_limit(0)
    assert dasc.dasc_decay_status(ws) == binding.ERR_TIMEOUT
    assert torch.equal(state, case.state)
    check(case, call(), expected(case), True)
    assert dasc.dasc_decay_status(ws) == binding.OK


# ---- streams and graphs ----


class Server:
    """A few requests with drafted tokens: score, verify, advance, and one plain step, all on the current stream."""

    def __init__(self, seed, R=5, H=4, V=1000, most=6, algo=dasc.ALGO_AUTO):
        gen = torch.Generator().manual_seed(seed)
        self.plan, self.mask = make_plan(1, H, H, 128, 128, seed)
        self.n = [int(x) for x in torch.randint(0, most, (R,), generator=gen)]
        self.n[0] = most
        self.R, self.H, self.most, self.algo = R, H, most, algo
        rows = sum(self.n) + R
        rnd = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
        bf = lambda x: x.bfloat16().cuda()  # noqa: E731
        self.q, self.k, self.v = bf(rnd(1, rows, H, 128) / 11), bf(rnd(1, rows, H, 128) / 11), bf(rnd(1, rows, H, 128))
        self.g = -torch.rand(1, rows, H, generator=gen).cuda()
        self.q1, self.k1, self.v1, self.g1 = bf(rnd(1, R, H, 128) / 11), bf(rnd(1, R, H, 128) / 11), bf(rnd(1, R, H, 128)), -torch.rand(1, R, H, generator=gen).cuda()
        drafts = torch.tensor([0, *self.n]).cumsum(0)
        self.cu_drafts = drafts.int().cuda()
        self.cu = (drafts + torch.arange(R + 1)).int().cuda()
        self.target = torch.softmax(2 * rnd(rows, V), -1).cuda()
        at = torch.tensor([int(drafts[r]) + r + j for r in range(R) for j in range(self.n[r])], dtype=torch.long)
        self.draft = torch.softmax(torch.log(self.target.cpu()[at]) + 0.5 * rnd(len(at), V), -1).cuda()
        self.tokens = torch.multinomial(self.draft.cpu(), 1, generator=gen)[:, 0].int().cuda()
        self.u, self.un = torch.rand(len(at), generator=gen).cuda(), torch.rand(R, generator=gen).cuda()
        self.state0 = rnd(R, 1, H, 128, 128).cuda()
        self.req = torch.randperm(R, generator=gen).int().cuda()
        self.state = self.state0.clone()
        self.o, self.o1 = torch.zeros_like(self.v), torch.zeros_like(self.v1)
        self.out = torch.zeros(R, most + 1, dtype=torch.int32, device="cuda")
        self.kept = torch.zeros(R, dtype=torch.int32, device="cuda")
        need = dasc.dasc_decay_workspace_bytes(self.plan, R, 1, rows, most + 1, algo)
        self.ws = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()

    def turn(self):
        rows, strides = self.q.shape[1], (self.H * 16384, self.H * 16384)
        common = dict(algo=self.algo, workspace=self.ws)
        dasc.dasc_decay_attn(self.plan, self.state, *strides, self.req, self.q, self.k, self.v, self.g, self.cu, rows, self.most + 1, o=self.o, mode=SCORE, **common)
        dasc.dasc_verify_draft(self.target, self.draft, self.tokens, self.cu_drafts, self.u, self.un, self.out, self.kept)
        dasc.dasc_decay_attn(self.plan, self.state, *strides, self.req, None, self.k, self.v, self.g, self.cu, rows, self.most + 1, seq_used=self.kept, **common)
        dasc.dasc_decay_step(self.plan, self.state, *strides, self.req, self.q1, self.k1, self.v1, self.g1, self.o1)

    def results(self):
        torch.cuda.synchronize()
        return [x.clone() for x in (self.state, self.o, self.o1, self.out, self.kept)]


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("algo", [SEQ, CHUNKED])
def test_a_turn_with_drafts_is_the_recurrence_over_the_tokens_that_stand(algo):
    s = Server(50, algo=algo)
    s.turn()
    state, o, o1, out, kept = (x.cpu() for x in s.results())
    cu, req = s.cu.tolist(), s.req.tolist()
    # off by: bf16 outputs (2^-8 of each term in chunks, of the sum else), fp32 states
    term = 2.0 ** -8
    for r in range(s.R):
        assert 1 <= int(kept[r]) <= s.n[r] + 1
        for h in range(s.H):
            S, A = (x.clone() for x in (s.state0[req[r], 0, h].cpu().double(), s.state0[req[r], 0, h].cpu().double().abs()))
            for t in range(cu[r], cu[r + 1]):
                e = torch.exp(s.g[0, t, h].cpu().double())
                k, v, q = (x[0, t, h].cpu().double() for x in (s.k, s.v, s.q))
                S, A = e * S + torch.outer(k, v), e * A + torch.outer(k.abs(), v.abs())
                want, bound = q @ S, q.abs() @ A
                assert bool(((o[0, t, h].double() - want).abs() <= 2.1 * term * bound).all())
                if t - cu[r] + 1 == int(kept[r]):
                    S1, A1 = S.clone(), A.clone()
            e = torch.exp(s.g1[0, r, h].cpu().double())
            k, v, q = (x[0, r, h].cpu().double() for x in (s.k1, s.v1, s.q1))
            S1, A1 = e * S1 + torch.outer(k, v), e * A1 + torch.outer(k.abs(), v.abs())
            assert bool(((state[req[r], 0, h].double() - S1).abs() <= 2.0 ** -13 * A1).all())  # (400 * 2^-23 of the chunked form, and the step's)
            assert bool(((o1[0, r, h].double() - q @ S1).abs() <= 1.1 * term * (q.abs() @ A1)).all())
        assert out[r, :int(kept[r]) - 1].tolist() == s.tokens[s.cu_drafts[r]:s.cu_drafts[r] + int(kept[r]) - 1].tolist()


@pytest.mark.parametrize("algo", [SEQ, CHUNKED])
def test_a_captured_turn_replays_as_the_calls_do(algo):
    s = Server(51, algo=algo)
    want = []
    for _ in range(3):
        s.turn()
        want.append(s.results())
    s.state.copy_(s.state0)
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph.capture_begin()
        s.turn()
        graph.capture_end()
    torch.cuda.synchronize()
    assert torch.equal(s.state, s.state0)
    for w in want:
        for x in (s.o, s.o1):
            x.zero_()
        graph.replay()
        assert same(s.results(), w)
    # other numbers in the same buffers
    s.state.copy_(s.state0)
    s.u.fill_(0.999)
    graph.replay()
    got = s.results()
    s.state.copy_(s.state0)
    s.turn()
    assert same(s.results(), got)


@pytest.mark.parametrize("algo", [SEQ, CHUNKED])
def test_turns_on_two_streams_at_once(algo):
    pair = [Server(seed, R=40, H=8, algo=algo) for seed in (52, 53)]
    want = []
    for s in pair:
        for _ in range(4):
            s.turn()
        want.append(s.results())
        s.state.copy_(s.state0)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in pair]
    for _ in range(4):
        for s, stream in zip(pair, streams):
            with torch.cuda.stream(stream):
                s.turn()
    for s, w in zip(pair, want):
        assert same(s.results(), w)


def test_prompts_and_drafts_over_states_from_the_pool():
    """Store and Load around the operators: what a plan keeps comes back, the prompt's tokens refresh the heads it omits, and drafts go on from there."""
    case = make_case(54, [90, 17, 200], H_v=6, H_k=3, rate_lo=0.05, spare=0)
    R, H = 3, case.H_v
    keep = torch.from_numpy(case.mask[0].astype(bool))
    slots = torch.arange(R, dtype=torch.int32, device="cuda")
    pool = torch.zeros(R, int(case.plan.slot_floats), device="cuda")
    dasc.dasc_pack(case.plan, case.state, *case.strides, case.req, pool, slots)
    state = torch.full_like(case.state, 9.0)
    dasc.dasc_restore(case.plan, pool, slots, state, *case.strides, case.req)
    torch.cuda.synchronize()
    got, _ = run(case, mode=MERGE, state=state, want_o=False)
    for r in range(R):
        assert torch.equal(got[case.req[r], 0][keep].cpu(), case.state[case.req[r], 0][keep].cpu())
    want = expected(case, mode=MERGE)
    check(case, (got, None), want, True)
    # the next tokens continue from it
    drafts = make_case(54, [5, 5, 5], H_v=6, H_k=3, spare=0)
    drafts.state = got
    check(drafts, run(drafts, mode=SCORE), expected(drafts, mode=SCORE), False)
    assert torch.equal(drafts.state, got)
    check(drafts, run(drafts, used=[1, 5, 3], want_o=False), expected(drafts, used=[1, 5, 3]), False)


def test_calls_without_requests_or_layers():
    case = make_case(55, [20, 3])
    none = torch.zeros(0, dtype=torch.int32, device="cuda")
    state = case.state.clone()
    empty = [x[:, :0] for x in (case.q, case.k, case.v, case.g)]
    dasc.dasc_decay_attn(case.plan, state, *case.strides, none, *empty, torch.zeros(1, dtype=torch.int32, device="cuda"), 0, 0, o=empty[2])
    dasc.dasc_decay_step(case.plan, state, *case.strides, none, *empty, empty[2])
    dasc.dasc_decay_attn(case.plan, state, *case.strides, case.req, *(x[:0] for x in (case.q, case.k, case.v, case.g)), case.cu.cuda(), case.T, 20, layer_begin=1,
                         layer_end=1)
    dasc.dasc_verify_draft(torch.zeros(0, 5, device="cuda"), None, none, torch.zeros(1, dtype=torch.int32, device="cuda"), none.float(), none.float(),
                           torch.zeros(0, 3, dtype=torch.int32, device="cuda"), none)
    torch.cuda.synchronize()
    assert torch.equal(state, case.state)


@pytest.mark.parametrize("algo", [SEQ, CHUNKED])
def test_a_state_that_hardly_decays_does_not_drift(algo):
    """A factor rounded to fp32 would be off by the same half ulp (up to 2^-25) at each of n applications: n 2^-25 of a state that nothing is added to.
    Here 8192 tokens of zero keys are run at several decays, so all of the error is the factors': token by token, rounded, it would come to
    2^-12 for some of them.  With what the factor is short of carried along, an application is off by the rounding of the state
    itself (2^-24, both ways about as often) and the sum of log-decays by an ulp.  1024 groups of 8 tokens (128 chunks of 64): at most 1024 * 2^-24 even
    if all roundings went one way, and 2^-22 * G for the exponents' relative error, G <= 1 in all."""
    n = 8192
    case = make_case(56, [n], H_v=4, H_k=4, decay="head", spare=0)
    g = torch.tensor([[-1.1e-5, -3.3e-5, -7.7e-5, -1.2e-4]], device="cuda")
    case.g = g
    case.k = torch.zeros_like(case.k)
    state, _ = run(case, algo=algo, want_o=False)
    want = case.state.double() * torch.exp(g.double() * n)[0].view(1, 1, 4, 1, 1)
    err = ((state.double() - want).abs() / want.abs()).max()
    assert float(err) <= 1024 * 2.0 ** -24 + 2.0 ** -22
