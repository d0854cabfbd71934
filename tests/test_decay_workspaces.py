"""A workspace of dasc_decay_attn that is sized once, for the largest calls, serves every smaller one."""
import random

import numpy as np
import pytest
import torch

import paper_2608_30386_b200 as dasc
from decay_helpers import make_case, run


def query(plan, n_req, layers, total, longest, algo=dasc.ALGO_AUTO):
    return dasc.dasc_decay_workspace_bytes(plan, n_req, layers, total, longest, algo)


@pytest.mark.parametrize("heads", [1, 4, 32, 48, 300])
def test_the_size_never_falls_as_a_call_grows(heads):
    n = 4 * heads
    plan = dasc.dasc_plan(dasc.GDN, 4, heads, heads, 128, 128, np.zeros(n, np.float32), np.zeros(n, np.float32), device=-1)
    rng = random.Random(heads)
    for algo in (dasc.ALGO_AUTO, dasc.ALGO_CHUNKED):
        assert query(plan, 64, 1, 64 * 32768, 32768, algo) >= query(plan, 1, 1, 32768, 32768, algo) >= query(plan, 1, 1, 2048, 2048, algo) > 0
        for _ in range(2000):
            small = [rng.randint(1, 40), rng.randint(1, 4), int(2 ** rng.uniform(0, 20)), int(2 ** rng.uniform(0, 16))]
            large = [x + rng.choice([0, 0, 1, x, 7 * x]) for x in small]
            large[1] = min(large[1], 4)
            assert query(plan, *large, algo) >= query(plan, *small, algo), (small, large)
        # streams so long that a call falls back to the other form do not make it fall either
        assert query(plan, 1, 4, 2 ** 31 - 1, 32768, algo) >= query(plan, 1, 1, 32768, 32768, algo)


@pytest.mark.gpu
def test_one_workspace_for_calls_of_every_size():
    H, most, longest = 20, 16, 2100
    plan = make_case(70, [1], L=2, H_v=H, H_k=H).plan
    size = query(plan, most, 2, most * longest, longest)
    memory = torch.full((size + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    for lens in ([2085], [300] * most, [1100, 40], [1024, 1025, 1500], [70], [1400] * 7, [3, 5], [2100] * 14):
        case = make_case(71, lens, L=2, H_v=H, H_k=H)
        for layers in ((0, 1), (0, 2)):
            want = run(case, layers=layers)
            got = run(case, layers=layers, workspace=memory[:size])
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), (lens, layers)
    assert bool((memory[size:] == 0x5A).all())


@pytest.mark.gpu
@pytest.mark.parametrize("offset", [0, 4, 16, 252])
def test_the_status_is_that_of_the_last_call_where_the_workspace_is_not_aligned(offset):
    """The form that needs no workspace takes any that begins at a whole word, and the status that it leaves there is its own."""
    case = make_case(72, [5, 3])
    memory = torch.full((8192,), 0xFF, dtype=torch.uint8, device="cuda")
    run(case, algo=dasc.ALGO_SEQUENTIAL, workspace=memory[offset:offset + 4096])  # (looks at the status)
    assert bool((memory[:offset] == 0xFF).all()) and bool((memory[offset + 4096:] == 0xFF).all())


@pytest.mark.gpu
@pytest.mark.parametrize("algo", [dasc.ALGO_SEQUENTIAL, dasc.ALGO_CHUNKED])
@pytest.mark.parametrize("offset", [1, 2, 255])
def test_a_workspace_between_words_is_refused(algo, offset):
    case = make_case(73, [5, 3])
    memory = torch.full((8192,), 0xFF, dtype=torch.uint8, device="cuda")
    with pytest.raises(dasc.DascError) as e:
        run(case, algo=algo, workspace=memory[offset:offset + 4096])
    assert e.value.status == dasc.binding.ERR_WORKSPACE
    assert bool((memory == 0xFF).all())


@pytest.mark.gpu
@pytest.mark.parametrize("o_dtype", [torch.float32, torch.bfloat16])
def test_long_requests_one_behind_the_other_in_one_workspace_and_replayed(o_dtype):
    """Calls that are split into segments, on one stream with nothing between them, as they are and from a graph."""
    cases = [make_case(74, [2085, 7], H_v=8, H_k=4), make_case(75, [1100, 1300], H_v=8, H_k=4, decay="head")]
    size = max(query(c.plan, 2, 1, c.T, max(c.lens)) for c in cases)
    ws = torch.full((size,), 0xFF, dtype=torch.uint8, device="cuda")
    want = [run(c, o_dtype=o_dtype) for c in cases]
    states, outs = [c.state.clone() for c in cases], [torch.zeros_like(w[1]) for w in want]
    cus = [c.cu.cuda() for c in cases]

    def calls():
        for c, state, o, cu in zip(cases, states, outs, cus):
            dasc.dasc_decay_attn(c.plan, state, *c.strides, c.req, c.q, c.k, c.v, c.g, cu, c.T, max(c.lens), q_scale=0.7, o=o, workspace=ws,
                                 decay=dasc.DECAY_PER_HEAD if c.g.dim() == 2 else dasc.DECAY_PER_TOKEN)

    def check_and_start_again():
        torch.cuda.synchronize()
        assert dasc.dasc_decay_status(ws) == 0
        for c, state, o, w in zip(cases, states, outs, want):
            owned = c.req.long()
            assert torch.equal(state[owned], w[0][owned]) and torch.equal(o[:, :c.T], w[1][:, :c.T])
            state.copy_(c.state)
            o.zero_()
        torch.cuda.synchronize()

    calls()
    check_and_start_again()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.stream(side):
        graph.capture_begin()
        calls()
        graph.capture_end()
    for _ in range(3):
        graph.replay()
        check_and_start_again()
