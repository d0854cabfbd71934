"""Blobs of more than one tile, and what lies behind 2^31 values: single tokens, forks, rows of logits."""
import pytest
import torch

import beam_helpers as bh
import delta_helpers as dh
import paper_2608_30386_b200 as dasc

pytestmark = pytest.mark.gpu
TILE = 1024  # vectors of 16 bytes that a thread block copies


@pytest.mark.parametrize("vecs", [1, TILE - 1, TILE, TILE + 1, 5003])
@pytest.mark.parametrize("states", [True, False], ids=["beside states", "alone"])
def test_convolution_blobs_of_several_tiles(vecs, states):
    """With a gap behind each blob; a beam that is continued three times, one that is dropped, one without a parent."""
    R, W, L, H = 5, 5, 2, 3
    gen = torch.Generator().manual_seed(vecs)
    plan = dh.make_plan(dasc.GDN, L, H, H, 32, 32)
    unit, n = H * 32 * 32, R * W + 2
    state = torch.randn(n, L, unit, generator=gen).cuda()
    pool = torch.randint(-2 ** 31, 2 ** 31 - 1, (n, vecs * 4 + 12), generator=gen, dtype=torch.int64).to(torch.int32).cuda()
    slots = torch.randperm(n, generator=gen)[:R * W].view(R, W)
    parent = torch.stack([torch.tensor([1, 1, 3, 1, 4])[torch.randperm(W, generator=gen)] for _ in range(R)])
    parent[2, 0] = -1
    want_state, want_pool = state.clone(), pool.clone()
    want_new = []
    for r in range(R):
        new, src = bh.assign(slots[r].tolist(), parent[r].tolist())
        want_new.append(new)
        for a, b in zip(new, src):
            if b >= 0 and a != b:
                want_state[a], want_pool[a, :vecs * 4] = state[b], pool[b, :vecs * 4]
    req, par = (x.to(torch.int32).cuda() for x in (slots, parent))
    new = torch.empty_like(req)
    before = state.clone()
    dasc.dasc_beam_reorder(plan, state if states else None, unit, L * unit, req, par, new, conv=pool[:, :vecs * 4])
    assert new.tolist() == want_new
    assert torch.equal(state, want_state if states else before) and torch.equal(pool, want_pool)


class Far:
    """Slots 2^26 values apart; the last one begins behind 2^31 values (8.5 GiB)."""

    def __init__(self, case, slots):
        self.case, self.unit = case, case.H_v * 128 * 128
        self.pool = torch.empty((max(slots) * 2 ** 26 + self.unit,), device="cuda")

    def at(self, slot):
        return self.pool[slot * 2 ** 26:slot * 2 ** 26 + self.unit]


@pytest.mark.parametrize("kind", [dasc.KDA, dasc.GDN], ids=["kda", "gdn"])
def test_a_step_far_away(kind):
    """In place, and from a near state to a far slot and the other way round."""
    case = dh.make_case(17, [1, 1], kind=kind, H_v=2)
    far = Far(case, (1, 33))
    args = (case.q, case.k, case.v, case.g, case.beta)
    want = dh.step(case)
    for i, slot in enumerate((33, 1)):
        far.at(slot).copy_(case.state[int(case.req[i])].flatten())
    o = torch.empty(1, 2, 2, 128, device="cuda")
    dasc.dasc_delta_step(case.plan, far.pool, far.unit, 2 ** 26, dh.i32([33, 1]), *args, o, q_scale=0.7)
    for i, slot in enumerate((33, 1)):
        assert torch.equal(far.at(slot), want[0][int(case.req[i])].flatten())
    assert torch.equal(o, want[1])
    for i, (slot, source) in enumerate(((33, 1), (1, 33))):
        far.at(source).copy_(case.state[int(case.req[i])].flatten())
        out = torch.empty(1, 1, 2, 128, device="cuda")
        dasc.dasc_delta_step(case.plan, far.pool, far.unit, 2 ** 26, dh.i32([slot]), *(y[:, i:i + 1].contiguous() for y in args), out, src_idx=dh.i32([source]),
                             beam_width=1, q_scale=0.7)
        assert torch.equal(far.at(slot), want[0][int(case.req[i])].flatten()) and torch.equal(out[:, 0], want[1][:, i])
        assert torch.equal(far.at(source), case.state[int(case.req[i])].flatten())


def test_forks_between_near_and_far_slots():
    case = dh.make_case(18, [1], H_v=2)
    far = Far(case, (0, 1, 33, 34))
    for i, slot in enumerate((0, 1, 33, 34)):
        far.at(slot).copy_(torch.randn(far.unit, generator=torch.Generator().manual_seed(i)).cuda())
    old = {slot: far.at(slot).clone() for slot in (0, 1, 33, 34)}
    req, new = dh.i32([[0, 33], [34, 1]]), dh.i32([[9, 9], [9, 9]])
    dasc.dasc_beam_reorder(case.plan, far.pool, far.unit, 2 ** 26, req, dh.i32([[0, 0], [0, 0]]), new)
    assert new.tolist() == [[0, 33], [34, 1]]
    for slot, src in ((0, 0), (33, 0), (34, 34), (1, 34)):
        assert torch.equal(far.at(slot), old[src])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("gap", [2 ** 31, 2 ** 31 + 7], ids=["aligned", "not aligned"])
def test_rows_of_logits_far_apart(dtype, gap):
    V = 20011
    x = torch.empty(gap + V, device="cuda", dtype=dtype).as_strided((1, 2, V), (2 * gap, gap, 1))
    gen = torch.Generator(device="cuda").manual_seed(9)
    x.copy_(torch.randn(1, 2, V, generator=gen, device="cuda") * 2.5)
    s = torch.tensor([[-3.0, -3.5]], device="cuda")
    bh.same(bh.call(x, s, 8), bh.define(x, s, None, -1, 8), x)
