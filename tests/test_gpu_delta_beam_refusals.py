"""Each argument that dasc_delta_step, dasc_delta_draft, dasc_beam_select and dasc_beam_reorder refuse, as the one thing wrong with a call that otherwise
runs: on a plan of a device, through the C entry points.  All of them are refused on the host, before anything is launched."""
import pytest
import torch

import delta_helpers as dh
import paper_2608_30386_b200 as dasc
from paper_2608_30386_b200 import binding

pytestmark = pytest.mark.gpu
KINDS = pytest.mark.parametrize("kind", [dasc.KDA, dasc.GDN], ids=["kda", "gdn"])

LAYER = 2 * 128 * 128  # floats of a layer's states


def call(name, defaults, **changes):
    assert set(changes) <= set(defaults)
    status = getattr(binding.lib(), name)(*{**defaults, **changes}.values())
    torch.cuda.synchronize()
    return status


class States:
    """Three requests of one token over two layers, as arguments of the step and of the draft."""

    def __init__(self, kind):
        self.case = case = dh.make_case(80, [1, 1, 1], kind=kind, L=2, H_v=2, H_k=2)
        self.o = torch.zeros(2, 3, 2, 128, device="cuda")
        self.cu = case.cu.cuda()
        p = {k: getattr(case, k).data_ptr() for k in ("q", "k", "v", "g", "beta", "state", "req")}
        streams = dict(q=p["q"], k=p["k"], v=p["v"], io=binding.IO_BF16, g=p["g"], beta=p["beta"])
        pool = dict(plan=case.plan.handle, state=p["state"], ls=LAYER, rs=2 * LAYER, req=p["req"])
        ends = dict(lb=0, le=2, scale=1.0, o=self.o.data_ptr(), o_io=binding.IO_FP32)
        self.step = dict(**pool, src=None, width=1, **streams, n=3, **ends, stream=None)
        self.draft = dict(**pool, **streams, cu=self.cu.data_ptr(), used=None, zero=None, n=3, total=3, longest=1, **ends, mode=dasc.DRAFT_ADVANCE, stream=None)
        torch.cuda.synchronize()


@KINDS
def test_a_beam_with_a_source_reaches_two_states(kind):
    """The state of its source and the slot it writes: strides that make them overlap are refused for a single request too."""
    s = States(kind)
    one = dict(n=1, src=s.case.req[1:].data_ptr())
    before = s.case.state.clone()
    for rs in (0, 4, LAYER - 4):
        assert call("dasc_delta_step", s.step, **one, rs=rs) == binding.ERR_INVALID_ARG
    assert torch.equal(s.case.state, before)
    assert call("dasc_delta_step", s.step, **one) == binding.OK
    assert call("dasc_delta_step", s.step, n=1, rs=0) == binding.OK  # (one state, whichever the stride)


def test_sizes_whose_offsets_pass_32_bits():
    """Between the rows of eight tokens (both calls), and inside a head's state (drafts)."""
    s = States(dasc.KDA)
    rows, state = dh.make_plan(dasc.KDA, 2, 1, 1, 32, 2 ** 27 + 32), dh.make_plan(dasc.KDA, 2, 1, 1, 128, 2 ** 24)
    assert call("dasc_delta_step", s.step, plan=rows.handle) == binding.ERR_SHAPE
    for plan in (rows, state):
        assert call("dasc_delta_draft", s.draft, plan=plan.handle) == binding.ERR_SHAPE


@KINDS
def test_scoring_nothing(kind):
    """No requests, or requests without a token: tensors without values have no address, and nothing is refused for it."""
    case = dh.make_case(82, [0, 0], kind=kind)
    before = case.state.clone()
    empty = lambda *shape: torch.empty(*shape, device="cuda")  # noqa: E731
    streams = [empty(1, 0, 2, 128), empty(1, 0, 2, 128), empty(1, 0, 2, 128), empty(1, 0, 2, 128) if kind == dasc.KDA else empty(1, 0, 2), empty(1, 0, 2)]
    for n in (0, 2):
        cu = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
        dasc.dasc_delta_draft(case.plan, case.state, *case.strides, case.req[:n], *streams, cu, 0, 0, o=empty(1, 0, 2, 128), mode=dasc.DRAFT_SCORE)
    assert torch.equal(case.state, before)
