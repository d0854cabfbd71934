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


SHARED = [dict(plan=None), dict(n=-1), dict(lb=-1), dict(lb=2, le=1), dict(le=3), dict(io=2), dict(io=-1), dict(o_io=7), dict(state=None), dict(req=None), dict(k=None),
          dict(v=None), dict(g=None), dict(beta=None), dict(q=None), dict(ls=-4), dict(rs=-4), dict(ls=LAYER + 2), dict(rs=2 * LAYER + 1)]
OVERLAPS = [dict(ls=0), dict(ls=LAYER - 4), dict(rs=0), dict(rs=LAYER - 4), dict(lb=1, rs=0), dict(n=1, ls=4)]


@KINDS
@pytest.mark.parametrize("name", ["dasc_delta_step", "dasc_delta_draft"])
def test_one_wrong_argument(kind, name):
    s = States(kind)
    ok = s.step if name == "dasc_delta_step" else s.draft
    assert call(name, ok) == binding.OK
    before, o = s.case.state.clone(), s.o.clone()
    misaligned = dict(state=4, q=8, k=2, v=4, o=8, g=4 if kind == dasc.KDA else 2, beta=2)
    bad = [*SHARED, *OVERLAPS, *({x: ok[x] + by} for x, by in misaligned.items())]
    if name == "dasc_delta_step":
        src = s.case.req.data_ptr()
        bad += [dict(o=None), *(dict(src=src, width=w) for w in (0, -1, 33, 2))]  # (two beams per request do not make three)
    else:
        bad += [dict(total=-1), dict(longest=-1), dict(mode=2), dict(mode=-1), dict(mode=dasc.DRAFT_SCORE, o=None), dict(cu=None)]
    for x in bad:
        assert call(name, ok, **x) == binding.ERR_INVALID_ARG, x
    too_large = dict(n=2 ** 31 - 1) if name == "dasc_delta_step" else dict(total=2 ** 31)
    assert call(name, ok, **too_large) == binding.ERR_SHAPE
    for d_k, d_v in ((16, 128), (48, 128), (256, 128), (128, 48), (128, 16)):
        odd = dh.make_plan(kind, 2, 2, 2, d_k, d_v)
        assert call(name, ok, plan=odd.handle) == binding.ERR_SHAPE, (d_k, d_v)
    assert torch.equal(s.case.state, before) and torch.equal(s.o, o)


@KINDS
def test_what_a_call_does_not_use_may_be_anything(kind):
    s = States(kind)
    assert call("dasc_delta_step", s.step, n=1, rs=0) == binding.OK
    assert call("dasc_delta_step", s.step, le=1, ls=0) == binding.OK
    assert call("dasc_delta_step", s.step, width=0) == binding.OK  # (no src_idx)
    assert call("dasc_delta_draft", s.draft, n=1, total=1, rs=0) == binding.OK
    assert call("dasc_delta_draft", s.draft, le=1, ls=0) == binding.OK
    assert call("dasc_delta_draft", s.draft, o=None, q=None, o_io=7) == binding.OK
    before = s.case.state.clone()
    for x in OVERLAPS:  # (nothing is written)
        assert call("dasc_delta_draft", s.draft, **{**x, **({"total": 1} if "n" in x else {})}, mode=dasc.DRAFT_SCORE) == binding.OK, x
    assert torch.equal(s.case.state, before)


def test_one_wrong_argument_of_the_selection():
    V, dev = 12, "cuda"
    t = dict(logits=torch.randn(3, 2, V, device=dev), scores=torch.randn(3, 2, device=dev), ended=torch.zeros(3, 2, dtype=torch.int32, device=dev),
             os=torch.zeros(3, 4, device=dev), **{k: torch.zeros(3, 4, dtype=torch.int32, device=dev) for k in ("op", "ot", "oe")})
    p = {k: x.data_ptr() for k, x in t.items()}
    host = torch.randn(3, 2, V)
    ok = dict(logits=p["logits"], stride=V, dtype=binding.IO_FP32, vocab=V, scores=p["scores"], ended=None, end=-1, n=3, width=2, n_out=4, os=p["os"], op=p["op"],
              ot=p["ot"], oe=None, stream=None)
    torch.cuda.synchronize()
    name = "dasc_beam_select"
    for good in ({}, dict(dtype=binding.IO_BF16), dict(ended=p["ended"], end=V - 1), dict(oe=p["oe"]), dict(ended=p["ended"], oe=p["oe"], end=0), dict(end=V),
                 dict(n=0, logits=None)):
        assert call(name, ok, **good) == binding.OK, good
    before = {k: x.clone() for k, x in t.items()}
    for bad in (dict(n=-1), dict(vocab=0), dict(vocab=-5), dict(width=0), dict(n_out=0), dict(dtype=2), dict(dtype=-1), dict(logits=None), dict(scores=None),
                dict(os=None), dict(op=None), dict(ot=None), dict(stride=V - 1), dict(stride=-V), dict(logits=p["logits"] + 2), dict(scores=p["scores"] + 1),
                dict(logits=p["logits"] + 1, dtype=binding.IO_BF16), dict(ended=p["ended"] + 2, end=1), dict(os=p["os"] + 2), dict(op=p["op"] + 1), dict(ot=p["ot"] + 3),
                dict(oe=p["oe"] + 2), dict(ended=p["ended"]), dict(ended=p["ended"], end=V), dict(ended=p["ended"], end=-2), dict(oe=p["oe"], end=-2), dict(oe=p["oe"], end=V),
                dict(os=p["scores"]), dict(ended=p["ended"], oe=p["ended"], end=1), dict(logits=host.data_ptr())):
        assert call(name, ok, **bad) == binding.ERR_INVALID_ARG, bad
    for big in (dict(width=33), dict(n_out=65), dict(n=2 ** 31 - 1), dict(vocab=2 ** 30, stride=2 ** 30)):
        assert call(name, ok, **big) == binding.ERR_SHAPE, big
    assert all(torch.equal(t[k], before[k]) for k in t)


def test_one_wrong_argument_of_the_reordering():
    case = dh.make_case(83, [1, 1, 1], L=2)
    conv = torch.randn(case.state.shape[0], 64, device="cuda")
    parent = dh.i32([1, 1, 2])
    new, src = torch.empty_like(case.req), torch.empty_like(case.req)
    p = dict(state=case.state.data_ptr(), conv=conv.data_ptr(), req=case.req.data_ptr(), parent=parent.data_ptr(), new=new.data_ptr(), src=src.data_ptr())
    ok = dict(plan=case.plan.handle, state=p["state"], ls=LAYER, rs=2 * LAYER, conv=p["conv"], cs=256, cb=256, req=p["req"], parent=p["parent"], n=1, width=3, lb=0, le=2,
              new=p["new"], src=p["src"], stream=None)
    torch.cuda.synchronize()
    name = "dasc_beam_reorder"
    for good in ({}, dict(src=None), dict(state=None, ls=-1, rs=-1), dict(conv=None, cs=-1, cb=-1), dict(state=None, conv=None), dict(n=0, req=None), dict(le=1, ls=0), dict(le=0)):
        assert call(name, ok, **good) == binding.OK, good
    before = [x.clone() for x in (case.state, conv, new, src)]
    for bad in (dict(plan=None), dict(n=-1), dict(width=0), dict(width=-1), dict(lb=-1), dict(lb=2, le=1), dict(le=3), dict(req=None), dict(parent=None), dict(new=None),
                dict(new=p["req"]), dict(new=p["parent"]), dict(src=p["req"]), dict(src=p["parent"]), dict(src=p["new"]), dict(state=p["state"] + 4), dict(ls=-4),
                dict(rs=-4), dict(ls=LAYER + 2), dict(rs=2 * LAYER + 1), dict(ls=0), dict(ls=LAYER - 4), dict(rs=0), dict(rs=LAYER - 4), dict(lb=1, rs=LAYER - 4),
                dict(conv=p["conv"] + 8), dict(cb=-16), dict(cb=8), dict(cs=240), dict(cs=264), dict(cs=-256)):
        assert call(name, ok, **bad) == binding.ERR_INVALID_ARG, bad
    for big in (dict(width=33), dict(n=2 ** 31 - 1), dict(n=2 ** 31 - 1, state=None), dict(cb=2 ** 36, cs=2 ** 36)):
        assert call(name, ok, **big) == binding.ERR_SHAPE, big
    assert all(torch.equal(x, y) for x, y in zip((case.state, conv, new, src), before))
