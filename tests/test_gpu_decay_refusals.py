"""Each argument that dasc_decay_attn, dasc_decay_step and dasc_verify_draft refuse, as the one thing wrong with a call that otherwise runs: on a plan
of a device, through the C entry points.  All of them are refused on the host, before anything is launched."""
import pytest
import torch

import paper_2608_30386_b200 as dasc
from decay_helpers import make_case, make_plan
from paper_2608_30386_b200 import binding

pytestmark = pytest.mark.gpu

LAYER = 2 * 128 * 128  # floats of a layer's states


def call(name, defaults, **changes):
    assert set(changes) <= set(defaults)
    status = getattr(binding.lib(), name)(*{**defaults, **changes}.values())
    torch.cuda.synchronize()
    return status


@pytest.fixture(scope="module")
def buffers():
    case = make_case(80, [1, 1, 1], L=2, H_v=2, H_k=2)
    o = torch.zeros(2, 3, 2, 128, device="cuda")
    ws = torch.zeros(dasc.dasc_decay_workspace_bytes(case.plan, 3, 2, 3, 100, dasc.ALGO_CHUNKED), dtype=torch.uint8, device="cuda")
    p = {k: getattr(case, k).data_ptr() for k in ("q", "k", "v", "g", "state", "req")}
    cu = case.cu.cuda()
    shared = dict(plan=case.plan.handle, state=p["state"], ls=LAYER, rs=2 * LAYER, req=p["req"], q=p["q"], k=p["k"], v=p["v"], io=binding.IO_BF16, g=p["g"], decay=0)
    attn = dict(**shared, cu=cu.data_ptr(), used=None, zero=None, n=3, total=3, longest=100, lb=0, le=2, scale=1.0, o=o.data_ptr(), o_io=binding.IO_FP32, mode=0,
                algo=0, ws=ws.data_ptr(), wsb=ws.numel(), stream=None)
    step = dict(**shared, n=3, lb=0, le=2, scale=1.0, o=o.data_ptr(), o_io=binding.IO_FP32, stream=None)
    torch.cuda.synchronize()
    return case, attn, step, (o, ws, cu)


SHARED = [dict(plan=None), dict(n=-1), dict(lb=-1), dict(lb=2, le=1), dict(le=3), dict(io=2), dict(io=-1), dict(o_io=7), dict(decay=2), dict(decay=-1),
          dict(state=None), dict(req=None), dict(k=None), dict(v=None), dict(g=None), dict(q=None), dict(ls=-4), dict(rs=-4), dict(ls=LAYER + 2), dict(rs=2 * LAYER + 1)]
OVERLAPS = [dict(ls=0), dict(ls=LAYER - 4), dict(rs=0), dict(rs=LAYER - 4), dict(lb=1, rs=0), dict(n=1, ls=4)]


@pytest.mark.parametrize("name", ["dasc_decay_attn", "dasc_decay_step"])
def test_one_wrong_argument(buffers, name):
    case, attn, step, _ = buffers
    ok = attn if name == "dasc_decay_attn" else step
    assert call(name, ok) == binding.OK
    before = case.state.clone()
    bad = [*SHARED, *OVERLAPS, *({x: ok[x] + by} for x, by in (("state", 4), ("q", 8), ("k", 2), ("v", 4), ("o", 8), ("g", 2)))]
    if name == "dasc_decay_attn":
        bad += [dict(total=-1), dict(longest=-1), dict(mode=3), dict(mode=-1), dict(algo=3), dict(algo=-1), dict(mode=2, o=None), dict(cu=None)]
        bad += [dict(x, mode=dasc.DECAY_SCRATCH_MERGE_LOCAL) for x in OVERLAPS]
    else:
        bad += [dict(o=None)]
    for x in bad:
        assert call(name, ok, **x) == binding.ERR_INVALID_ARG, x
    too_large = dict(n=2 ** 31 - 1) if name == "dasc_decay_step" else dict(total=2 ** 31)
    assert call(name, ok, **too_large) == binding.ERR_SHAPE
    odd, _ = make_plan(2, 2, 2, 48, 128)
    assert call(name, ok, plan=odd.handle) == binding.ERR_SHAPE
    assert torch.equal(case.state, before)


def test_strides_that_a_single_request_or_layer_never_uses(buffers):
    _, attn, step, _ = buffers
    for name, ok in (("dasc_decay_attn", attn), ("dasc_decay_step", step)):
        assert call(name, ok, n=1, rs=0, **({"total": 1} if ok is attn else {})) == binding.OK
        assert call(name, ok, le=1, ls=0) == binding.OK


def test_scoring_may_share_a_state():
    """Nothing is written, so requests may score over one state, by equal entries of req_idx or a stride of zero."""
    case = make_case(81, [5, 5, 5], H_v=2)
    want = torch.zeros(1, 15, 2, 128, device="cuda")
    got = torch.zeros_like(want)
    first = case.state[:1].contiguous()
    zeros = torch.zeros(3, dtype=torch.int32, device="cuda")
    for o, rs, req in ((want, LAYER, zeros), (got, 0, case.req)):
        dasc.dasc_decay_attn(case.plan, first, LAYER, rs, req, case.q, case.k, case.v, case.g, case.cu.cuda(), 15, 5, o=o, mode=dasc.DECAY_SCORE)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and bool((want != 0).all())


def test_one_wrong_argument_of_the_verification():
    V, dev = 12, "cuda"
    t = dict(target=torch.rand(4, V, device=dev), draft=torch.rand(3, V, device=dev), tokens=torch.ones(3, dtype=torch.int32, device=dev),
             cu=torch.tensor([0, 3], dtype=torch.int32, device=dev), ua=torch.rand(3, device=dev), un=torch.rand(1, device=dev),
             out=torch.zeros(1, 4, dtype=torch.int32, device=dev), kept=torch.zeros(1, dtype=torch.int32, device=dev))
    p = {k: x.data_ptr() for k, x in t.items()}
    host = torch.rand(4, V)
    ok = dict(target=p["target"], ts=V, draft=p["draft"], ds=V, dtype=binding.IO_FP32, vocab=V, tokens=p["tokens"], cu=p["cu"], ua=p["ua"], un=p["un"], n=1, most=3,
              out=p["out"], os=4, kept=p["kept"], stream=None)
    torch.cuda.synchronize()
    assert call("dasc_verify_draft", ok) == binding.OK
    assert call("dasc_verify_draft", ok, draft=None, ds=0) == binding.OK
    before = t["out"].clone(), t["kept"].clone()
    for bad in (dict(n=-1), dict(most=-1), dict(vocab=0), dict(vocab=-5), dict(dtype=2), dict(target=None), dict(cu=None), dict(un=None), dict(out=None),
                dict(kept=None), dict(tokens=None), dict(ua=None), dict(ts=V - 1), dict(ds=V - 1), dict(os=3), dict(target=p["target"] + 2),
                dict(draft=p["draft"] + 1), dict(target=host.data_ptr())):
        assert call("dasc_verify_draft", ok, **bad) == binding.ERR_INVALID_ARG, bad
    assert torch.equal(t["out"], before[0]) and torch.equal(t["kept"], before[1])
