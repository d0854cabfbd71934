"""What dasc_delta_step, dasc_delta_draft, dasc_beam_select and dasc_beam_reorder refuse, without a GPU: the library's own checks through ctypes (a host-only
plan, addresses that nobody follows) and those of the Python calls; and what their sources promise."""
import os
import re

import numpy as np
import pytest
import torch

import paper_2608_30386_b200 as dasc
from paper_2608_30386_b200 import binding, build

P = 0x1000  # an aligned address that is never followed


def plan(kind=dasc.KDA, d_k=128, d_v=128, L=2, H=2):
    n = L * H * (d_k if kind == dasc.KDA else 1)
    return dasc.dasc_plan(kind, L, H, H, d_k, d_v, np.zeros(n, np.float32), np.zeros(n, np.float32), w_max=16.0, device=-1)


def test_states_calls_refuse_before_any_launch():
    p = plan()
    step = lambda **kw: binding.lib().dasc_delta_step(*{  # noqa: E731
        **dict(plan=p.handle, state=P, ls=32768, rs=65536, req=P, src=None, width=1, q=P, k=P, v=P, io=0, g=P, beta=P, n=2, lb=0, le=2, scale=1.0, o=P, o_io=0,
               stream=None), **kw}.values())
    draft = lambda **kw: binding.lib().dasc_delta_draft(*{  # noqa: E731
        **dict(plan=p.handle, state=P, ls=32768, rs=65536, req=P, q=P, k=P, v=P, io=0, g=P, beta=P, cu=P, used=None, zero=None, n=1, total=1, longest=1, lb=0,
               le=2, scale=1.0, o=P, o_io=0, mode=0, stream=None), **kw}.values())
    for call in (step, draft):
        assert call() == binding.ERR_INVALID_ARG  # no device
        for bad in (dict(plan=None), dict(n=-1), dict(lb=-1), dict(lb=2, le=1), dict(le=3), dict(io=2), dict(o_io=7)):
            assert call(**bad) == binding.ERR_INVALID_ARG, bad
    for bad in (dict(total=-1), dict(longest=-1), dict(mode=2), dict(mode=1, o=None)):
        assert draft(**bad) == binding.ERR_INVALID_ARG, bad
    for bad in (dict(src=P, width=0), dict(src=P, width=33), dict(src=P, width=2, n=3)):
        assert step(**bad) == binding.ERR_INVALID_ARG, bad


def test_selection_refuses_before_any_launch():
    call = lambda **kw: binding.lib().dasc_beam_select(*{  # noqa: E731
        **dict(logits=P, stride=10, dtype=1, vocab=10, scores=P, ended=None, end=-1, n=1, width=2, n_out=4, os=P + 16, op=P + 32, ot=P + 48, oe=None, stream=None),
        **kw}.values())
    for bad in (dict(n=-1), dict(vocab=0), dict(width=0), dict(n_out=0), dict(dtype=2), dict(logits=None), dict(scores=None), dict(os=None), dict(op=None),
                dict(ot=None), dict(stride=9), dict(logits=P + 2), dict(scores=P + 1), dict(ended=P), dict(ended=P, end=10), dict(oe=P, end=-2), dict(os=P)):
        assert call(**bad) == binding.ERR_INVALID_ARG, bad
    for big in (dict(width=33), dict(n_out=65), dict(n=2 ** 31 - 1), dict(vocab=2 ** 30, stride=2 ** 30)):
        assert call(**big) == binding.ERR_SHAPE, big
    assert call(n=0) == binding.OK


def test_reordering_refuses_before_any_launch():
    p = plan()
    call = lambda **kw: binding.lib().dasc_beam_reorder(*{  # noqa: E731
        **dict(plan=p.handle, state=P, ls=32768, rs=65536, conv=None, cs=0, cb=0, req=P, parent=P + 64, n=1, width=4, lb=0, le=2, new=P + 128, src=None,
               stream=None), **kw}.values())
    assert call() == binding.ERR_INVALID_ARG  # no device
    for bad in (dict(plan=None), dict(n=-1), dict(width=0)):
        assert call(**bad) == binding.ERR_INVALID_ARG, bad


class Stream:
    cuda_stream = 0


def test_python_calls_look_at_their_tensors():
    p = plan(L=1)
    f, i = torch.zeros(1, 4, 2, 128), torch.zeros(4, dtype=torch.int32)
    args = [p, torch.zeros(8), 32768, 32768, i, f, f, f, f, torch.zeros(1, 4, 2)]
    with pytest.raises(ValueError, match="not on the current CUDA device"):  # tensors of the host
        dasc.dasc_delta_step(*args, f, stream=Stream())
    with pytest.raises(ValueError, match="not on the current CUDA device"):
        dasc.dasc_delta_draft(*args, torch.zeros(5, dtype=torch.int32), 4, 4, o=f, stream=Stream())
    with pytest.raises(TypeError, match="type"):
        dasc.dasc_delta_step(p, torch.zeros(8, dtype=torch.float64), *args[2:], f, stream=Stream())
    with pytest.raises(TypeError):
        dasc.dasc_delta_step(*args[:2], 32768.0, *args[3:], f, stream=Stream())
    x, s = torch.zeros(2, 3, 10), torch.zeros(2, 3)
    out, idx = torch.zeros(2, 4), torch.zeros(2, 4, dtype=torch.int32)
    for bad in ((x[:, :2], s, out, idx, idx), (x, s, out, idx[:1], idx), (x[..., ::2], s, out, idx, idx), (torch.zeros(2, 4, 10)[:, :3], s, out, idx, idx)):
        with pytest.raises(ValueError):
            dasc.dasc_beam_select(*bad, stream=Stream())
    with pytest.raises(ValueError):
        dasc.dasc_beam_select(x, s, out, idx, idx, ended=idx, end_token=1, stream=Stream())
    with pytest.raises(ValueError):
        dasc.dasc_beam_reorder(p, None, 0, 0, idx, idx[:1], idx.clone(), stream=Stream())
    with pytest.raises(ValueError, match="not on the current CUDA device"):
        dasc.dasc_beam_reorder(p, None, 0, 0, idx, idx, idx.clone(), stream=Stream())


@pytest.mark.parametrize("name", ["delta_decode.cu", "beam.cu"])
def test_nothing_is_read_past_what_an_earlier_kernel_may_still_be_writing(name):
    code = re.sub(r"//[^\n]*|/\*.*?\*/", "", open(os.path.join(build.CSRC, name)).read(), flags=re.S)
    assert not re.search(r"\.nc\b|__ldg|__restrict__", code)
    assert len(re.findall(r"__global__", code)) <= len(re.findall(r"stream_order_(?:wait|begin)\(\)", code))
