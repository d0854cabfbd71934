"""What the calls of decayed linear attention and draft verification refuse, without a GPU: the library's own checks through ctypes (a
host-only plan, addresses that nobody follows) and those of the Python calls."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2608_30386_b200 as dasc
from paper_2608_30386_b200 import binding

P = 0x1000  # an aligned address that is never followed


def plan(kind=dasc.GDN, d_k=128, d_v=128, L=2, H=2):
    n = L * H * (d_k if kind == dasc.KDA else 1)
    return dasc.dasc_plan(kind, L, H, H, d_k, d_v, np.zeros(n, np.float32), np.zeros(n, np.float32), w_max=16.0, device=-1)


def test_a_host_only_plan_and_bad_arguments_are_refused_before_any_launch():
    p = plan()
    attn = lambda **kw: binding.lib().dasc_decay_attn(*{  # noqa: E731
        **dict(plan=p.handle, state=P, ls=32768, rs=65536, req=P, q=P, k=P, v=P, io=0, g=P, decay=0, cu=P, used=None, zero=None, n=1, total=1, longest=1,
               lb=0, le=2, scale=1.0, o=P, o_io=0, mode=0, algo=0, ws=None, wsb=0, stream=None), **kw}.values())
    step = lambda **kw: binding.lib().dasc_decay_step(*{  # noqa: E731
        **dict(plan=p.handle, state=P, ls=32768, rs=65536, req=P, q=P, k=P, v=P, io=0, g=P, decay=0, n=1, lb=0, le=2, scale=1.0, o=P, o_io=0,
               stream=None), **kw}.values())
    for call in (attn, step):
        assert call() == binding.ERR_INVALID_ARG  # no device
        assert call(plan=None) == binding.ERR_INVALID_ARG
    for bad in (dict(n=-1), dict(total=-1), dict(longest=-1), dict(lb=-1), dict(lb=2, le=1), dict(le=3), dict(io=2), dict(o_io=7), dict(decay=2), dict(mode=3),
                dict(algo=3), dict(mode=2, o=None)):
        assert attn(**bad) == binding.ERR_INVALID_ARG, bad


def test_workspace_query():
    n = C.c_size_t(5)
    f = binding.lib().dasc_decay_workspace_bytes
    p = plan()
    assert f(None, 1, 1, 1, 1, 0, C.byref(n)) == binding.ERR_INVALID_ARG
    assert f(p.handle, 1, 1, 1, 1, 0, None) == binding.ERR_INVALID_ARG
    for bad in ((-1, 1, 1, 1, 0), (1, -1, 1, 1, 0), (1, 1, -1, 1, 0), (1, 1, 1, 1, 9)):
        assert f(p.handle, *bad, C.byref(n)) == binding.ERR_INVALID_ARG
    assert dasc.dasc_decay_workspace_bytes(p, 4, 1, 4, 1, dasc.ALGO_SEQUENTIAL) == 0
    assert dasc.dasc_decay_status(None) == binding.OK


def test_verification_refuses_before_any_launch():
    call = lambda **kw: binding.lib().dasc_verify_draft(*{  # noqa: E731
        **dict(target=P, ts=10, draft=P, ds=10, dtype=1, vocab=10, tokens=P, cu=P, ua=P, un=P, n=1, most=2, out=P, os=3, kept=P, stream=None), **kw}.values())
    for bad in (dict(n=-1), dict(most=-1), dict(vocab=0), dict(dtype=5), dict(target=None), dict(cu=None), dict(un=None), dict(out=None), dict(kept=None),
                dict(tokens=None), dict(ua=None), dict(ts=9), dict(ds=9), dict(os=2), dict(target=P + 2), dict(draft=P + 1)):
        assert call(**bad) == binding.ERR_INVALID_ARG, bad
    assert call(n=0) == binding.OK
    assert call(n=2 ** 31 - 1) == binding.ERR_SHAPE


class Stream:
    cuda_stream = 0


def test_python_calls_look_at_their_tensors():
    p = plan(L=1)
    f, i = torch.zeros(1, 4, 2, 128), torch.zeros(4, dtype=torch.int32)
    args = [p, torch.zeros(8), 32768, 32768, i, f, f, f, torch.zeros(1, 4, 2), torch.zeros(5, dtype=torch.int32), 4, 4]
    with pytest.raises(ValueError, match="not on the current CUDA device"):  # tensors of the host
        dasc.dasc_decay_attn(*args, o=f, stream=Stream())
    with pytest.raises(TypeError, match="type"):
        dasc.dasc_decay_step(p, torch.zeros(8, dtype=torch.float64), 32768, 32768, i, f, f, f, f, f, stream=Stream())
    with pytest.raises(TypeError):
        dasc.dasc_decay_attn(*args[:2], 32768.0, *args[3:], o=f, stream=Stream())
    with pytest.raises(ValueError):
        dasc.dasc_verify_draft(torch.zeros(3, 10), torch.zeros(2, 10), i[:2], i[:3], torch.zeros(2), torch.zeros(2), torch.zeros(2, 3, dtype=torch.int32), i[:2],
                               stream=Stream())  # a row short
    with pytest.raises(ValueError):
        dasc.dasc_verify_draft(torch.zeros(4, 10), torch.zeros(2, 9), i[:2], i[:3], torch.zeros(2), torch.zeros(2), torch.zeros(2, 3, dtype=torch.int32), i[:2],
                               stream=Stream())  # another vocabulary
