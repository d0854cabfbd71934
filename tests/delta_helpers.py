"""The gated delta rule in 64 bits, token by token, and the bound that its terms set on rounding errors of fp32 arithmetic."""
from __future__ import annotations

from dataclasses import dataclass

import numpy as np
import torch

import paper_2608_30386_b200 as dasc


def reference(S, q, k, v, g, beta, scale):
    """One head: S [dk, dv], q/k [T, dk], v [T, dv], g [T, dk] or [T], beta [T], all float64.  Returns (o [T, dv], S)."""
    o = torch.empty(k.shape[0], S.shape[1], dtype=torch.float64)
    for t in range(k.shape[0]):
        a = torch.exp(g[t])
        S = (a[:, None] if a.dim() else a) * S
        S = S + k[t][:, None] * (beta[t] * (v[t] - k[t] @ S))[None, :]
        o[t] = scale * (q[t] @ S)
    return o, S


def absolute(S, q, k, v, g, beta, scale):
    """The same sums with every term's absolute value."""
    o = torch.empty(k.shape[0], S.shape[1], dtype=torch.float64)
    S, q, k, v, beta = S.abs(), q.abs(), k.abs(), v.abs(), beta.abs()
    for t in range(k.shape[0]):
        a = torch.exp(g[t])
        S = (a[:, None] if a.dim() else a) * S
        S = S + k[t][:, None] * (beta[t] * (v[t] + k[t] @ S))[None, :]
        o[t] = abs(scale) * (q[t] @ S)
    return o, S


@dataclass
class Case:
    kind: int
    L: int
    H_v: int
    H_k: int
    d_k: int
    d_v: int
    lens: list
    plan: object
    cu: torch.Tensor
    q: torch.Tensor
    k: torch.Tensor
    v: torch.Tensor
    g: torch.Tensor
    beta: torch.Tensor
    state: torch.Tensor  # [slots, L, H_v, d_k, d_v]
    req: torch.Tensor    # int32 [n_req]

    @property
    def T(self):
        return int(self.cu[-1])

    @property
    def strides(self):
        unit = self.d_k * self.d_v
        return self.H_v * unit, self.L * self.H_v * unit


def make_plan(kind, L, H_v, H_k, d_k, d_v, device=0):
    n = L * H_v * (d_k if kind == dasc.KDA else 1)
    z = np.zeros(n, np.float32)
    return dasc.dasc_plan(kind, L, H_v, H_k, d_k, d_v, z, z, w_max=16.0, device=device)


def make_case(seed, lens, *, kind=dasc.KDA, L=1, H_v=2, H_k=2, d_k=128, d_v=128, dtype=torch.bfloat16, rate_lo=1e-3, rate_hi=2.0, device="cuda", spare=2):
    gen = torch.Generator().manual_seed(seed)
    T, R = sum(lens), len(lens)
    cu = torch.tensor([0, *lens]).cumsum(0).to(torch.int32)
    normal = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    q, k = ((lambda x: x / x.norm(dim=-1, keepdim=True))(normal(L, T, H_k, d_k)).to(dtype) for _ in range(2))
    v = normal(L, T, H_v, d_v).to(dtype)
    gates = (H_v, d_k) if kind == dasc.KDA else (H_v,)
    rates = torch.exp(torch.empty(L, *gates).uniform_(float(np.log(rate_lo)), float(np.log(rate_hi)), generator=gen))
    g = -torch.nn.functional.softplus(normal(L, T, *gates)) * rates[:, None]
    beta = torch.sigmoid(normal(L, T, H_v))
    state = normal(R + spare, L, H_v, d_k, d_v)
    req = torch.randperm(R + spare, generator=gen)[:R].to(torch.int32)
    return Case(kind, L, H_v, H_k, d_k, d_v, list(lens), make_plan(kind, L, H_v, H_k, d_k, d_v), cu,
                *(x.contiguous().to(device) for x in (q, k, v, g, beta, state, req)))


def i32(x, device="cuda"):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device=device)


def run(case, *, mode=dasc.DRAFT_ADVANCE, used=None, zero=None, o_dtype=torch.float32, want_o=True, scale=0.7, req=None, state=None, layers=None,
        stream=None):
    """(state after dasc_delta_draft, o or None); o starts as a pattern that must survive where nothing is written."""
    lb, le = layers or (0, case.L)
    sl = slice(lb, le)
    state = case.state.clone() if state is None else state
    o = torch.full((le - lb, case.T, case.H_v, case.d_v), 7.0, device="cuda", dtype=o_dtype) if want_o else None
    dasc.dasc_delta_draft(case.plan, state, *case.strides, case.req if req is None else i32(req), case.q[sl].contiguous() if want_o else None,
                          case.k[sl].contiguous(), case.v[sl].contiguous(), case.g[sl].contiguous(), case.beta[sl].contiguous(), case.cu.cuda(), case.T,
                          max(case.lens, default=0), seq_used=i32(used), from_zero=i32(zero), layer_begin=lb, layer_end=le, q_scale=scale, o=o, mode=mode,
                          stream=stream)
    torch.cuda.synchronize()
    return state, o


def step(case, *, o_dtype=torch.float32, scale=0.7, req=None, src=None, width=1, layers=None, state=None):
    """(state after dasc_delta_step, o): every request has one token."""
    lb, le = layers or (0, case.L)
    sl = slice(lb, le)
    state = case.state.clone() if state is None else state
    o = torch.full((le - lb, case.T, case.H_v, case.d_v), 7.0, device="cuda", dtype=o_dtype)
    dasc.dasc_delta_step(case.plan, state, *case.strides, case.req if req is None else i32(req), *(x[sl].contiguous() for x in
                         (case.q, case.k, case.v, case.g, case.beta)), o, src_idx=i32(src), beam_width=width, layer_begin=lb, layer_end=le, q_scale=scale)
    torch.cuda.synchronize()
    return state, o


def expected(case, *, score=False, used=None, zero=None, scale=0.7, req=None, src=None, layers=None):
    """(state, o) in 64 bits, and for each the sums of absolute terms that bound its rounding errors."""
    lb, le = layers or (0, case.L)
    req = case.req.tolist() if req is None else req
    old = case.state.cpu().double()
    state, o = old.clone(), torch.full((le - lb, case.T, case.H_v, case.d_v), 7.0, dtype=torch.float64)
    state_abs, o_abs = torch.zeros_like(state), torch.zeros_like(o)
    q, k, v, g, beta = (x.cpu().double() for x in (case.q, case.k, case.v, case.g, case.beta))
    for r, n in enumerate(case.lens):
        if req[r] < 0 or (src is not None and src[r] < 0):
            continue
        b = int(case.cu[r])
        n = n if used is None else min(n, max(used[r], 0))
        for layer in range(lb, le):
            for h in range(case.H_v):
                S0 = old[req[r] if src is None else src[r], layer, h]
                S0 = torch.zeros_like(S0) if zero is not None and zero[r] != 0 else S0
                kh = h // (case.H_v // case.H_k)
                x = (q[layer, b:b + n, kh], k[layer, b:b + n, kh], v[layer, b:b + n, h], g[layer, b:b + n, h], beta[layer, b:b + n, h])
                out, S = reference(S0, *x, scale)
                out_abs, S_abs = absolute(S0, *x, scale)
                o[layer - lb, b:b + n, h], o_abs[layer - lb, b:b + n, h] = out, out_abs
                if not score:
                    state[req[r], layer, h], state_abs[req[r], layer, h] = S, S_abs
    return state, o, state_abs, o_abs


def roundoff(case):
    """How far a computed sum may be off, relative to the sum of its terms' absolute values.  Along a token, a term passes an exponential and products of up to
    eight of them (good to 2^-22 and 2^-24 each: under 48 roundings of 2^-24 in all), and sums of d_k products, each of whose additions rounds once;
    sums over at most eight earlier tokens and the update of the state are among the 48.  An error made at a token passes the later ones as a
    term of theirs does, so they add up: (T + 1)(d_k + 48) 2^-24."""
    return (max(case.lens, default=0) + 1) * (case.d_k + 48) * 2.0 ** -24


def check(case, got, want, o_dtype=torch.float32):
    (state, o), (rs, ro, sa, oa) = got, want
    u = roundoff(case)
    err = (state.cpu().double() - rs).abs()
    assert bool((err <= u * sa + 2.0 ** -126).all()), f"state: {float((err / (sa + 1e-30)).max()):.3e} > {u:.3e}"
    if o is not None:
        half = torch.finfo(o_dtype).eps / 2
        err = (o.cpu().double() - ro).abs()
        bound = u * oa + half * (ro.abs() + u * oa) + 2.0 ** -120
        assert bool((err <= bound).all()), f"o: {float((err - bound).max()):.3e} over the bound"


def worst(got, want):
    """max |x - ref| / max |ref|, the library's own measure for fp32 inputs (bar 1e-5)."""
    return float((got.cpu().double() - want).abs().max() / want.abs().max())
