"""Plain form of decayed linear attention in 64 bits, token by token, and the bound that its terms set on rounding errors."""
from __future__ import annotations

from dataclasses import dataclass

import numpy as np
import torch

import paper_2608_30386_b200 as dasc


def reference(S, q, k, v, g, scale):
    """One head: S [dk, dv], q/k [T, dk], v [T, dv], g [T], all float64.  Returns (o [T, dv], S)."""
    o = torch.empty(k.shape[0], v.shape[1], dtype=torch.float64)
    for t in range(k.shape[0]):
        S = torch.exp(g[t]) * S + k[t][:, None] * v[t][None, :]
        o[t] = scale * (q[t] @ S)
    return o, S


@dataclass
class Case:
    L: int
    H_v: int
    H_k: int
    d_k: int
    d_v: int
    lens: list
    plan: object
    mask: np.ndarray         # [L][H_v], 1 = retained
    cu: torch.Tensor
    q: torch.Tensor
    k: torch.Tensor
    v: torch.Tensor
    g: torch.Tensor
    state: torch.Tensor      # [pool slots, L, H_v, d_k, d_v]
    req: torch.Tensor        # int32 [n_req]

    @property
    def T(self):
        return int(self.cu[-1])

    @property
    def strides(self):
        unit = self.d_k * self.d_v
        return self.H_v * unit, self.L * self.H_v * unit


def make_plan(L, H_v, H_k, d_k, d_v, seed=0, device=0):
    mask = np.random.default_rng(seed).integers(0, 2, (L, H_v)).astype(np.uint8)
    z = np.zeros(L * H_v, np.float32)
    return dasc.dasc_plan(dasc.GDN, L, H_v, H_k, d_k, d_v, z, z, sel=dasc.SEL_EXPLICIT, explicit_mask=mask, device=device), mask


def make_case(seed, lens, *, L=1, H_v=2, H_k=2, d_k=128, d_v=128, dtype=torch.bfloat16, decay="token", rate_lo=1e-4, rate_hi=3.0, device="cuda", spare=2):
    gen = torch.Generator().manual_seed(seed)
    plan, mask = make_plan(L, H_v, H_k, d_k, d_v, seed)
    T, R = sum(lens), len(lens)
    cu = torch.tensor([0, *lens]).cumsum(0).to(torch.int32)
    q, k = (torch.randn(L, T, H_k, d_k, generator=gen).div(d_k ** 0.5).to(dtype) for _ in range(2))
    v = torch.randn(L, T, H_v, d_v, generator=gen).to(dtype)
    rates = torch.exp(torch.empty(L, H_v).uniform_(float(np.log(rate_lo)), float(np.log(rate_hi)), generator=gen))
    g = -rates if decay == "head" else -rates[:, None] * torch.exp(0.7 * torch.randn(L, T, H_v, generator=gen))
    state = torch.randn(R + spare, L, H_v, d_k, d_v, generator=gen)
    req = torch.randperm(R + spare, generator=gen)[:R].to(torch.int32)
    return Case(L, H_v, H_k, d_k, d_v, list(lens), plan, mask, cu, *(x.contiguous().to(device) for x in (q, k, v, g, state, req)))


def run(case, *, mode=dasc.DECAY_CONTINUE, algo=dasc.ALGO_AUTO, used=None, zero=None, o_dtype=torch.float32, want_o=True, scale=0.7, req=None,
        state=None, layers=None, stream=None, longest=None, workspace=None):
    """(state after the call, o or None); o starts as a pattern that must survive where nothing is written."""
    dev = case.q.device
    lb, le = layers or (0, case.L)
    sl = slice(lb, le)
    state = case.state.clone() if state is None else state
    o = torch.full((le - lb, case.T, case.H_v, case.d_v), 7.0, device=dev, dtype=o_dtype) if want_o else None
    longest = max(case.lens, default=0) if longest is None else longest
    i32 = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device=dev)  # noqa: E731
    need = dasc.dasc_decay_workspace_bytes(case.plan, len(case.lens), le - lb, case.T, longest, algo)
    ws = workspace if workspace is not None else torch.randint(0, 255, (need,), dtype=torch.uint8, device=dev) if need else None
    g = case.g[sl]
    dasc.dasc_decay_attn(case.plan, state, *case.strides, case.req if req is None else i32(req), case.q[sl].contiguous(), case.k[sl].contiguous(),
                         case.v[sl].contiguous(), g.contiguous(), case.cu.to(dev), case.T, longest, seq_used=i32(used), from_zero=i32(zero),
                         decay=dasc.DECAY_PER_HEAD if g.dim() == 2 else dasc.DECAY_PER_TOKEN, layer_begin=lb, layer_end=le, q_scale=scale, o=o, mode=mode,
                         algo=algo, workspace=ws, stream=stream)
    torch.cuda.synchronize()
    assert dasc.dasc_decay_status(ws) == 0
    return state, o


def expected(case, *, mode=dasc.DECAY_CONTINUE, used=None, zero=None, scale=0.7, req=None, layers=None):
    """(state, o) of run(..., o_dtype=fp32) in 64 bits, and for each the sums of absolute terms that bound its rounding errors."""
    lb, le = layers or (0, case.L)
    req = case.req.tolist() if req is None else req
    state, o = case.state.cpu().double(), torch.full((le - lb, case.T, case.H_v, case.d_v), 7.0, dtype=torch.float64)
    state_abs, o_abs = torch.zeros_like(state), torch.zeros_like(o)
    q, k, v, g = (x.cpu().double() for x in (case.q, case.k, case.v, case.g))
    for r, n in enumerate(case.lens):
        if req[r] < 0:
            continue
        b = int(case.cu[r])
        n = n if used is None else min(n, max(used[r], 0))
        for layer in range(lb, le):
            for h in range(case.H_v):
                fresh = mode == dasc.DECAY_SCRATCH_MERGE_LOCAL or (zero is not None and zero[r] != 0)
                S0 = torch.zeros(case.d_k, case.d_v, dtype=torch.float64) if fresh else state[req[r], layer, h]
                kh = h // (case.H_v // case.H_k)
                gg = g[layer, h].expand(n) if g.dim() == 2 else g[layer, b:b + n, h]
                x = (q[layer, b:b + n, kh], k[layer, b:b + n, kh], v[layer, b:b + n, h])
                out, S = reference(S0, *x, gg, scale)
                out_abs, S_abs = reference(S0.abs(), *(y.abs() for y in x), gg, abs(scale))
                o[layer - lb, b:b + n, h], o_abs[layer - lb, b:b + n, h] = out, out_abs
                keep = mode == dasc.DECAY_SCORE or (mode == dasc.DECAY_SCRATCH_MERGE_LOCAL and case.mask[layer, h])
                if not keep:
                    state[req[r], layer, h], state_abs[req[r], layer, h] = S, S_abs
    return state, o, state_abs, o_abs


def unit_roundoff(case, chunked):
    """How far a computed sum may be off, relative to the sum of its terms' absolute values: (state, outputs).

    Token by token: each token multiplies by a rounded exponential (2 ulp, 2^-22 relative) and adds a rounded product (three
    roundings of 2^-24), the read-out sums d_k products: (T + 1) 2^-21 + d_k 2^-24.
    Chunks of 64 tokens: a value in n parts of bf16 is good to 2^-8n (a rounding of 8 bits of mantissa, spacing 2^-7, is off by half of that;
    what is left is rounded likewise).  Decayed values are in three parts, weights inside a chunk and the state on its way to the
    outputs in two (2^-16 each, one of them per term).  Sums of at most 192 terms per product on the tensor cores, each addition good to
    2^-23; factors from sums of log-decays (2^-24 of at most 16, or negligible terms) and ex2 (2^-22), one per chunk and one per term:
    400 * 2^-23 + 2^-20 (T / 64 + 1), and 2^-16 + 2^-16 for the outputs."""
    T = max(case.lens, default=0)
    if chunked:
        u = 400 * 2.0 ** -23 + 2.0 ** -20 * (T / 64 + 1)
        return u, u + 2 * 2.0 ** -16
    u = (T + 1) * 2.0 ** -21 + case.d_k * 2.0 ** -24
    return u, u


def check(case, got, want, chunked, o_dtype=torch.float32):
    (state, o), (rs, ro, sa, oa) = got, want
    us, uo = unit_roundoff(case, chunked)
    # 2^-126 and 2^-120: what ex2 and the tensor cores may flush, and sums of it
    err = (state.cpu().double() - rs).abs()
    assert bool((err <= us * sa + 2.0 ** -126).all()), f"state: {float((err / (sa + 1e-30)).max()):.3e} > {us:.3e}"
    if o is not None:
        half = torch.finfo(o_dtype).eps / 2
        if chunked and o_dtype == torch.bfloat16:
            # where outputs are rounded to bf16, weights and state are in one part on the way there: 2^-8 of each term
            uo = us + 2.0 ** -8
        err = (o.cpu().double() - ro).abs()
        bound = uo * oa + half * (ro.abs() + uo * oa) + 2.0 ** -120
        assert bool((err <= bound).all()), f"o: {float((err - bound).max()):.3e} over the bound"
