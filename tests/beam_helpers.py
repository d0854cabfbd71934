"""Beam search in 64 bits: the continuations of a selection, and the slots and states behind them."""
from __future__ import annotations

import numpy as np
import torch

import paper_2608_30386_b200 as dasc


def define(logits, scores, ended, end_token, n_out):
    """logits [R, W, V] (any float type), scores [R, W], ended [R, W] or None -> (scores, parent, token) [R, n_out] as numpy arrays."""
    x, s0 = logits.float().cpu().numpy().astype(np.float64), scores.cpu().numpy().astype(np.float64)
    R, W, V = x.shape
    out, parent, token = np.full((R, n_out), -np.inf), np.full((R, n_out), -1), np.full((R, n_out), -1)
    for r in range(R):
        found = []
        for b in range(W):
            if not np.isfinite(s0[r, b]):
                continue
            if ended is not None and ended[r][b]:
                found.append((np.array([s0[r, b]]), np.array([b]), np.array([0.0]), np.array([end_token])))
                continue
            v = np.nonzero(np.isfinite(x[r, b]))[0]
            if len(v) == 0:
                continue
            y = x[r, b, v]
            best = np.lexsort((v, -y))[:n_out]
            lse = y.max() + np.log(np.exp(y - y.max()).sum())
            found.append((s0[r, b] + (y[best] - lse), np.full(len(best), b), y[best], v[best]))
        if not found:
            continue
        total, beam, logit, v = (np.concatenate(z) for z in zip(*found))
        order = np.lexsort((v, -logit, beam, -total))[:n_out]
        n = len(order)
        out[r, :n], parent[r, :n], token[r, :n] = total[order], beam[order], v[order]
    return out, parent, token


def call(logits, scores, n_out, ended=None, end_token=-1, want_ended=False):
    R = scores.shape[0]
    out = torch.full((R, n_out), 9.0, device="cuda")
    parent, token, over = (torch.full((R, n_out), 99, dtype=torch.int32, device="cuda") for _ in range(3))
    e = None if ended is None else torch.tensor(ended, dtype=torch.int32, device="cuda")
    dasc.dasc_beam_select(logits, scores, out, parent, token, ended=e, out_ended=over if want_ended else None, end_token=end_token)
    torch.cuda.synchronize()
    return (out, parent, token) + ((over,) if want_ended else ())


def same(got, want, logits):
    """Beams and tokens are equal; scores are off by what the sum of V exponentials may be: each is good to 2^-21 (its rounded argument, below 32 for all
    that counts, 2^-20 of it where it is that far down; ex2 2^-22), sums in fp32 of at most 64 of them 2^-18 at most, and the result is rounded to fp32."""
    np.testing.assert_array_equal(got[1].cpu().numpy(), want[1])
    np.testing.assert_array_equal(got[2].cpu().numpy(), want[2])
    s, w = got[0].cpu().numpy().astype(np.float64), want[0]
    np.testing.assert_array_equal(np.isfinite(s), np.isfinite(w))
    m = np.isfinite(w)
    assert np.all(np.abs(s[m] - w[m]) <= 2.0 ** -17 + 2.0 ** -24 * np.abs(w[m]))


def assign(slots, parent):
    """One request's new slots and sources, as the header says."""
    W = len(slots)
    parent = [p if 0 <= p < W else -1 for p in parent]
    free, new, src, seen = [slots[b] for b in range(W) if b not in parent], [], [], set()
    for p in parent:
        src.append(slots[p] if p >= 0 else -1)
        if p >= 0 and p not in seen:
            seen.add(p)
            new.append(slots[p])
        else:
            new.append(free.pop(0))
    return new, src
