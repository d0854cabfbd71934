"""Decoding over the states of delta-rule layers: single tokens, drafted tokens, and beam search.

``step``     ``dasc_delta_step``: the gated delta rule for one token per request, in place on the pool; beams that continue the same state read it
             once and write their own.
``draft``    ``dasc_delta_draft``: drafted tokens scored (outputs only, the state stays), or the state advanced over those that stand.
``select``   ``dasc_beam_select``: the best continuations over beams and vocabulary, from logits.
``reorder``  ``dasc_beam_reorder``: every new beam gets a slot with the state of the beam it continues.

Shapes are those of the benchmark configurations: KDA with 32 heads, GDN with 32 value and 16 key heads, d_k = d_v = 128, bf16 token streams, fp32
states, one layer of a forward pass, a rank of a tensor-parallel group holding fewer heads; the tiny fp32 configuration has 4 heads of 64.
The states of all 24 layers are reordered at once.  Vocabularies and beam widths are generic, odd ones among them.
"""
import math
import random

import torch

own = False

DEVICE = "cuda"
RATE_LO = {"KDA": 1e-3, "GDN": 1e-4}  # decay rates are log-uniform from here to 1
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
MOST_STEP, MOST_DRAFT, MOST_LOGITS, MOST_COPY = 1.1e9, 5e8, 1.6e8, 3.3e9  # bytes of the largest listed calls


def _step(requests, width=1, kind="KDA", v_heads=32, dim=128, streams="bf16", layers=1):
    return {"op": "step", "requests": requests, "width": width, "kind": kind, "v_heads": v_heads, "k_heads": v_heads if kind == "KDA" else v_heads // 2,
            "dim": dim, "streams": streams, "layers": layers}


def _draft(requests, tokens, ragged, mode, kind="KDA", v_heads=32, dim=128, streams="bf16", layers=1):
    return {"op": "draft", "requests": requests, "tokens": tokens, "ragged": ragged, "mode": mode, "kind": kind, "v_heads": v_heads,
            "k_heads": v_heads if kind == "KDA" else v_heads // 2, "dim": dim, "streams": streams, "layers": layers}


def _select(requests, width, vocab, picks, logits="bf16", ended=0, masked=False):
    return {"op": "select", "requests": requests, "width": width, "vocab": vocab, "picks": picks, "logits": logits, "ended": ended, "masked": masked}


def _reorder(requests, width, dropped, layers=24, v_heads=32, conv=0):
    return {"op": "reorder", "requests": requests, "width": width, "dropped": dropped, "layers": layers, "v_heads": v_heads, "dim": 128, "conv": conv}


def listed():
    return [
        # decoding: a single request, a full batch, the head-wise kind with fewer requests
        {"name": "step_one", **_step(1)},
        {"name": "step_batch", **_step(256)},
        {"name": "step_gdn", **_step(37, kind="GDN")},
        # beam search: 32 requests of 8 beams, several of which continue the same one
        {"name": "step_beams", **_step(32, width=8)},
        # a batch scores its last token and four drafted ones; the states must stay
        {"name": "score_batch", **_draft(64, 5, False, "score")},
        # and is advanced over those that stand
        {"name": "advance_batch", **_draft(64, 5, False, "advance", kind="GDN")},
        # longer drafts of very different lengths, scored
        {"name": "score_ragged", **_draft(13, 12, True, "score", kind="GDN")},
        # one request of 4 beams; a batch over a large vocabulary with twice as many candidates as beams; an odd vocabulary in fp32, some beams ended
        {"name": "select_one", **_select(1, 4, 32000, 4)},
        {"name": "select_batch", **_select(64, 8, 131072, 16)},
        {"name": "select_odd", **_select(37, 5, 50257, 5, logits="fp32", ended=1, masked=True)},
        # states of all layers after a selection: one request, and a batch with convolution states beside them
        {"name": "reorder_one", **_reorder(1, 4, 1)},
        {"name": "reorder_batch", **_reorder(16, 4, 2, conv=24 * 9216)},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    x = rng.random()
    kind, heads = rng.choice(["KDA", "GDN"]), rng.choice([4, 8, 16, 32, 32])
    dim, streams = rng.choice([(128, "bf16")] * 5 + [(64, "fp32"), (128, "fp32")])
    if x < 0.25:
        width = rng.choice([1, 1, 1, rng.randint(2, 8)])
        return _shrink(_step(_log_uniform(rng, 1, 256 // width), width, kind, heads, dim, streams), MOST_STEP)
    if x < 0.5:
        ragged = rng.random() < 0.5
        return _shrink(_draft(_log_uniform(rng, 1, 64), rng.randint(2, 16 if ragged else 9), ragged, rng.choice(["score", "advance"]), kind, heads, dim, streams),
                       MOST_DRAFT)
    if x < 0.75:
        width = rng.randint(1, 16)
        return _shrink(_select(_log_uniform(rng, 1, 64), width, _log_uniform(rng, 2000, 160000), rng.choice([width, 2 * width]),
                               rng.choice(["bf16", "bf16", "fp32"]), rng.choice([0, 0, width // 4]), rng.random() < 0.3), MOST_LOGITS)
    width = rng.randint(2, 8)
    return _shrink(_reorder(_log_uniform(rng, 1, 16), width, rng.randint(1, width - 1), rng.choice([6, 12, 24]), heads, rng.choice([0, 24 * 9216])), MOST_COPY)


def _shrink(case, most):
    while case["requests"] > 1 and (work(case)["bytes"] > most or _held(case) > 4e9):
        case["requests"] = max(1, case["requests"] * 3 // 4)
    return case


def _held(case):
    """Bytes of the states that a case keeps."""
    if case["op"] == "select":
        return 0
    return case["requests"] * case.get("width", 1) * case["layers"] * case["v_heads"] * case["dim"] ** 2 * 4


def _lens(case):
    """Tokens of each request: fixed by the case."""
    if not case["ragged"]:
        return [case["tokens"]] * case["requests"]
    r = random.Random(case["requests"] * 1000003 + case["tokens"])
    return [r.randint(1, 2 * case["tokens"] - 1) for _ in range(case["requests"])]


def _sources(width):
    """How many beams of `width` are continued when each new beam takes one at random, on average."""
    return width * (1 - (1 - 1 / width) ** width)


def work(case):
    R = case["requests"]
    if case["op"] == "select":
        rows = R * (case["width"] - case["ended"])
        return {"bytes": rows * case["vocab"] * TYPES[case["logits"]].itemsize + R * (case["picks"] * 16 + case["width"] * 8), "flops": 3 * rows * case["vocab"]}
    L, H, d = case["layers"], case["v_heads"], case["dim"]
    if case["op"] == "reorder":
        return {"bytes": R * (case["dropped"] * 2 * (L * H * d * d * 4 + case["conv"]) + case["width"] * 16), "flops": 0}
    K, size = case["k_heads"], TYPES[case["streams"]].itemsize
    gates = d if case["kind"] == "KDA" else 1
    if case["op"] == "step":
        T, out, states = R * case["width"], True, R * (_sources(case["width"]) + case["width"])
    else:
        T, out, states = sum(_lens(case)), case["mode"] == "score", R * (1 if case["mode"] == "score" else 2)
        if not out:
            T = T // 2  # about half of the drafted tokens stand
    stream = T * L * ((2 if out else 1) * K * d * size + (2 if out else 1) * H * d * size + H * (gates + 1) * 4)
    return {"bytes": stream + states * L * H * d * d * 4, "flops": T * L * H * d * d * (7 if out else 5)}


# ---- inputs ------------------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    return {"step": _prepare_layers, "draft": _prepare_layers, "select": _prepare_select, "reorder": _prepare_reorder}[case["op"]](case, gen)


def _normal(gen, *shape):
    return torch.randn(*shape, device=DEVICE, generator=gen)


def _plan(case):
    import paper_2608_30386_b200 as dasc
    L, H, K, d = case["layers"], case["v_heads"], case.get("k_heads", case["v_heads"]), case["dim"]
    kda = case.get("kind", "KDA") == "KDA"
    n = L * H * (d if kda else 1)
    return dasc.dasc_plan(dasc.KDA if kda else dasc.GDN, L, H, K, d, d, torch.zeros(n), torch.zeros(n), sel=dasc.SEL_TOP_RATIO, keep_ratio=0.38)


def _prepare_layers(case, gen):
    L, H, K, d = case["layers"], case["v_heads"], case["k_heads"], case["dim"]
    t = TYPES[case["streams"]]
    gates = (H, d) if case["kind"] == "KDA" else (H,)
    lo = RATE_LO[case["kind"]]
    rates = torch.exp(torch.empty(L, *gates).uniform_(math.log(lo), 0.0, generator=torch.Generator().manual_seed(L * 977 + H))).to(DEVICE)
    R = case["requests"] * case.get("width", 1)
    s = {"case": case, "scale": d ** -0.5, "req": torch.randperm(R, generator=gen, device=DEVICE).to(torch.int32)}
    if case["op"] == "step":
        T = R
        s["src"] = None
        if case["width"] > 1:  # what a selection and the slots' assignment left: new slots, and where each beam's state is
            parent = torch.randint(0, case["width"], (case["requests"], case["width"]), generator=gen, device=DEVICE).to(torch.int32)
            s["req"], s["src"] = (x.flatten() for x in _assign(s["req"].view(case["requests"], -1), parent))
    else:
        lens = _lens(case)
        T = sum(lens)
        s["T"], s["longest"] = T, max(lens)
        s["cu"] = torch.tensor([0] + lens).cumsum(0).to(torch.int32).to(DEVICE)
        s["used"] = None
        if case["mode"] == "advance":  # one more than the drafted tokens that stood
            s["used"] = (torch.rand(R, device=DEVICE, generator=gen) * torch.tensor(lens, device=DEVICE)).to(torch.int32) + 1
    s["state"] = _normal(gen, R, L, H, d, d) * 0.3
    s["q"], s["k"] = ((lambda x: x / x.norm(dim=-1, keepdim=True))(_normal(gen, L, T, K, d)).to(t) for _ in range(2))
    s["v"] = _normal(gen, L, T, H, d).to(t)
    s["g"] = -torch.nn.functional.softplus(_normal(gen, L, T, *gates)) * rates[:, None]
    s["beta"] = torch.sigmoid(_normal(gen, L, T, H))
    want = case["op"] == "step" or case["mode"] == "score"
    s["o"] = torch.zeros(L, T, H, d, device=DEVICE, dtype=t) if want else None
    if own:
        s["plan"] = _plan(case)
    return s


def _prepare_select(case, gen):
    R, W, V = case["requests"], case["width"], case["vocab"]
    # beams of a request agree in most of what they expect
    x = 2.2 * _normal(gen, R, 1, V) + 1.2 * _normal(gen, R, W, V)
    if case["masked"]:  # tokens that a grammar or a list of bad words leaves out
        x = torch.where(torch.rand(R, 1, V, device=DEVICE, generator=gen) < 0.3, -torch.inf, x)
    ended = torch.rand(R, W, device=DEVICE, generator=gen).argsort(-1) < case["ended"]
    return {"case": case, "logits": x.to(TYPES[case["logits"]]), "scores": -12.0 + 1.5 * _normal(gen, R, W), "ended": ended.to(torch.int32), "end_token": 2,
            "out_scores": torch.zeros(R, case["picks"], device=DEVICE),
            **{k: torch.zeros(R, case["picks"], device=DEVICE, dtype=torch.int32) for k in ("parent", "token", "out_ended")}}


def _prepare_reorder(case, gen):
    R, W, L, H, d = case["requests"], case["width"], case["layers"], case["v_heads"], case["dim"]
    # `dropped` beams of each request end, others are continued in their place
    order = torch.rand(R, W, device=DEVICE, generator=gen).argsort(-1)
    alive = W - case["dropped"]
    again = torch.randint(0, alive, (R, case["dropped"]), device=DEVICE, generator=gen)
    parent = torch.cat([order[:, :alive], order.gather(1, again)], 1)
    parent = parent.gather(1, torch.rand(R, W, device=DEVICE, generator=gen).argsort(-1)).to(torch.int32).contiguous()
    s = {"case": case, "parent": parent, "req": torch.randperm(R * W, generator=gen, device=DEVICE).to(torch.int32).view(R, W),
         "state": _normal(gen, R * W, L, H, d, d), "conv": None, "new": torch.zeros(R, W, dtype=torch.int32, device=DEVICE),
         "src": torch.zeros(R, W, dtype=torch.int32, device=DEVICE)}
    if case["conv"]:
        s["conv"] = torch.randint(-32768, 32767, (R * W, case["conv"] // 2), generator=gen, device=DEVICE, dtype=torch.int16)
    if own:
        s["plan"] = _plan(case)
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------------------

def run(s):
    case = s["case"]
    return {"step": _run_step, "draft": _run_draft, "select": _run_select, "reorder": _run_reorder}[case["op"]](s, case)


def _strides(case):
    unit = case["dim"] * case["dim"]
    return case["v_heads"] * unit, case["layers"] * case["v_heads"] * unit


def _token(S, q, k, v, g, beta, scale):
    """One token of every request: S [L, R, H, d, d], the rest in fp32 with H heads."""
    S = (g.exp() if g.dim() == 4 else g.exp()[..., None])[..., None] * S
    u = beta[..., None] * (v - (k[..., None, :] @ S)[..., 0, :])
    S = S + k[..., :, None] * u[..., None, :]
    return S, (q[..., None, :] @ S)[..., 0, :] * scale


def _streams(s, case):
    share = case["v_heads"] // case["k_heads"]
    return [s[x].float().repeat_interleave(share, dim=2) for x in ("q", "k")] + [s["v"].float(), s["g"], s["beta"]]


def _run_step(s, case):
    if own:
        import paper_2608_30386_b200 as dasc
        dasc.dasc_delta_step(s["plan"], s["state"], *_strides(case), s["req"], s["q"], s["k"], s["v"], s["g"], s["beta"], s["o"], src_idx=s["src"],
                             beam_width=case["width"], q_scale=s["scale"])
    else:
        S = s["state"][(s["req"] if s["src"] is None else s["src"]).long()].transpose(0, 1)
        S, o = _token(S, *_streams(s, case), s["scale"])
        s["o"].copy_(o)
        s["state"].index_copy_(0, s["req"].long(), S.transpose(0, 1).contiguous())
    return {"o": s["o"], "state": s["state"]}


def _run_draft(s, case):
    score = case["mode"] == "score"
    if own:
        import paper_2608_30386_b200 as dasc
        dasc.dasc_delta_draft(s["plan"], s["state"], *_strides(case), s["req"], s["q"], s["k"], s["v"], s["g"], s["beta"], s["cu"], s["T"], s["longest"],
                              seq_used=s["used"], q_scale=s["scale"], o=s["o"], mode=dasc.DRAFT_SCORE if score else dasc.DRAFT_ADVANCE)
    else:
        cu = s["cu"].long()
        n = cu[1:] - cu[:-1]
        if s["used"] is not None:
            n = torch.minimum(n, s["used"].long())
        S = s["state"][s["req"].long()].transpose(0, 1)
        streams, outs = _streams(s, case), []
        for t in range(s["longest"]):
            at = (cu[:-1] + t).clamp(max=s["T"] - 1)
            new, o = _token(S, *(x[:, at] for x in streams), s["scale"])
            S = torch.where((t < n)[None, :, None, None, None], new, S)
            outs.append(o)
        if score:
            t = torch.arange(s["T"], device=DEVICE)
            r = torch.searchsorted(cu, t, right=True) - 1
            s["o"].copy_(torch.stack(outs, 2)[:, r, t - cu[r]])
        else:
            s["state"].index_copy_(0, s["req"].long(), S.transpose(0, 1).contiguous())
    return {"o": s["o"]} if score else {"state": s["state"]}


def _run_select(s, case):
    if own:
        import paper_2608_30386_b200 as dasc
        dasc.dasc_beam_select(s["logits"], s["scores"], s["out_scores"], s["parent"], s["token"], ended=s["ended"], out_ended=s["out_ended"],
                              end_token=s["end_token"])
    else:
        x = s["logits"].double()  # (sums over the vocabulary, and candidates next to one another)
        top = x.amax(-1, keepdim=True)
        total = s["scores"].double()[..., None] + (x - (top + (x - top).exp().sum(-1, keepdim=True).log()))
        at_end = torch.arange(case["vocab"], device=DEVICE) == s["end_token"]
        over = s["ended"][..., None] != 0
        total = torch.where(over, torch.where(at_end, s["scores"].double()[..., None], -torch.inf), total).flatten(1)
        for i in range(case["picks"]):  # the lowest index of equal ones first
            best = total.argmax(1, keepdim=True)
            s["out_scores"][:, i:i + 1] = total.gather(1, best)
            s["parent"][:, i:i + 1] = best // case["vocab"]
            s["token"][:, i:i + 1] = best % case["vocab"]
            total.scatter_(1, best, -torch.inf)
        s["out_ended"].copy_((s["ended"].gather(1, s["parent"].long()) != 0) | (s["token"] == s["end_token"]))
    return {"scores": s["out_scores"], "parent": s["parent"], "token": s["token"], "ended": s["out_ended"]}


def _assign(req, parent):
    """The first new beam of each continued one keeps its slot, the others get the slots of beams that nobody continues, both in ascending order.
    Returns the new beams' slots and the slots their states are in; [R, W] each."""
    W = parent.shape[1]
    same = parent[:, :, None] == parent[:, None, :]
    first = ~(same & torch.ones(W, W, device=parent.device, dtype=torch.bool).tril(-1)).any(-1)
    continued = (parent[:, None, :] == torch.arange(W, device=parent.device)[None, :, None]).any(-1)  # [R, old beam]
    free = continued.int().argsort(dim=1, stable=True)  # those that nobody continues, then the others
    src = req.gather(1, parent.long())
    turn = (~first).int().cumsum(1) - 1
    return torch.where(first, src, req.gather(1, free.gather(1, turn.clamp(min=0).long()))), src


def _run_reorder(s, case):
    if own:
        import paper_2608_30386_b200 as dasc
        dasc.dasc_beam_reorder(s["plan"], s["state"], *_strides(case), s["req"], s["parent"], s["new"], src_idx=s["src"], conv=s["conv"])
    else:
        new, src = _assign(s["req"], s["parent"])
        s["new"].copy_(new)
        s["src"].copy_(src)
        moved = (new != src).flatten().nonzero()[:, 0]
        to, of = new.flatten()[moved].long(), src.flatten()[moved].long()
        s["state"].index_copy_(0, to, s["state"][of])
        if s["conv"] is not None:
            s["conv"].index_copy_(0, to, s["conv"][of])
    return {"new": s["new"], "src": s["src"], "state": s["state"], **({"conv": s["conv"]} if s["conv"] is not None else {})}


# ---- the definition in 64 bits -----------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"step": _exact_step, "draft": _exact_draft, "select": _exact_select, "reorder": _exact_reorder}[case["op"]](s, case)


def _recur(S, q, k, v, g, beta, scale):
    """Tokens of one request and layer in 64 bits, one behind the other, each as S <- (I - beta k k^T) Diag(alpha) S + beta k v^T; heads side by side."""
    H, d = v.shape[1], v.shape[2]
    heads = torch.arange(H, device=DEVICE) // (H // k.shape[1])
    eye, outs = torch.eye(d, device=DEVICE, dtype=torch.float64), []
    for t in range(v.shape[0]):
        key, b = k[t].double()[heads], beta[t].double()[:, None, None]
        alpha = g[t].double().exp()
        alpha = alpha[:, None, None] if alpha.dim() == 1 else alpha[:, :, None]
        S = torch.bmm(eye - b * torch.einsum("hi,hj->hij", key, key), alpha * S) + b * torch.einsum("hi,hj->hij", key, v[t].double())
        outs.append(scale * torch.einsum("hij,hi->hj", S, q[t].double()[heads]))
    return S, outs


def _exact_step(s, case):
    src = (s["req"] if s["src"] is None else s["src"]).tolist()
    old, state, o = s["state"].double(), s["state"].double(), s["o"].double()
    for i, r in enumerate(s["req"].tolist()):
        for layer in range(case["layers"]):
            S, out = _recur(old[src[i], layer], *(s[x][layer, i:i + 1] for x in ("q", "k", "v", "g", "beta")), s["scale"])
            state[r, layer], o[layer, i] = S, out[0]
    return {"o": o, "state": state}


def _exact_draft(s, case):
    cu, req = s["cu"].tolist(), s["req"].tolist()
    used = None if s["used"] is None else s["used"].tolist()
    score = case["mode"] == "score"
    result = s["o"].double() if score else s["state"].double()
    for r, slot in enumerate(req):
        b, e = cu[r], cu[r + 1]
        if used is not None:
            e = min(e, b + used[r])
        for layer in range(case["layers"]):
            S, outs = _recur(s["state"][slot, layer].double(), *(s[x][layer, b:e] for x in ("q", "k", "v", "g", "beta")), s["scale"])
            if score:
                result[layer, b:e] = torch.stack(outs)
            else:
                result[slot, layer] = S
    return {"o": result} if score else {"state": result}


def _exact_select(s, case):
    W, V, n = case["width"], case["vocab"], case["picks"]
    scores, parent, token, ended = (torch.zeros_like(s[x]) for x in ("out_scores", "parent", "token", "out_ended"))
    scores = scores.double()
    for r in range(case["requests"]):
        x = s["logits"][r].double()
        total = s["scores"][r].double()[:, None] + x - torch.logsumexp(x, 1, keepdim=True)
        for b in range(W):
            if s["ended"][r, b]:
                total[b] = -torch.inf
                total[b, s["end_token"]] = s["scores"][r, b].double()
        value, at = torch.sort(total.flatten(), descending=True, stable=True)
        scores[r], parent[r], token[r] = value[:n], at[:n] // V, at[:n] % V
        ended[r] = (s["ended"][r][parent[r].long()] != 0) | (token[r] == s["end_token"])
    return {"scores": scores, "parent": parent, "token": token, "ended": ended}


def _exact_reorder(s, case):
    new, src, state = s["new"].clone(), s["src"].clone(), s["state"].clone()
    conv = None if s["conv"] is None else s["conv"].clone()
    for r in range(case["requests"]):
        slots, parents = s["req"][r].tolist(), s["parent"][r].tolist()
        free, taken = [slots[b] for b in range(case["width"]) if b not in parents], set()
        for i, p in enumerate(parents):
            src[r, i] = slots[p]
            new[r, i] = free.pop(0) if p in taken else slots[p]
            if p in taken:
                state[new[r, i]] = s["state"][slots[p]]
                if conv is not None:
                    conv[new[r, i]] = s["conv"][slots[p]]
            taken.add(p)
    return {"new": new, "src": src, "state": state, **({"conv": conv} if conv is not None else {})}
