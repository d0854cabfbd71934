"""Linear attention with a decay per head over the active-state pool, and the verification of drafted tokens.

``attn``    ``dasc_decay_attn``: the chunked form for prompts (state read, advanced and written back, outputs of every token); scoring of drafted tokens
            (outputs only, the state stays); the advance over the tokens that stand (no outputs, per-request token counts on the GPU).
``step``    ``dasc_decay_step``: one token per request, in place on the pool.
``verify``  ``dasc_verify_draft``: how many drafted tokens of each request stand, and its next token.

Shapes are those of the benchmark configurations: 32 value heads with 32 or 16 key heads, d_k = d_v = 128, bf16 token streams, fp32 states, one layer
of a forward pass or a group of layers, a rank of a tensor-parallel group holding fewer heads; the tiny fp32 configuration has 4 heads of 64.
Vocabularies are generic, odd ones among them.
"""
import math
import random

import torch

own = False

DEVICE = "cuda"
CHUNK = 64                            # tokens per chunk of the plain form
RATE_LO, RATE_HI = 1e-4, 1.0          # decay rates per token of the heads, log-uniform
MOST_BYTES = 1.2e9                    # what the largest listed case moves
MOST_PADDED = 64 * 4 * 256 * 32       # token-heads of the plain form, padded to the longest request
CONTINUE, MERGE, SCORE = 0, 1, 2      # modes of dasc_decay_attn
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _attn(requests, tokens, ragged, layers=1, v_heads=32, k_heads=32, dim=128, streams="bf16", mode="continue", out=True, used=False, decay="token",
          fresh=False):
    return {"op": "attn", "requests": requests, "tokens": tokens, "ragged": ragged, "layers": layers, "v_heads": v_heads, "k_heads": k_heads, "dim": dim,
            "streams": streams, "mode": mode, "out": out, "used": used, "decay": decay, "fresh": fresh}


def _step(requests, layers=1, v_heads=32, k_heads=32, dim=128, streams="bf16", decay="token"):
    return {"op": "step", "requests": requests, "layers": layers, "v_heads": v_heads, "k_heads": k_heads, "dim": dim, "streams": streams, "decay": decay}


def _verify(requests, drafts, vocab, ragged, q=True, probs="fp32"):
    return {"op": "verify", "requests": requests, "drafts": drafts, "vocab": vocab, "ragged": ragged, "q": q, "probs": probs}


def listed():
    return [
        # one prompt on its own, a length that is no multiple of a chunk: latency, one layer of the forward pass
        {"name": "prompt_one", **_attn(1, 509, False, fresh=True)},
        # one long prompt: few heads for the whole GPU
        {"name": "prompt_long", **_attn(1, 32768, False, fresh=True)},
        # a batch over a group of layers with shared key heads, continuing from restored states
        {"name": "prompt_batch", **_attn(64, 256, False, layers=4, k_heads=16)},
        # mixed serving trace: prompts of 1 .. 1023 tokens, a constant decay per head
        {"name": "prompt_ragged", **_attn(64, 512, True, decay="head")},
        # the tiny fp32 configuration
        {"name": "prompt_fp32_tiny", **_attn(1, 64, False, v_heads=4, k_heads=4, dim=64, streams="fp32")},
        # a batch scores its last token and four drafted ones; the states must stay
        {"name": "score_batch", **_attn(64, 5, False, mode="score")},
        # and is advanced over those that stand
        {"name": "advance_batch", **_attn(64, 5, False, out=False, used=True)},
        # decoding: a single request, and a full batch
        {"name": "step_one", **_step(1)},
        {"name": "step_batch", **_step(256)},
        # verification for one request, a small vocabulary; a batch over a large one; a drafter without probabilities, bf16 rows of an odd vocabulary
        {"name": "verify_one", **_verify(1, 4, 32000, False)},
        {"name": "verify_batch", **_verify(64, 8, 131072, True)},
        {"name": "verify_lookup", **_verify(37, 5, 50257, True, q=False, probs="bf16")},
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.random()
    heads = rng.choice([4, 8, 16, 32, 32])
    k_heads = rng.choice([heads, heads, heads // 2])
    decay = rng.choice(["token", "token", "head"])
    if kind < 0.25:
        case = _verify(_log_uniform(rng, 1, 128), rng.randint(1, 8), _log_uniform(rng, 2000, 160000), rng.random() < 0.5, rng.random() < 0.7,
                       rng.choice(["fp32", "fp32", "bf16"]))
        while work(case)["bytes"] > MOST_BYTES or case["requests"] * (case["drafts"] + 1) * case["vocab"] > 2e8:
            case["requests"] = max(1, case["requests"] * 3 // 4)
        return case
    if kind < 0.5:
        return _step(_log_uniform(rng, 1, 256), 1, heads, k_heads, *rng.choice([(128, "bf16")] * 4 + [(64, "fp32"), (128, "fp32")]), decay=decay)
    if kind < 0.65:  # drafted tokens: scored, or the state advanced over those that stand
        score = rng.random() < 0.5
        return _attn(_log_uniform(rng, 1, 64), rng.randint(2, 9), False, 1, heads, k_heads, mode="score" if score else "continue", out=score,
                     used=not score, decay=decay)
    if kind < 0.75:  # fp32 streams: small models and checks
        return _attn(_log_uniform(rng, 1, 8), _log_uniform(rng, 16, 256), rng.random() < 0.5, 1, rng.choice([4, 8]), 4, rng.choice([64, 128]), "fp32",
                     decay=decay)
    case = _attn(_log_uniform(rng, 1, 64), _log_uniform(rng, 5, 8192), rng.random() < 0.6, rng.choice([1, 1, 2, 4]), heads, k_heads,
                 mode=rng.choice(["continue", "continue", "merge"]), decay=decay, fresh=rng.random() < 0.3)
    while work(case)["bytes"] > MOST_BYTES or case["requests"] * case["layers"] * heads * max(_lens(case)) > MOST_PADDED:
        if case["requests"] > 1:
            case["requests"] = case["requests"] * 3 // 4
        else:
            case["tokens"] //= 2
    return case


def _lens(case):
    """Tokens of each request: fixed by the case."""
    if not case["ragged"]:
        return [case["tokens"]] * case["requests"]
    r = random.Random(case["requests"] * 1000003 + case["tokens"])
    return [r.randint(1, 2 * case["tokens"] - 1) for _ in range(case["requests"])]


def _drafts(case):
    if not case["ragged"]:
        return [case["drafts"]] * case["requests"]
    r = random.Random(case["requests"] * 1000003 + case["drafts"])
    return [r.randint(1, case["drafts"]) for _ in range(case["requests"])]


def work(case):
    if case["op"] == "verify":
        size = 2 if case["probs"] == "bf16" else 4
        n = sum(_drafts(case))
        # one row of the target per request, and one of the drafter, since most requests reject somewhere; a probability or two per drafted token
        rows = case["requests"] * (2 if case["q"] else 1)
        return {"bytes": rows * case["vocab"] * size + n * (8 + 2 * size) + case["requests"] * 12 + (n + case["requests"]) * 4,
                "flops": rows * case["vocab"] * 2}
    size = 2 if case["streams"] == "bf16" else 4
    L, H, K, d, R = case["layers"], case["v_heads"], case["k_heads"], case["dim"], case["requests"]
    T = R if case["op"] == "step" else sum(_lens(case))
    out = case.get("out", True)
    if case.get("used"):
        T = T // 2  # about half of the drafted tokens stand
    stream = T * L * ((2 if out else 1) * K * d + (2 if out else 1) * H * d) * size + (T if case["decay"] == "token" else 1) * L * H * 4
    mode = case.get("mode", "continue")
    reads = 0 if case.get("fresh") or mode == "merge" else 1
    writes = 0 if mode == "score" else 0.5 if mode == "merge" else 1
    return {"bytes": stream + (reads + writes) * R * L * H * d * d * 4, "flops": T * L * H * d * d * (5 if out else 3)}


# ---- inputs ------------------------------------------------------------------------------------------------------------------

def _plan_inputs(case, gen):
    L, H = case["layers"], case["v_heads"]
    rates = torch.exp(torch.empty(L, H).uniform_(math.log(RATE_LO), math.log(RATE_HI), generator=torch.Generator().manual_seed(L * 977 + H)))
    return rates.to(DEVICE)


def _streams(case, T, gen, rates):
    L, H, K, d = case["layers"], case["v_heads"], case["k_heads"], case["dim"]
    t = TYPES[case["streams"]]
    normal = lambda *s: torch.randn(*s, device=DEVICE, generator=gen)  # noqa: E731
    q, k = ((lambda x: x / x.norm(dim=-1, keepdim=True))(normal(L, T, K, d)).to(t) for _ in range(2))
    v = normal(L, T, H, d).to(t)
    if case["decay"] == "head":
        g = -rates
    else:
        g = -rates[:, None] * torch.exp(0.5 * normal(L, T, H))  # rates that the tokens modulate
    return q, k, v, g.contiguous()


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    if case["op"] == "verify":
        return _prepare_verify(case, gen)
    L, H, K, d, R = case["layers"], case["v_heads"], case["k_heads"], case["dim"], case["requests"]
    rates = _plan_inputs(case, gen)
    s = {"case": case, "scale": d ** -0.5, "req": torch.randperm(R, generator=gen, device=DEVICE).to(torch.int32)}
    s["state"] = torch.randn(R, L, H, d, d, device=DEVICE, generator=gen) * 0.3
    # half of the heads, those that forget most slowly, are kept in checkpoints: what the merge mode leaves alone
    s["keep"] = (rates < rates.median(dim=1, keepdim=True).values)
    if case["op"] == "step":
        s["q"], s["k"], s["v"], s["g"] = _streams(case, R, gen, rates)
        s["o"] = torch.zeros(L, R, H, d, device=DEVICE, dtype=TYPES[case["streams"]])
    else:
        lens = _lens(case)
        T = sum(lens)
        s["T"], s["longest"] = T, max(lens)
        s["cu"] = torch.tensor([0] + lens).cumsum(0).to(torch.int32).to(DEVICE)
        s["q"], s["k"], s["v"], s["g"] = _streams(case, T, gen, rates)
        s["o"] = torch.zeros(L, T, H, d, device=DEVICE, dtype=TYPES[case["streams"]]) if case["out"] else None
        s["used"] = None
        if case["used"]:
            s["used"] = (torch.rand(R, device=DEVICE, generator=gen) * torch.tensor(lens, device=DEVICE)).to(torch.int32) + 1
        s["zero"] = torch.ones(R, dtype=torch.int32, device=DEVICE) if case["fresh"] else None
    if own:
        import paper_2608_30386_b200 as dasc
        mask = s["keep"].cpu().numpy()
        s["plan"] = dasc.dasc_plan(dasc.GDN, L, H, K, d, d, torch.zeros(L, H), torch.zeros(L, H), sel=dasc.SEL_EXPLICIT, explicit_mask=mask)
        if case["op"] == "attn":
            need = dasc.dasc_decay_workspace_bytes(s["plan"], R, L, s["T"], s["longest"])
            s["ws"] = torch.empty(need, dtype=torch.uint8, device=DEVICE) if need else None
    return s


def _prepare_verify(case, gen):
    R, V, n = case["requests"], case["vocab"], _drafts(case)
    N, t = sum(n), TYPES[case["probs"]]
    cu = torch.tensor([0] + n).cumsum(0).to(torch.int32).to(DEVICE)
    logits = torch.randn(N + R, V, device=DEVICE, generator=gen) * 2.5
    target = torch.softmax(logits, -1)
    at = torch.arange(N, device=DEVICE) + torch.repeat_interleave(torch.arange(R, device=DEVICE), torch.tensor(n, device=DEVICE), output_size=N)
    # the drafter: the target's logits with noise, its tokens drawn from its own probabilities
    draft = torch.softmax(logits[at] + torch.randn(N, V, device=DEVICE, generator=gen), -1)
    pick = torch.rand(N, 1, device=DEVICE, generator=gen, dtype=torch.float64)
    tokens = (draft.double().cumsum(-1) <= pick * draft.double().sum(-1, keepdim=True)).sum(-1).clamp(max=V - 1).to(torch.int32)
    return {"case": case, "cu": cu, "target": target.to(t), "draft": draft.to(t) if case["q"] else None, "tokens": tokens, "most": case["drafts"],
            "u": torch.rand(N, device=DEVICE, generator=gen), "u_next": torch.rand(R, device=DEVICE, generator=gen),
            "out": torch.zeros(R, case["drafts"] + 1, dtype=torch.int32, device=DEVICE), "kept": torch.zeros(R, dtype=torch.int32, device=DEVICE)}


# ---- one pass ----------------------------------------------------------------------------------------------------------------

def run(s):
    case = s["case"]
    return {"attn": _run_attn, "step": _run_step, "verify": _run_verify}[case["op"]](s, case)


def _strides(case):
    unit = case["dim"] * case["dim"]
    return case["v_heads"] * unit, case["layers"] * case["v_heads"] * unit


def _run_attn(s, case):
    mode = {"continue": CONTINUE, "merge": MERGE, "score": SCORE}[case["mode"]]
    if own:
        import paper_2608_30386_b200 as dasc
        dasc.dasc_decay_attn(s["plan"], s["state"], *_strides(case), s["req"], s["q"], s["k"], s["v"], s["g"], s["cu"], s["T"], s["longest"],
                             seq_used=s["used"], from_zero=s["zero"], q_scale=s["scale"], o=s["o"], mode=mode,
                             decay=dasc.DECAY_PER_HEAD if case["decay"] == "head" else dasc.DECAY_PER_TOKEN, workspace=s["ws"])
    else:
        _plain_attn(s, case, mode)
    return {k: s[k] for k in (["o"] if case["out"] else []) + (["state"] if mode != SCORE else [])}


def _plain_attn(s, case, mode):
    """Chunks of CHUNK tokens of every request at once: products inside a chunk, each chunk's own contribution to the state, and the states at the
    chunks' starts as sums of decayed contributions.  Sums of log-decays and their differences in 64 bits, the rest in 32."""
    L, R, H, K, d = case["layers"], case["requests"], case["v_heads"], case["k_heads"], case["dim"]
    cu, T = s["cu"].long(), s["T"]
    n = cu[1:] - cu[:-1]
    if s["used"] is not None:
        n = torch.minimum(n, s["used"].long())
    C = CHUNK if s["longest"] > 16 else 16
    N = -(-s["longest"] // C)
    place = torch.arange(N * C, device=DEVICE)
    valid = place < n[:, None]
    idx = (cu[:-1, None] + place).clamp(max=T - 1)

    def chunks(x, heads):  # [L, T, heads, e] -> [L, R, H, N, C, e]
        x = torch.where(valid[None, :, :, None, None], x[:, idx].float(), 0.0)
        if heads != H:
            x = x.repeat_interleave(H // heads, dim=3)
        return x.view(L, R, N, C, H, -1).permute(0, 1, 4, 2, 3, 5)

    k, v = chunks(s["k"], K), chunks(s["v"], H)
    g = s["g"].double()
    g = g[:, None].expand(L, T, H) if case["decay"] == "head" else g
    G = torch.where(valid[None, :, :, None], g[:, idx], 0.0).view(L, R, N, C, H).permute(0, 1, 4, 2, 3).cumsum(-1)  # [L, R, H, N, C]
    end = G[..., -1:]
    own_part = (k * torch.exp(end - G).float()[..., None]).transpose(-1, -2) @ v  # [L, R, H, N, d, d]
    E = torch.cat([torch.zeros_like(end[..., 0][..., :1]), end[..., 0].cumsum(-1)], -1)  # log-decay up to the start of chunk 0 .. N
    before = torch.ones(N + 1, N, device=DEVICE, dtype=torch.bool).tril(-1)
    share = torch.where(before, E[..., :, None] - E[..., None, 1:], -torch.inf).exp().float()  # [L, R, H, N + 1, N]
    start = (share @ own_part.reshape(L, R, H, N, d * d)).view(L, R, H, N + 1, d, d)
    if mode != MERGE and s["zero"] is None:
        first = s["state"][s["req"].long()].transpose(0, 1)  # [L, R, H, d, d]
        start = start + E.exp().float()[..., None, None] * first[:, :, :, None]
    if s["o"] is not None:
        q = chunks(s["q"], K)
        inside = torch.ones(C, C, device=DEVICE, dtype=torch.bool).tril()
        p = (q @ k.transpose(-1, -2)) * torch.where(inside, G[..., :, None] - G[..., None, :], -torch.inf).exp().float()
        o = p @ v + (q * G.exp().float()[..., None]) @ start[..., :N, :, :]
        o = (o * s["scale"]).permute(0, 1, 3, 4, 2, 5).reshape(L, R, N * C, H, d)
        t = torch.arange(T, device=DEVICE)
        r = torch.searchsorted(cu, t, right=True) - 1
        at = t - cu[r]
        s["o"].copy_(torch.where((at < n[r])[None, :, None, None], o[:, r, at].to(s["o"].dtype), s["o"]))
    if mode != SCORE:
        last = start[..., N, :, :]
        if mode == MERGE:
            last = torch.where(s["keep"][:, None, :, None, None], s["state"][s["req"].long()].transpose(0, 1), last)
        s["state"].index_copy_(0, s["req"].long(), last.transpose(0, 1).contiguous())


def _run_step(s, case):
    if own:
        import paper_2608_30386_b200 as dasc
        dasc.dasc_decay_step(s["plan"], s["state"], *_strides(case), s["req"], s["q"], s["k"], s["v"], s["g"], s["o"], q_scale=s["scale"],
                             decay=dasc.DECAY_PER_HEAD if case["decay"] == "head" else dasc.DECAY_PER_TOKEN)
    else:
        share = case["v_heads"] // case["k_heads"]
        q, k = (s[x].float().repeat_interleave(share, dim=2) for x in ("q", "k"))
        a = s["g"].exp() if case["decay"] == "token" else s["g"].exp()[:, None]
        S = s["state"][s["req"].long()].transpose(0, 1)  # [L, R, H, d, d]
        S = a[..., None, None] * S + k[..., :, None] * s["v"].float()[..., None, :]
        s["o"].copy_((q[..., None, :] @ S)[..., 0, :] * s["scale"])
        s["state"].index_copy_(0, s["req"].long(), S.transpose(0, 1).contiguous())
    return {"o": s["o"], "state": s["state"]}


def _run_verify(s, case):
    if own:
        import paper_2608_30386_b200 as dasc
        dasc.dasc_verify_draft(s["target"], s["draft"], s["tokens"], s["cu"], s["u"], s["u_next"], s["out"], s["kept"])
        return {"out": s["out"], "kept": s["kept"]}
    R, V, cu = case["requests"], case["vocab"], s["cu"].long()
    n, j, r = cu[1:] - cu[:-1], torch.arange(s["most"], device=DEVICE), torch.arange(R, device=DEVICE)
    at = (cu[:-1, None] + j).clamp(max=s["tokens"].numel() - 1)  # [R, most]: drafted token j of request r
    x = s["tokens"].long()[at]
    rows = (cu[:-1] + r)[:, None] + torch.minimum(j, n[:, None])
    p = s["target"][rows, x].double()
    q = s["draft"][at, x].double() if s["draft"] is not None else 1.0
    stands = ((s["u"][at].double() * q < p) & (j < n[:, None])).long().cumprod(1)
    count = stands.sum(1)
    all_stand = count == n
    P = s["target"][cu[:-1] + r + count].double()
    last = (cu[:-1] + count).clamp(max=s["tokens"].numel() - 1)
    if s["draft"] is not None:
        Q = s["draft"][last].double()
    else:
        Q = (torch.arange(V, device=DEVICE) == s["tokens"].long()[last][:, None]).double()
    w = torch.where(all_stand[:, None], P, P - Q).clamp(min=0)
    w = torch.where(w.sum(1, keepdim=True) > 0, w, P.clamp(min=0))
    cdf = w.cumsum(1)
    token = (cdf <= s["u_next"].double()[:, None] * w.sum(1, keepdim=True)).sum(1).clamp(max=V - 1)
    wide = torch.cat([x, torch.full((R, 1), -1, device=DEVICE)], 1)
    place = torch.arange(s["most"] + 1, device=DEVICE)
    out = torch.where(place < count[:, None], wide, torch.where(place == count[:, None], token[:, None], -1))
    s["out"].copy_(out)
    s["kept"].copy_(count + 1)
    return {"out": s["out"], "kept": s["kept"]}


# ---- the definition in 64 bits -----------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "verify":
        return _exact_verify(s, case)
    L, R, H, K, d = case["layers"], case["requests"], case["v_heads"], case["k_heads"], case["dim"]
    req = s["req"].tolist()
    if case["op"] == "step":
        state, o = s["state"].double(), torch.empty(L, R, H, d, device=DEVICE, dtype=torch.float64)
        for i, r in enumerate(req):
            for h in range(H):
                g = s["g"][:, h] if case["decay"] == "head" else s["g"][:, i, h]
                kh = h // (H // K)
                S = g.double().exp()[:, None, None] * state[r, :, h] + torch.einsum("lk,lv->lkv", s["k"][:, i, kh].double(), s["v"][:, i, h].double())
                state[r, :, h] = S
                o[:, i, h] = s["scale"] * torch.einsum("lk,lkv->lv", s["q"][:, i, kh].double(), S)
        return {"o": o, "state": state}
    # every output as its whole causal sum, blocks of queries against all keys before them; every state as one decayed sum
    cu = s["cu"].tolist()
    o = s["o"].double() if case["out"] else None
    state = s["state"].double() if case["mode"] != "score" else s["state"]
    heads = torch.arange(H, device=DEVICE) // (H // K)
    for layer in range(L):
        for r in range(R):
            b, e = cu[r], cu[r + 1]
            if s["used"] is not None:
                e = min(e, b + int(s["used"][r]))
            k, v = s["k"][layer, b:e].double().transpose(0, 1)[heads], s["v"][layer, b:e].double().transpose(0, 1)
            g = s["g"][layer].double()
            g = g[:, None].expand(H, e - b) if case["decay"] == "head" else g[b:e].T
            G = g.cumsum(1)  # [H, n]
            zero = case["mode"] == "merge" or s["zero"] is not None
            S = torch.zeros(H, d, d, device=DEVICE, dtype=torch.float64) if zero else s["state"][req[r], layer].double()
            if o is not None:
                q = s["q"][layer, b:e].double().transpose(0, 1)[heads]
                step = max(16, min(e - b, 2 ** 25 // max(1, H * (e - b))))
                for t in range(0, e - b, step):
                    u = min(e - b, t + step)
                    far = G[:, t:u, None] - G[:, None, :u]
                    far = far.masked_fill(torch.arange(u, device=DEVICE) > torch.arange(t, u, device=DEVICE)[:, None], -torch.inf)
                    out = (q[:, t:u] @ k[:, :u].transpose(1, 2) * far.exp()) @ v[:, :u] + G[:, t:u, None].exp() * (q[:, t:u] @ S)
                    o[layer, b + t:b + u] = s["scale"] * out.transpose(0, 1)
            if case["mode"] != "score":
                new = G[:, -1, None, None].exp() * S + (k * (G[:, -1:] - G).exp()[..., None]).transpose(1, 2) @ v
                if case["mode"] == "merge":
                    new = torch.where(s["keep"][layer][:, None, None], state[req[r], layer], new)
                state[req[r], layer] = new
    return {**({"o": o} if case["out"] else {}), **({"state": state} if case["mode"] != "score" else {})}


def _exact_verify(s, case):
    cu, tokens, u = s["cu"].tolist(), s["tokens"].tolist(), s["u"].tolist()
    out, kept = torch.full_like(s["out"], -1), torch.zeros_like(s["kept"])
    for r in range(case["requests"]):
        n, count = cu[r + 1] - cu[r], 0
        while count < n:
            i = cu[r] + count
            x = tokens[i]
            q = float(s["draft"][i, x]) if s["draft"] is not None else 1.0
            if not u[i] * q < float(s["target"][i + r, x]):
                break
            out[r, count] = x
            count += 1
        w = s["target"][cu[r] + r + count].double().clone()
        if count < n:
            rest = w.clone()
            if s["draft"] is not None:
                rest -= s["draft"][cu[r] + count].double()
            else:
                rest[tokens[cu[r] + count]] -= 1.0
            rest = rest.clamp(min=0)
            w = rest if float(rest.sum()) > 0 else w
        cdf = w.cumsum(0)
        out[r, count] = int(torch.searchsorted(cdf, s["u_next"][r].double() * cdf[-1], right=True).clamp(max=case["vocab"] - 1))
        kept[r] = count + 1
    return {"out": out, "kept": kept}
