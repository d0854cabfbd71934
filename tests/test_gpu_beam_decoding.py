"""The decoding calls together, as a serving loop makes them: beam search over delta-rule layers, and drafted tokens; as calls, captured and replayed, and on
two streams at once."""
import numpy as np
import pytest
import torch

import beam_helpers as bh
import delta_helpers as dh
import paper_2608_30386_b200 as dasc

pytestmark = pytest.mark.gpu


class Toy:
    """Two delta-rule layers between random tables: what a beam's next logits are depends on its states and its last token only."""

    def __init__(self, kind, V, slots, H=2, d=64, L=2, seed=0):
        gen = torch.Generator().manual_seed(seed)
        n = lambda *s: torch.randn(*s, generator=gen).cuda()  # noqa: E731
        self.kind, self.V, self.H, self.d, self.L = kind, V, H, d, L
        self.plan = dh.make_plan(kind, L, H, H, d, d)
        unit = lambda x: x / x.norm(dim=-1, keepdim=True)  # noqa: E731
        self.q, self.k, self.v = unit(n(L, V, H, d)), unit(n(L, V, H, d)), n(L, V, H, d)
        self.g = -torch.nn.functional.softplus(n(L, V, H, d) if kind == dasc.KDA else n(L, V, H)) * 0.2
        self.beta = torch.sigmoid(n(L, V, H))
        self.head = n(L * H * d, V) / 4
        self.state = torch.zeros(slots, L, H, d, d, device="cuda")
        self.strides = (H * d * d, L * H * d * d)

    def streams(self, tokens):
        return [x[:, tokens.long()].contiguous() for x in (self.q, self.k, self.v, self.g, self.beta)]

    def logits(self, o):  # [L, n, H, d]
        return o.transpose(0, 1).reshape(o.shape[1], -1) @ self.head


def beam_loop(toy, R, W, steps, fused):
    """Tokens and scores of every beam; the first token is 0, token 1 ends a beam."""
    slots = torch.randperm(R * W, generator=torch.Generator().manual_seed(1)).to(torch.int32).cuda().view(R, W)
    scores = torch.full((R, W), -float("inf"), device="cuda")
    scores[:, 0] = 0.0
    ended = torch.zeros(R, W, dtype=torch.int32, device="cuda")
    token, parent, new = torch.zeros_like(slots), torch.zeros_like(slots), torch.empty_like(slots)
    src = slots.clone()
    history = torch.zeros(R, W, 0, dtype=torch.int32, device="cuda")
    toy.state.zero_()
    for _ in range(steps):
        o = torch.empty(toy.L, R * W, toy.H, toy.d, device="cuda")
        for layer in range(toy.L):
            x = [y[layer:layer + 1] for y in toy.streams(token.flatten())]
            dasc.dasc_delta_step(toy.plan, toy.state, *toy.strides, slots.flatten(), *x, o[layer:layer + 1], layer_begin=layer, layer_end=layer + 1,
                                 **({"src_idx": src.flatten(), "beam_width": W} if fused else {}))
        dasc.dasc_beam_select(toy.logits(o).view(R, W, toy.V), scores, scores, parent, token, ended=ended, out_ended=ended, end_token=1)
        new = torch.empty_like(slots)
        dasc.dasc_beam_reorder(toy.plan, None if fused else toy.state, *toy.strides, slots, parent, new, src_idx=src)
        slots = new
        at = parent.clamp(min=0).long()[..., None].expand(-1, -1, history.shape[2])
        history = torch.cat([history.gather(1, at), token[..., None]], 2)
    return history.cpu().numpy(), scores.cpu().numpy()


def host_beams(toy, W, steps):
    """The same search over whole token sequences in 64 bits, every state computed from its beam's tokens."""
    q, k, v, g, beta, head = (x.cpu().double() for x in (toy.q, toy.k, toy.v, toy.g, toy.beta, toy.head))
    beams = [([0], 0.0, False)]
    for _ in range(steps):
        found = []
        for b, (tokens, score, over) in enumerate(beams):
            if over:
                found.append((score, b, 1, True))
                continue
            outs = []
            for layer in range(toy.L):
                for h in range(toy.H):
                    x = [y[layer, tokens, h] for y in (q, k, v, g, beta)]
                    outs.append(dh.reference(torch.zeros(toy.d, toy.d, dtype=torch.float64), *x, 1.0)[0][-1])
            logp = torch.log_softmax(torch.cat(outs) @ head, -1)
            best = logp.topk(min(W, toy.V))
            found += [(score + float(p), b, int(t), int(t) == 1) for p, t in zip(*best)]
        found.sort(key=lambda x: (-x[0], x[1], x[2]))
        beams = [(beams[b][0] + [t], s, over) for s, b, t, over in found[:W]]
    return np.array([b[0][1:] for b in beams]), np.array([b[1] for b in beams])


@pytest.mark.parametrize("kind", [dasc.KDA, dasc.GDN], ids=["kda", "gdn"])
@pytest.mark.parametrize("fused", [False, True], ids=["copied", "read where they are"])
def test_beam_search_finds_what_it_finds_on_the_host(kind, fused):
    R, W, steps = 3, 4, 7
    toy = Toy(kind, 211, R * W, seed=5 + kind)
    tokens, scores = beam_loop(toy, R, W, steps, fused)
    want_tokens, want_scores = host_beams(toy, W, steps)
    for r in range(R):
        np.testing.assert_array_equal(tokens[r], want_tokens)
        # outputs of 14 tokens of d = 64 in fp32 and logits of 256 products of them: (8 * 112 + 256) 2^-24 of sums below 100 per step, 7 steps
        np.testing.assert_allclose(scores[r], want_scores, rtol=0, atol=7 * 100 * 1152 * 2.0 ** -24)


@pytest.mark.parametrize("kind", [dasc.KDA, dasc.GDN], ids=["kda", "gdn"])
def test_drafts_are_scored_verified_and_advanced_over(kind):
    """Score, verify, advance by n_kept: the states are those of the tokens that stand, and the outputs those of a token by token run."""
    R, n, V = 9, 4, 97
    toy = Toy(kind, V, R, seed=3)
    gen = torch.Generator(device="cuda").manual_seed(2)
    toy.state.normal_(generator=gen)
    start = toy.state.clone()
    last = torch.randint(0, V, (R, 1), generator=gen, device="cuda")
    drafts = torch.randint(0, V, (R, n), generator=gen, device="cuda")
    tokens = torch.cat([last, drafts], 1).flatten()
    req = torch.arange(R, dtype=torch.int32, device="cuda")
    cu = torch.arange(0, R * (n + 1) + 1, n + 1, dtype=torch.int32, device="cuda")
    x = toy.streams(tokens)
    o = torch.empty(toy.L, R * (n + 1), toy.H, toy.d, device="cuda")
    dasc.dasc_delta_draft(toy.plan, toy.state, *toy.strides, req, *x, cu, R * (n + 1), n + 1, o=o, mode=dasc.DRAFT_SCORE)
    assert torch.equal(toy.state, start)
    probs = torch.softmax(toy.logits(o) / 8, -1)
    out = torch.empty(R, n + 1, dtype=torch.int32, device="cuda")
    kept = torch.empty(R, dtype=torch.int32, device="cuda")
    cu_drafts = torch.arange(0, R * n + 1, n, dtype=torch.int32, device="cuda")
    u = torch.rand(R * n, generator=gen, device="cuda") * 0.01
    dasc.dasc_verify_draft(probs, None, drafts.flatten().to(torch.int32), cu_drafts, u, torch.rand(R, generator=gen, device="cuda"), out, kept)
    dasc.dasc_delta_draft(toy.plan, toy.state, *toy.strides, req, None, *x[1:], cu, R * (n + 1), n + 1, seq_used=kept)
    # token by token
    state, stepped = start.clone(), torch.empty_like(o)
    for t in range(n + 1):
        still = torch.where(kept > t, req, -1)
        one = toy.streams(tokens.view(R, -1)[:, t])
        o1 = torch.full((toy.L, R, toy.H, toy.d), 5.0, device="cuda")
        dasc.dasc_delta_step(toy.plan, state, *toy.strides, still, *one, o1)
        stepped.view(toy.L, R, n + 1, toy.H, toy.d)[:, :, t] = o1
    assert 1 <= int(kept.min()) and int(kept.max()) > 1
    assert dh.worst(toy.state, state.cpu().double()) < 1e-5
    mask = (torch.arange(n + 1, device="cuda") < kept[:, None]).flatten()
    assert dh.worst(o[:, mask], stepped[:, mask].cpu().double()) < 1e-5


def test_captured_and_replayed_on_two_streams():
    """Two graphs of one loop's calls, each on its own buffers, replayed side by side: no workspace, nothing shared."""
    R, W, V = 4, 3, 5001
    toys = [Toy(dasc.KDA, 64, R * W, seed=s) for s in (1, 2)]
    graphs, held = [], []
    for i, toy in enumerate(toys):
        gen = torch.Generator(device="cuda").manual_seed(i)
        toy.state.normal_(generator=gen)
        logits = torch.randn(R, W, V, generator=gen, device="cuda")
        scores = torch.randn(R, W, generator=gen, device="cuda")
        slots = torch.arange(R * W, dtype=torch.int32, device="cuda").view(R, W)
        parent, token, new, src = (torch.empty_like(slots) for _ in range(4))
        out = torch.empty(R, W, device="cuda")
        x = toy.streams(torch.randint(0, 64, (R * W,), generator=gen, device="cuda"))
        o = torch.empty(toy.L, R * W, toy.H, toy.d, device="cuda")
        cu = torch.arange(R * W + 1, dtype=torch.int32, device="cuda")

        def calls(toy=toy, logits=logits, scores=scores, slots=slots, parent=parent, token=token, new=new, src=src, out=out, x=x, o=o, cu=cu):
            dasc.dasc_beam_select(logits, scores, out, parent, token)
            dasc.dasc_beam_reorder(toy.plan, None, 0, 0, slots, parent, new, src_idx=src)
            dasc.dasc_delta_step(toy.plan, toy.state, *toy.strides, new.flatten(), *x, o, src_idx=src.flatten(), beam_width=W)
            dasc.dasc_delta_draft(toy.plan, toy.state, *toy.strides, new.flatten(), *x, cu, R * W, 1, o=o)
            dasc.dasc_beam_reorder(toy.plan, toy.state, *toy.strides, slots, parent, new, src_idx=src)

        start = toy.state.clone()
        calls()
        torch.cuda.synchronize()
        want = [toy.state.clone(), o.clone(), new.clone(), out.clone()]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            calls()
        graphs.append(graph)
        held.append((toy, start, o, new, out, want, calls))  # (a graph's inputs live as long as it does: `calls` holds them)
    streams = [torch.cuda.Stream() for _ in toys]
    for _ in range(5):
        for toy, start, o, new, out, *_ in held:
            toy.state.copy_(start)
            o.zero_()
            out.zero_()
        torch.cuda.synchronize()
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for toy, start, o, new, out, want, _ in held:
            for a, b in zip((toy.state, o, new, out), want):
                assert torch.equal(a, b)


def test_calls_follow_what_the_same_stream_wrote():
    """Inputs written by a kernel on a side stream just ahead of each call."""
    case = dh.make_case(21, [3] * 40, H_v=8)
    want = dh.run(case)
    x, s = torch.randn(8, 4, 30000, device="cuda"), torch.randn(8, 4, device="cuda")
    sel = bh.call(x, s, 8)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            state, q, v = (torch.empty_like(y) for y in (case.state, case.q, case.v))
            o = torch.empty(1, case.T, 8, 128, device="cuda")
            y, out = torch.empty_like(x), torch.empty(8, 8, device="cuda")
            parent, token = (torch.empty(8, 8, dtype=torch.int32, device="cuda") for _ in range(2))
            torch.cuda._sleep(2_000_000)
            state.copy_(case.state), q.copy_(case.q), v.copy_(case.v)
            dasc.dasc_delta_draft(case.plan, state, *case.strides, case.req, q, case.k, v, case.g, case.beta, case.cu.cuda(), case.T, 3, o=o, q_scale=0.7)
            torch.cuda._sleep(2_000_000)
            y.copy_(x)
            dasc.dasc_beam_select(y, s, out, parent, token)
            side.synchronize()
            assert torch.equal(state, want[0]) and torch.equal(o, want[1])
            assert torch.equal(out, sel[0]) and torch.equal(parent, sel[1]) and torch.equal(token, sel[2])
