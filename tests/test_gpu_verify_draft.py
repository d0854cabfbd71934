"""dasc_verify_draft against its definition in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2608_30386_b200 as dasc

pytestmark = pytest.mark.gpu


def define(target, draft, tokens, cu, ua, un, most):
    """Token by token on the host; probabilities that are none count as nothing."""
    clean = lambda x: np.where((x > 0) & np.isfinite(x), x, 0.0)  # noqa: E731
    target = target.float().cpu().numpy().astype(np.float64)
    draft = None if draft is None else draft.float().cpu().numpy().astype(np.float64)
    ua, un = np.asarray(ua, np.float32), np.asarray(un, np.float32)
    V, R = target.shape[1], len(cu) - 1
    out, kept = np.full((R, most + 1), -1), np.zeros(R, int)
    for r in range(R):
        n, c = min(cu[r + 1] - cu[r], most), 0
        while c < n:
            i, x = cu[r] + c, tokens[cu[r] + c]
            if not 0 <= x < V or not float(ua[i]) * (1.0 if draft is None else draft[i, x]) < target[i + r, x]:
                break
            out[r, c] = x
            c += 1
        p = clean(target[cu[r] + r + c])
        w = p
        if c < n:
            q = np.zeros(V)
            if draft is not None:
                q = clean(draft[cu[r] + c])
            elif 0 <= tokens[cu[r] + c] < V:
                q[tokens[cu[r] + c]] = 1.0
            w = np.maximum(p - q, 0)
            w = w if w.sum() > 0 else p
        run = np.cumsum(w)
        if run[-1] > 0:
            out[r, c] = min(int(np.searchsorted(run, float(un[r]) * run[-1], side="right")), int(np.nonzero(w)[0][-1]))
        kept[r] = c + 1
    return out, kept


def call(target, draft, tokens, cu, ua, un, most, stride=None):
    R = len(cu) - 1
    out = torch.full((R, stride or most + 1), 99, dtype=torch.int32, device="cuda")
    kept = torch.full((R,), 99, dtype=torch.int32, device="cuda")
    i32, f32 = (lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")), (lambda x: torch.tensor(x, dtype=torch.float32, device="cuda"))
    dasc.dasc_verify_draft(target, draft, i32(tokens), i32(cu), f32(ua), f32(un), out[:, :most + 1], kept)
    torch.cuda.synchronize()
    if stride:
        assert bool((out[:, most + 1:] == 99).all())
    return out[:, :most + 1].cpu().numpy(), kept.cpu().numpy()


def same(got, want):
    np.testing.assert_array_equal(got[0], want[0])
    np.testing.assert_array_equal(got[1], want[1])


def make(seed, n, V, dtype=torch.float32, spread=2.0, noise=0.7):
    gen = torch.Generator().manual_seed(seed)
    cu = np.concatenate([[0], np.cumsum(n)]).astype(int)
    N, R = int(cu[-1]), len(n)
    logits = torch.randn(N + R, V, generator=gen) * spread
    rows = torch.tensor([cu[r] + r + j for r in range(R) for j in range(n[r])], dtype=torch.long)
    draft = torch.softmax(logits[rows] + noise * torch.randn(N, V, generator=gen), -1)
    tokens = torch.multinomial(draft, 1, generator=gen)[:, 0].tolist() if N else []
    u = lambda k: torch.rand(k, generator=gen).tolist()  # noqa: E731
    return torch.softmax(logits, -1).to(dtype).cuda(), draft.to(dtype).cuda(), tokens, cu.tolist(), u(N), u(R)


@pytest.mark.parametrize("V", [1, 2, 5, 127, 128, 129, 1000, 4099, 32000, 131072])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("q", [True, False])
def test_vocabularies(V, dtype, q):
    target, draft, tokens, cu, ua, un = make(V, [3, 0, 1, 4, 2], V, dtype)
    draft = draft if q else None
    same(call(target, draft, tokens, cu, ua, un, 4), define(target, draft, tokens, cu, ua, un, 4))


@pytest.mark.parametrize("n", [1, 7, 33, 64, 100])
def test_numbers_of_drafts(n):
    target, draft, tokens, cu, ua, un = make(n, [n, n // 2, 0, n], 300, noise=0.0)
    ua = [0.0 if i % 40 else 0.999 for i in range(len(ua))]  # most stand, past a warp's width too
    same(call(target, draft, tokens, cu, ua, un, n), define(target, draft, tokens, cu, ua, un, n))


def test_nobody_drafted():
    target, _, _, cu, _, un = make(8, [0, 0, 0], 500)
    for draft in (None, torch.empty(0, 500, device="cuda")):
        for most in (0, 3):
            same(call(target, draft, [], cu, [], un, most), define(target, None, [], cu, [], un, most))


def test_many_requests_have_the_distribution_of_the_target():
    """With q from the drafter and the residual drawn as defined, accepted-or-resampled first tokens follow the target: every one
    of them equals the definition's, and their counts are within five standard deviations of the target's probabilities."""
    R, V = 6000, 5
    p, q = torch.tensor([0.5, 0.2, 0.15, 0.1, 0.05]), torch.tensor([0.1, 0.3, 0.2, 0.2, 0.2])
    gen = torch.Generator().manual_seed(1)
    tokens = torch.multinomial(q, R, replacement=True, generator=gen).tolist()
    target, draft = p.expand(2 * R, V).contiguous().cuda(), q.expand(R, V).contiguous().cuda()
    ua, un = torch.rand(R, generator=gen).tolist(), torch.rand(R, generator=gen).tolist()
    cu = list(range(R + 1))
    got = call(target, draft, tokens, cu, ua, un, 1)
    same(got, define(target, draft, tokens, cu, ua, un, 1))
    count = np.bincount(got[0][:, 0], minlength=V)
    sd = np.sqrt(R * p.numpy() * (1 - p.numpy()))
    assert (np.abs(count - R * p.numpy()) < 5 * sd).all()


def test_borders_of_the_random_numbers():
    """u = 0 takes the first token with any weight, u just below 1 the last; a number on a border belongs to the next token."""
    w = [0.0, 0.25, 0.0, 0.25, 0.5, 0.0]
    target = torch.tensor([w] * 5).cuda()
    un = [0.0, 0.25, 0.5, float(np.float32(1) - np.float32(2) ** -24), float(np.float32(0.25) - np.float32(2) ** -26)]
    got, kept = call(target, None, [], [0] * 6, [], un, 2)
    assert got[:, 0].tolist() == [1, 3, 4, 4, 1] and kept.tolist() == [1] * 5 and (got[:, 1:] == -1).all()
    # u * q < p is strict: p = q and u = 0 stands where p > 0, p = 0 never does
    t = torch.tensor([[0.5, 0.5, 0.0], [1.0, 0.0, 0.0]] * 2).cuda()
    d = torch.tensor([[0.5, 0.5, 0.0], [0.0, 0.0, 1.0]]).cuda()
    got, kept = call(t, d, [1, 2], [0, 1, 2], [0.0, 0.0], [0.0, 0.0], 1)
    assert got.tolist() == [[1, 0], [0, -1]] and kept.tolist() == [2, 1]


def test_rows_that_leave_nothing():
    nan, inf = float("nan"), float("inf")
    rows = [[0.0, 0.0, 0.0, 0.0], [nan, nan, 0.0, -1.0], [nan, 0.5, inf, -3.0], [0.25, 0.25, 0.25, 0.25]]
    got, kept = call(torch.tensor(rows).cuda(), None, [], [0] * 5, [], [0.9] * 4, 1)
    assert got[:, 0].tolist() == [-1, -1, 1, 3]
    # a token that does not stand and leaves an empty residual: the target's own row
    t = torch.tensor([[0.0, 0.5, 0.5, 0.0], [1.0, 0.0, 0.0, 0.0]]).cuda()
    d = torch.tensor([[0.0, 0.5, 0.5, 0.0]]).cuda()
    got, kept = call(t, d, [3], [0, 1], [0.5], [0.6], 1)
    assert got.tolist() == [[2, -1]] and kept.tolist() == [1]


def test_tokens_outside_the_vocabulary_do_not_stand():
    target, draft, tokens, cu, ua, un = make(5, [2, 2], 50, noise=0.0)
    ua = [0.0] * 4
    tokens[1], tokens[2] = 50, -1
    for q in (draft, None):
        got, want = call(target, q, tokens, cu, ua, un, 2), define(target, q, tokens, cu, ua, un, 2)
        same(got, want)
        assert got[1].tolist() == [2, 1]


def test_strided_rows_and_outputs_and_too_many_drafts():
    target, draft, tokens, cu, ua, un = make(6, [3, 1, 5], 777)
    wide = torch.full((target.shape[0], 801), 5.0, device="cuda")
    wide[:, :777] = target
    wide_d = torch.full((draft.shape[0], 780), 5.0, device="cuda")
    wide_d[:, :777] = draft
    want = define(target, draft, tokens, cu, ua, un, 5)
    same(call(wide[:, :777], wide_d[:, :777], tokens, cu, ua, un, 5, stride=9), want)
    # five drafts where two are allowed: cut to two
    same(call(target, draft, tokens, cu, [0.0] * 9, un, 2), define(target, draft, tokens, cu, [0.0] * 9, un, 2))


@pytest.mark.parametrize("R", [32, 33, 64, 65, 148, 149])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_numbers_of_requests(R, dtype):
    target, draft, tokens, cu, ua, un = make(R, [r % 4 for r in range(R)], 2003, dtype)
    for q in (draft, None):
        same(call(target, q, tokens, cu, ua, un, 3), define(target, q, tokens, cu, ua, un, 3))


@pytest.mark.parametrize("R,V", [(1, 2 ** 20 + 129), (2, 1300001), (149, 131072 + 4), (150, 140001), (66, 262144 + 1000)])
def test_rows_so_long_that_a_sum_stands_for_several_tiles(R, V):
    target, draft, tokens, cu, ua, un = make(R + V, [2] + [0] * (R - 1), V, spread=1.0)
    same(call(target, draft, tokens, cu, ua, un, 2), define(target, draft, tokens, cu, ua, un, 2))
    un = [0.999999] * R
    same(call(target, draft, tokens, cu, [1.0, 1.0], un, 2), define(target, draft, tokens, cu, [1.0, 1.0], un, 2))
