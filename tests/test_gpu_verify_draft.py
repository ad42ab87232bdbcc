"""Verification of drafted tokens against its definition in 64 bits: whole numbers, which have to be equal."""
import math

import pytest
import torch

from paper_2510_03246_amd import strp

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def ld8(n):
    return (n + 7) // 8 * 8


@pytest.fixture(scope="module")
def ctx():
    return strp.Context(0)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def floats(x):
    return torch.tensor(x, dtype=F32, device="cuda")


def logits(V, cols, seed, dt, spread=2.5, ld=None):
    """[V x ld] with NaN behind the columns"""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.full((V, ld or ld8(max(cols, 1))), float("nan"), dtype=dt, device="cuda")
    x[:, :cols] = (torch.randn((V, cols), generator=g, device="cuda") * spread).to(dt)
    return x


def softmax64(x, tau):
    x = x.double() / tau
    e = torch.exp(x - x.amax(0))
    return e / e.sum(0)


def reference(target, draft, ids, u, u_next, starts, tau):
    """accepted, next_ids, and how near each next token's threshold lies to another sum (relative)"""
    acc, nxt, gap = [], [], []
    for s, (a, e) in enumerate(zip(starts, starts[1:])):
        n, at = e - a, 0
        p = softmax64(target[:, a + s:e + s + 1], tau)
        q = softmax64(draft[:, a:e], tau) if n else None
        while at < n and 0 <= ids[a + at] < p.shape[0] and u[a + at] * float(q[ids[a + at], at]) < float(p[ids[a + at], at]):
            at += 1
        r = p[:, at]
        if at < n:
            rest = (r - q[:, at]).clamp_min(0)
            r = rest if float(rest.sum()) > 0 else r
        c = torch.cumsum(r, 0)
        goal = u_next[s] * float(c[-1])
        over = (c > goal).nonzero()
        acc.append(at)
        nxt.append(int(over[0]) if len(over) else int((r > 0).nonzero()[-1]))
        gap.append(float((c - goal).abs().min() / c[-1]))
    return acc, nxt, gap


def verify_case(ctx, V, counts, dt, tau=1.0, seed=0, near=0.7, fix=None, ld=None):
    starts = [0]
    for n in counts:
        starts.append(starts[-1] + n)
    T, n_seq = starts[-1], len(counts)
    target = logits(V, T + n_seq, seed, dt, ld=ld)
    at = [a + s + i for s, (a, e) in enumerate(zip(starts, starts[1:])) for i in range(e - a)]
    draft = logits(V, T, seed + 1, dt, near)
    if T:
        draft[:, :T] = (draft[:, :T].float() + target[:, at].float()).to(dt)
    if fix:
        fix(target, draft)
    g = torch.Generator(device="cuda").manual_seed(seed + 2)
    ids = torch.multinomial(softmax64(draft[:, :T], tau).nan_to_num(1.0).t(), 1, generator=g)[:, 0].to(torch.int32) if T else ints([])
    u, u_next = torch.rand(T, generator=g, device="cuda"), torch.rand(n_seq, generator=g, device="cuda")
    got = ctx.strp_verify_draft(target, draft if T else None, ids if T else None, u if T else None, u_next, ints(starts) if n_seq > 1 else None, tau)
    acc, nxt, gap = reference(target, draft, ids.tolist(), u.tolist(), u_next.tolist(), starts, tau)
    # sums of V terms in another order: V 2^-52 of the whole at most
    for s in range(n_seq):
        assert int(got["accepted"][s]) == acc[s], (s, counts[s])
        assert int(got["next_ids"][s]) == nxt[s] or gap[s] < V * 2.0 ** -52, (s, int(got["next_ids"][s]), nxt[s], gap[s])
    return got


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("V", [1, 2, 31, 255, 256, 257, 1000, 5003, 50000, 130001])
def test_verify(ctx, V, dt):
    verify_case(ctx, V, [4], dt)
    verify_case(ctx, V, [0], dt, seed=1)
    verify_case(ctx, V, [0, 3, 1, 0, 7, 2, 12, 0], dt, tau=0.7, seed=2)
    verify_case(ctx, V, [0] * 5, dt, tau=1.5, seed=3)


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("counts", [[i % 6 for i in range(70)], [4] * 128, [1] * 33, [40], [9, 0, 33, 5]], ids=lambda c: f"{len(c)}x{c[0]}")
def test_verify_batches(ctx, counts, dt):
    verify_case(ctx, 3001, counts, dt, seed=5)
    verify_case(ctx, 3001, counts, dt, seed=6, near=0.05, ld=ld8(sum(counts) + len(counts)) + 24)      # nearly all kept


@pytest.mark.parametrize("dt", [BF16, F32])
def test_verify_temperatures_and_spreads(ctx, dt):
    for tau in (0.01, 0.2, 5.0, 100.0, 1e6):
        verify_case(ctx, 2000, [3, 0, 5], dt, tau=tau, seed=7)


@pytest.mark.parametrize("dt", [BF16, F32])
def test_verify_masked_and_far_entries(ctx, dt):
    def mask(target, draft):
        target[100:], draft[50:] = -math.inf, -math.inf
        target[:3] = -math.inf                  # a slice that begins with nothing
    verify_case(ctx, 5000, [5, 0, 2, 8], dt, seed=8, fix=mask)

    def far(target, draft):
        target += torch.arange(0, target.shape[0], device="cuda")[:, None] * 3.0      # thousands apart, the best last
        draft.copy_(target[:, :draft.shape[1]])
    verify_case(ctx, 3000, [5, 0, 2, 8], F32, seed=9, fix=far)

    def one(target, draft):
        target.fill_(-math.inf)
        draft.fill_(-math.inf)
        target[7], draft[7] = 3.0, -2.0
    got = verify_case(ctx, 300, [3, 0, 2], dt, seed=10, fix=one)
    assert got["accepted"].tolist() == [3, 0, 2] and got["next_ids"].tolist() == [7, 7, 7]


def test_verify_the_same_distribution_keeps_all(ctx):
    x = logits(1000, 5, 1, F32)
    got = ctx.strp_verify_draft(x, x.clone(), ints([1, 2, 3, 4]), floats([0.0, 0.5, 0.99, 0.999999]), floats([0.3]))
    assert got["accepted"].tolist() == [4]


def test_verify_borders_of_the_random_numbers(ctx):
    """Equal probabilities: the sums are whole multiples, u_next on them takes the next; 0 the first and 1 and more the last with a weight."""
    V = 8
    x = torch.full((V, 8), -math.inf, device="cuda")
    x[2:6] = 0.0
    for un, want in ((0.0, 2), (0.25, 3), (0.2499999, 2), (0.5, 4), (0.75, 5), (0.9999999, 5), (1.0, 5), (7.0, 5), (-1.0, 2), (float("nan"), 5)):
        got = ctx.strp_verify_draft(x, None, None, None, floats([un]))
        assert got["next_ids"].tolist() == [want] and got["accepted"].tolist() == [0], un
    # a token on the border: u q = p is not kept
    d = torch.full((V, 8), -math.inf, device="cuda")
    d[2:4] = 0.0                               # q = 1/2, p = 1/4
    for u, kept in ((0.4999999, 1), (0.5, 0), (0.0, 1), (float("nan"), 0)):
        got = ctx.strp_verify_draft(x, d, ints([3]), floats([u]), floats([0.6]))
        assert got["accepted"].tolist() == [kept], u
        assert got["next_ids"].tolist() == [4 if kept else 5]      # of p = 1/4 on 2..5; of the rest, 1/2 on 4 and 5
    # the rest is zero everywhere: the target's own
    got = ctx.strp_verify_draft(x, x.clone(), ints([1]), floats([0.5]), floats([0.3]))
    assert got["accepted"].tolist() == [0] and got["next_ids"].tolist() == [3]


def test_verify_what_has_no_answer(ctx):
    """NaN, +inf, nothing but -inf, in target or draft: the sequence ends there, the others are as ever; ids outside the vocabulary are not kept."""
    V, counts = 700, [3] * 8
    base_t, base_d = logits(V, 32, 1, F32), logits(V, 24, 2, F32)
    base_d[:, :24] = base_t[:, [4 * s + i for s in range(8) for i in range(3)]]      # the same: all kept
    ids, u, un = ints([5] * 24), floats([0.5] * 24), floats([0.5] * 8)
    starts = ints(list(range(0, 25, 3)))
    want = ctx.strp_verify_draft(base_t, base_d, ids, u, un, starts)
    assert want["accepted"].tolist() == [3] * 8
    t, d = base_t.clone(), base_d.clone()
    t[9, 4 * 0 + 1] = float("nan")
    t[699, 4 * 1 + 3] = float("inf")
    t[:, 4 * 2] = -math.inf
    d[0, 3 * 3 + 2] = float("nan")
    d[4, 3 * 4 + 0] = float("inf")
    d[:, 3 * 5 + 1] = -math.inf
    i2 = ids.clone()
    i2[3 * 6 + 1], i2[3 * 7] = -1, V
    got = ctx.strp_verify_draft(t, d, i2, u, un, starts)
    assert got["accepted"].tolist() == [1, 3, 0, 2, 0, 1, 1, 0]
    assert got["next_ids"].tolist()[:6] == [-1] * 6 and min(got["next_ids"].tolist()[6:]) >= 0


def test_verify_wrong_offsets_stay_in_bounds(ctx):
    t, d = logits(500, 16, 1, F32, ld=16), logits(500, 8, 2, F32, ld=8)
    for starts in ([5, 2, 9, -3], [0, 1 << 30, 3, 8], [-1 << 31, 8, 8, 8], [8, 8, 8, 0]):
        got = ctx.strp_verify_draft(t, d, ints([3] * 8), floats([0.5] * 8), floats([0.5] * 3), ints(starts))
        assert all(0 <= a <= 8 for a in got["accepted"].tolist())


def test_verify_beyond_32_bit_offsets(ctx):
    V, cols = 130000, 20000
    target = torch.zeros((V, cols), dtype=BF16, device="cuda")
    target[V - 1, cols - 1] = 20.0
    target[:, 1].fill_(-math.inf)
    target[V - 1, 1] = 1.0
    got = ctx.strp_verify_draft(target, None, None, None, torch.full((cols,), 0.5, device="cuda"))
    n = got["next_ids"].tolist()
    assert n[0] == V // 2 and n[1] == V - 1 and n[-1] == V - 1 and n[-2] == V // 2


def test_verify_captured_and_replayed(ctx):
    V, counts = 5000, [4, 0, 2, 3]
    starts = ints([0, 4, 4, 6, 9])
    t, d = logits(V, 13, 1, BF16), logits(V, 9, 2, BF16)
    g = torch.Generator(device="cuda").manual_seed(3)
    ids, u, un = torch.randint(0, V, (9,), generator=g, device="cuda", dtype=torch.int32), torch.rand(9, generator=g, device="cuda"), torch.rand(4, generator=g, device="cuda")
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        c = strp.Context(0)
        c.strp_verify_draft(t, d, ids, u, un, starts)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            out = c.strp_verify_draft(t, d, ids, u, un, starts)
    for i in range(4):
        un.copy_(torch.rand(4, generator=g, device="cuda"))
        u.copy_(torch.rand(9, generator=g, device="cuda") * 0.2)
        t[:, :13] = t[:, :13].flip(0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = ctx.strp_verify_draft(t, d, ids, u, un, starts)
        assert torch.equal(out["accepted"], want["accepted"]) and torch.equal(out["next_ids"], want["next_ids"]), i


def test_tokens_are_distributed_as_the_target_s(ctx):
    """20000 sequences of one drafted token each: what comes out first is distributed as p.  64 entries, each count within five of its standard deviations (one entry in
    10^6 is not; the random numbers are fixed)."""
    V, n = 64, 20000
    g = torch.Generator(device="cuda").manual_seed(11)
    p, q = torch.randn(V, generator=g, device="cuda") * 1.5, torch.randn(V, generator=g, device="cuda") * 1.5
    target, draft = p[:, None].expand(V, 2 * n).contiguous(), q[:, None].expand(V, n).contiguous()
    ids = torch.multinomial(torch.softmax(q, 0), n, replacement=True, generator=g).to(torch.int32)
    u, un = torch.rand(n, generator=g, device="cuda"), torch.rand(n, generator=g, device="cuda")
    got = ctx.strp_verify_draft(target, draft, ids, u, un, ints(list(range(n + 1))))
    first = torch.where(got["accepted"] == 1, ids, got["next_ids"])
    want = softmax64(p[:, None], 1.0)[:, 0]
    counts = torch.bincount(first.long(), minlength=V).double()
    assert ((counts - n * want).abs() <= 5 * torch.sqrt(n * want * (1 - want))).all()
    keep = float(torch.minimum(want, softmax64(q[:, None], 1.0)[:, 0]).sum())      # sum of q min(1, p / q)
    assert abs(float(got["accepted"].double().mean()) - keep) <= 5 * math.sqrt(keep * (1 - keep) / n)


def test_binding_refusals(ctx):
    t, d, ids, u, un = logits(100, 8, 1, F32), logits(100, 8, 2, F32), ints([1, 2]), floats([0.5, 0.5]), floats([0.5])
    for err, call in ((ValueError, lambda: ctx.strp_verify_draft(t[:, :2], d, ids, u, un)),
                      (ValueError, lambda: ctx.strp_verify_draft(t, d[:50], ids, u, un)),
                      (TypeError, lambda: ctx.strp_verify_draft(t, d.to(BF16), ids, u, un)),
                      (TypeError, lambda: ctx.strp_verify_draft(t.half(), d, ids, u, un)),
                      (TypeError, lambda: ctx.strp_verify_draft(t, d, ids.long(), u, un)),
                      (ValueError, lambda: ctx.strp_verify_draft(t, d, ids, u[:1], un)),
                      (ValueError, lambda: ctx.strp_verify_draft(t, None, ids, u, un)),
                      (ValueError, lambda: ctx.strp_verify_draft(t, d, ids, u, un.cpu())),
                      (ValueError, lambda: ctx.strp_verify_draft(t, d, ids, u, un, ints([0]))),
                      (strp.StrpError, lambda: ctx.strp_verify_draft(t, d, ids, u, floats([0.5, 0.5]))),
                      (strp.StrpError, lambda: ctx.strp_verify_draft(t, d, ids, u, un, temperature=0.0)),
                      (strp.StrpError, lambda: ctx.strp_verify_draft(t, d, ids, u, un, temperature=float("nan"))),
                      (strp.StrpError, lambda: ctx.strp_verify_draft(t, None, None, None, un[:0]))):
        with pytest.raises(err):
            call()


# ---- temperatures at which a logit is 10^10 of them and more ----
def softmax_apart(x, tau):
    """Differences first: exact, or within 2^-53, where x / tau would lose them."""
    x = x.double()
    e = torch.exp((x - x.amax(0)) / tau)
    return e / e.sum(0)


def ties(V, cols, seed, dt, level, rows):
    """Random logits below `level` and, in every column, `rows` of them at it: what is left of the distribution at a temperature of next to nothing."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.full((V, ld8(max(cols, 1))), float("nan"), dtype=dt, device="cuda")
    top = torch.full((), level, device="cuda").to(dt).float()
    x[:, :cols] = (top - top.abs() * (2.0 ** -6 + torch.rand((V, cols), generator=g, device="cuda"))).to(dt)
    x[rows, :cols] = top.to(dt)
    return x


COLD = [1.0, 1e-3, 1e-6, 1e-10, 1e-12, 1e-14, 1e-16, 1e-18, 1e-21, 1e-24, 1e-30]


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("level", [20.3, -20.3, 3.0e4, -3.1e4, 1.0e30])
def test_verify_the_normaliser_at_low_temperatures(ctx, dt, level):
    """Five equal best tokens in the target and four in the draft, three of them the same; another level in the draft, so that nothing cancels.  Where the others
    have no weight, p = 1/5 and q = 1/4, and a draft is kept below u = 0.8: fp32's neighbours of that are 1.5e-8 and 4.5e-8 away, while exponentials to 2^-43, a
    factor 1 / temperature and a difference rounded once each (40 * 2^-52 where a weight counts) and sums of V terms make less than 2^-40."""
    V, tol = 700, 2.0 ** -40
    best_t, best_d = [3, 77, 300, 512, 699], [77, 300, 512, 613]
    counts = [1, 1, 0, 3, 2, 0, 1]
    starts = [0]
    for n in counts:
        starts.append(starts[-1] + n)
    T, n_seq = starts[-1], len(counts)
    above = float(torch.tensor(0.8, dtype=F32))                   # the nearest, above 0.8
    below = above - 2.0 ** -24
    assert below < 0.8 < above
    target, draft = ties(V, T + n_seq, 1, dt, level, best_t), ties(V, T, 2, dt, level * 0.83, best_d)
    ids = [300, 300, 77, 512, 300, 512, 77, 613]
    us = [below, above, below, below, above, 0.1, 0.7, 0.3]
    un = [0.1, 0.3, 0.5, 0.7, 0.9, 0.99, 0.19]
    for tau in COLD:
        got = ctx.strp_verify_draft(target, draft, ints(ids), floats(us), floats(un), ints(starts), tau)
        none = ctx.strp_verify_draft(target[:, :ld8(n_seq)].contiguous(), None, None, None, floats(un), None, tau)
        p, q = softmax_apart(target[:, :T + n_seq], tau), softmax_apart(draft[:, :T], tau)
        if tau < 1e-2 * abs(level) / 700:
            assert abs(float(p[3, 0]) - 0.2) < 1e-15 and abs(float(q[77, 0]) - 0.25) < 1e-15
        for s, a in enumerate(starts[:-1]):
            n, at = counts[s], 0
            u32, goal = floats(us).double().tolist(), float(floats(un)[s])
            while at < n:
                left, right = u32[a + at] * float(q[ids[a + at], a + at]), float(p[ids[a + at], a + s + at])
                assert abs(left - right) > tol * right            # the case is no matter of rounding
                if not left < right:
                    break
                at += 1
            assert int(got["accepted"][s]) == at, (tau, s, int(got["accepted"][s]), at)
            r = p[:, a + s + at]
            if at < n:
                r = (r - q[:, a + at]).clamp_min(0)
            for r, answer in ((r, int(got["next_ids"][s])), (p[:, s], int(none["next_ids"][s]))):
                c = torch.cumsum(r, 0)
                over = int((c > goal * float(c[-1])).nonzero()[0])
                assert answer == over or float((c - goal * float(c[-1])).abs().min()) < tol, (tau, s, answer, over)
        assert none["accepted"].tolist() == [0] * n_seq


def test_verify_neighbouring_logits_at_a_temperature_between(ctx):
    """fp32 neighbours that are some hundred temperatures apart: 64 and what follows it, 763 at 1e-8.  Only the larger ones, one entry in a hundred, have a weight: p = 1 / N, and a
    draft of q = 1 / M, M of the same entries, is kept below u = M / N."""
    V, n_seq = 50000, 64
    g = torch.Generator(device="cuda").manual_seed(3)
    more = torch.rand((V, 2 * n_seq), generator=g, device="cuda") < 0.01
    more[0] = False
    more[7] = True
    more[:, 1::2] = more[:, ::2]                                  # a sequence's position and the one behind it
    N = more[:, ::2].sum(0)
    M = N - N // 20
    of = more[:, ::2]
    draft = torch.where(of & (torch.cumsum(of, 0) <= M), 0.0, -math.inf)
    u_next = torch.rand(n_seq, generator=g, device="cuda")
    ids, starts = torch.full((n_seq,), 7, dtype=torch.int32, device="cuda"), ints(list(range(n_seq + 1)))
    for low in (64.0, -64.0, 1.0, 3.7e-3):
        lo = torch.full((V, 2 * n_seq), low, device="cuda")
        hi = torch.nextafter(lo, torch.full_like(lo, math.inf))
        x = torch.where(more, hi, lo)
        for apart in (260.0, 400.0, 520.0, 700.0, 763.0, 990.0, 1020.0, 1500.0):
            tau = float(hi[0, 0].double() - lo[0, 0].double()) / apart
            for factor, kept in ((0.999, 1), (1.001, 0)):
                got = ctx.strp_verify_draft(x, draft, ids, (M / N * factor).float(), u_next, starts, tau)
                assert got["accepted"].tolist() == [kept] * n_seq, (low, apart, factor)
                if kept:
                    for s in range(0, n_seq, 7):
                        at = of[:, s].nonzero()[:, 0]
                        place = float(u_next[s]) * len(at)
                        assert abs(place - round(place)) > 1e-6   # equal weights: the answer's place among them
                        assert int(got["next_ids"][s]) == int(at[math.floor(place)]), (low, apart, s)
