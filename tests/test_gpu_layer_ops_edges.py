"""The decoder layer's operators where they can go wrong: how exact a result is, which variant runs, what lies beside the data.

U = 2^-23 bounds what one fp32 operation or one step of a matrix-core sum adds, relative to the magnitudes that meet there; H(t) is half a
step of an output of type t."""
import math

import pytest
import torch

import layer_ops_sizes as sizes
from paper_2510_03246_amd import strp
from test_gpu_layer_ops import linear_case, logprobs_check, norm_check, padded

pytestmark = pytest.mark.gpu

U = 2.0 ** -23
BF16, F32 = torch.bfloat16, torch.float32


def H(dt):
    return torch.finfo(dt).eps / 2


def ld8(T):
    return (T + 7) // 8 * 8


@pytest.fixture(scope="module")
def ctx():
    return strp.Context(0)


@pytest.fixture(scope="module")
def fast():
    c = strp.Context(0)
    c.set_precision(strp.PREC_FAST)
    return c


def rand(shape, seed, dt=F32, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dt)


# ---- attention ------------------------------------------------------------------------------------------------------
def attention_exact(Q, K, V, heads, kv_of, starts, scale, probs):
    """result and bound, where a probability is within `probs` of its value, relative, as it meets V"""
    dt, dh = Q.dtype, Q.shape[0] // heads
    out = torch.zeros((heads * dh, starts[-1]), dtype=torch.float64, device="cuda")
    tol = torch.zeros_like(out)
    for a, e in zip(starts, starts[1:]):
        n = e - a
        seen = torch.ones((n, n), dtype=torch.bool, device="cuda").tril()
        for h in range(heads):
            r, rk = slice(h * dh, (h + 1) * dh), slice(kv_of[h] * dh, (kv_of[h] + 1) * dh)
            q, k, v = Q[r, a:e].double(), K[rk, a:e].double(), V[rk, a:e].double()
            p = torch.softmax(torch.where(seen, scale * (q.t() @ k), -math.inf), 1)
            out[r, a:e] = v @ p.t()
            # a score is off by dh + 4 steps of its magnitudes, its probability by twice the largest of these of its row (the maximum's and its own), relative, and by 16 steps of the
            # exponential; the two sums have n terms each
            mag = torch.where(seen, scale * (q.abs().t() @ k.abs()), 0.0).max(1).values
            rel = 2 * (dh + 4) * U * mag + 16 * U + 2 * n * U + probs
            tol[r, a:e] = 2 * rel * (v.abs() @ p.t()) + H(dt) * out[r, a:e].abs() + 1e-37
    return out, tol


def attention_close(c, lens, heads, kv, dh, dt, probs, kv_of=None, seed=0):
    starts = [0]
    for n in lens:
        starts.append(starts[-1] + n)
    T = starts[-1]
    Q, K, V = (torch.full(((heads if i == 0 else kv) * dh, ld8(T)), float("nan"), dtype=dt, device="cuda") for i in range(3))
    for i, x in enumerate((Q, K, V)):
        x[:, :T] = rand((x.shape[0], T), seed + i, dt, 1.5 if i < 2 else 1.0)
    got = c.strp_attention(Q, K, V, T, heads, kv, torch.tensor(starts, dtype=torch.int32, device="cuda"),
                           kv_of_head=torch.tensor(kv_of, dtype=torch.int32, device="cuda") if kv_of else None)[:, :T].double()
    want, tol = attention_exact(Q[:, :T], K[:, :T], V[:, :T], heads, kv_of or [h // (heads // kv) for h in range(heads)], starts, dh ** -0.5, probs)
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), (lens, heads, kv, dh, int(bad.sum()), float(((got - want).abs() / tol).max()))


@pytest.mark.parametrize("dh", [8, 16, 31, 64, 80, 96, 128])
@pytest.mark.parametrize("lens", [[1], [64], [130, 1, 63], [300]], ids=str)
def test_attention_holds_the_probabilities_in_two_terms(ctx, lens, dh):
    """bf16, as a context comes: a probability meets V within 2^-16 of its value (the remainder of its upper 16 bits, below 2^-7 of it, rounded to nine)."""
    attention_close(ctx, lens, 4, 2, dh, BF16, 2.0 ** -16)


@pytest.mark.parametrize("dh", [1, 7, 8, 16, 31, 32, 33, 48, 63, 64, 65, 80, 96, 97, 100, 127, 128])
def test_attention_with_rounded_probabilities(fast, dh):
    attention_close(fast, [70, 1, 140], 4, 2, dh, BF16, H(BF16))
    attention_close(fast, [130, 1, 1, 250, 63], 3, 3, dh, BF16, H(BF16), kv_of=[2, 0, 2])


@pytest.mark.parametrize("dh", [64, 96, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_what_every_query_of_a_tile_sees_shows_itself(ctx, fast, bad, dh):
    """A value of V that is not finite at token 5 of 400 is that in its channel of every later token, also where its probability is a half, a quarter or too small to count;
    the other channels and the tokens before it have the bits they had."""
    T = 400
    for c in (ctx, fast):
        Q, K, V = (rand((2 * dh, T), i, BF16, s) for i, s in enumerate((0.0, 1.0, 1.0)))          # scores of zero: probabilities of 1 / (t + 1), many of them whole in eight bits
        V2 = V.clone()
        V2[3, 5] = bad
        rows = torch.arange(2 * dh, device="cuda") != 3
        for q in (Q, rand((2 * dh, T), 7, BF16, 1.5), rand((2 * dh, T), 7, BF16, 40.0)):
            clean, got = (c.strp_attention(q, K, v, T, 2, 2) for v in (V, V2))
            assert torch.equal(got[rows], clean[rows]) and torch.equal(got[3, :5], clean[3, :5])
            assert not torch.isfinite(got[3, 5:]).any()
        got = c.strp_attention(Q, K, V2, T, 2, 2)[3, 5:]
        assert bool(torch.isnan(got).all()) if bad != bad else bool((got == bad).all())


# ---- the workspace --------------------------------------------------------------------------------------------------
def leave_a_failure(c):
    """A refit whose matrix is not positive definite."""
    G = torch.diag(torch.tensor([1.0, 2.0, -3.0, 4.0, 5.0, 6.0, 7.0, 8.0], device="cuda"))
    A = rand((8, 64), 1)
    c.strp_refit(strp.SIDE_FC2, G, 0.0, A, A, 64, torch.arange(8, dtype=torch.int32, device="cuda"), torch.empty((8, 8), device="cuda"))


@pytest.mark.parametrize("call", ["linear", "logprobs", "mask", "set_workspace"])
def test_a_larger_workspace_keeps_a_failure_that_was_not_polled(call):
    c = strp.Context(0)
    c.set_workspace(1 << 17)
    leave_a_failure(c)
    size = c.ws.numel()
    if call == "linear":
        c.strp_linear(rand((512, 4096), 1, BF16), rand((4096, 512), 2, BF16), 512)
    elif call == "logprobs":
        c.strp_token_logprobs(rand((50000, 512), 1), 512, n_top=1)
    elif call == "mask":
        c.strp_mask_topk(rand(3000000, 1), 1000)
    else:
        c.set_workspace(1 << 22)
    assert c.ws.numel() > size
    assert c.poll() == strp.ENOTPD
    assert c.poll() == strp.OK


def test_a_captured_call_does_not_replace_the_workspace():
    """It is refused where it would have to, and the context is as it was; with room set before, every replay leaves a pending failure where it is."""
    W, X = rand((512, 4096), 1, BF16, 0.05), rand((4096, 512), 2, BF16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c = strp.Context(0)
        c.set_workspace(4096)
        out = torch.empty((512, 512), dtype=BF16, device="cuda")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            with pytest.raises(strp.StrpError) as e:
                c.strp_linear(W, X, 512, out=out)
            out.zero_()
        assert e.value.status == strp.ESTATE and c.ws.numel() == 4096
        want = c.strp_linear(W, X, 512)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            c.strp_linear(W, X, 512, out=out)
        for _ in range(3):
            out.zero_()
            leave_a_failure(c)
            graph.replay()
            assert torch.equal(out, want) and c.poll() == strp.ENOTPD
    torch.cuda.synchronize()


@pytest.mark.parametrize("call", ["gram", "scores", "mask", "energy"])
def test_a_graph_of_any_call_keeps_the_workspace_that_a_larger_call_replaces(call):
    """Captured, then a linear on the same context takes a larger workspace, then replayed: the result of the eager call, and nothing else is written."""
    A = rand((256, 512), 1)
    score, energies, W = torch.empty(256, device="cuda"), torch.zeros(1, dtype=torch.float64, device="cuda"), rand((64, 256), 2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c = strp.Context(0)
        c.set_workspace(4 << 20)
        values = rand(60000, 3)

        def run():
            if call == "gram":
                return c.strp_gram(A, 512)
            if call == "scores":
                c.strp_score_alloc(A, 512, strp.WANDA, score, energies, 0, 1, What=W)
                return score
            if call == "mask":
                return c.strp_mask_topk(values, 777)[1]
            energies.zero_()
            c.strp_weight_energy([A, W], 0.1, 0.1, 1.0, energies)
            return energies

        want = run().clone()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = run()
        size = c.ws.numel()
        c.strp_linear(rand((512, 4096), 1, BF16), rand((4096, 512), 2, BF16), 512)
        assert c.ws.numel() > size
        others = [torch.full((size,), 7, dtype=torch.uint8, device="cuda") for _ in range(4)]
        for _ in range(3):
            got.zero_()
            graph.replay()
            assert torch.equal(got, want) and torch.equal(run(), want)
        assert all(bool((o == 7).all()) for o in others)
    torch.cuda.synchronize()


def test_workspaces_of_graphs_that_are_gone_are_freed():
    """A replaced workspace lasts while a graph may write to it, and no longer than forget_graphs says."""
    A = rand((64, 512), 1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c = strp.Context(0)
        c.set_workspace(1 << 28)
        c.strp_gram(A, 512)
        c.set_workspace(1 << 29)                   # no graph: replaced and freed
        assert not c.kept
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            c.strp_gram(A, 512)
        c.set_workspace(1 << 28)
        c.set_workspace(1 << 27)                   # no graph has this one
        assert [w.numel() for w in c.kept] == [1 << 29]
        del graph
        torch.cuda.synchronize()
        before = torch.cuda.memory_allocated()
        c.forget_graphs()
        assert not c.kept and before - torch.cuda.memory_allocated() == 1 << 29
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            c.strp_gram(A, 512)
        del graph
        torch.cuda.synchronize()
        c.forget_graphs()
        c.set_workspace(1 << 28)
        assert not c.kept
    torch.cuda.synchronize()


# ---- linear ---------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("xt", [BF16, F32])
def test_linear_of_the_weights_that_a_refit_leaves(ctx, xt):
    """A head module's refit onto 45 of 51 channels, then the pruned projection twice: all columns, and the kept ones alone."""
    T, d, out = 600, 51, 37
    C, Y = torch.zeros((d, ld8(T)), dtype=xt, device="cuda"), torch.zeros((out, ld8(T)), device="cuda")
    C[:, :T], Y[:, :T] = rand((d, T), 1, xt), rand((out, T), 2)
    idx = torch.tensor([i for i in range(d) if i % 9 != 4], dtype=torch.int32, device="cuda")
    ctx.ensure_workspace(1 << 24)
    W = torch.zeros((out, d), device="cuda")
    ctx.strp_refit(strp.SIDE_FC2, ctx.strp_gram(C, T, idx=idx), 1.0, Y, C, T, idx, W)
    assert ctx.poll() == strp.OK
    with pytest.raises(strp.StrpError):
        ctx.strp_linear(W, C, T)
    got = ctx.strp_linear(strp.aligned_rows(W), C, T, out=torch.empty((out, ld8(T)), device="cuda"))
    kept = C[idx.long()].contiguous()
    compact = ctx.strp_linear(strp.aligned_rows(W[:, idx.long()]), kept, T, out=torch.empty((out, ld8(T)), device="cuda"))
    w, c = W.double(), C[:, :T].double()
    tol = (d + 4) * U * (w.abs() @ c.abs()) + H(F32) * (w @ c).abs() + 1e-37
    assert ((got[:, :T].double() - w @ c).abs() <= tol).all() and ((compact[:, :T].double() - w @ c).abs() <= tol).all()


# ---- together -------------------------------------------------------------------------------------------------------
def test_the_readme_s_example(ctx):
    """The example of a decoder layer is run as it stands, on a decoder of one layer in fp32, and its perplexity is that of the model in 64 bits: norm before either block, a residual
    round either, a norm before the head.  Every one of the ten results on the longest path is off by at most 400 steps, relative (sums of up to 512 terms, whose errors add up like their
    square root), and passes the earlier ones on with a factor of order one."""
    import os
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")).read()
    code, = [b.split("```")[0] for b in text.split("```python\n")[1:] if "strp_token_logprobs" in b]
    d, f, V, heads, T = 128, 512, 999, 4, 203
    w = {n: rand((r, c), i, F32, c ** -0.5) for i, (n, r, c) in enumerate([("q", d, d), ("k", d, d), ("v", d, d), ("Wo", d, d), ("W1", f, d), ("W2", d, f), ("E", V, d)])}
    b = {n: 0.1 * rand(r, 20 + i) for i, (n, r) in enumerate([("q", d), ("k", d), ("v", d), ("bo", d), ("b1", f), ("b2", d)])}
    norms = {n: (1.0 if n[0] == "g" else 0.0) + 0.5 * rand(d, 30 + i) for i, n in enumerate(("gain1", "bias1", "gain2", "bias2", "gain_f", "bias_f"))}
    H0, starts = rand((d, ld8(T)), 50), [0, 60, T]
    next_ids = torch.randint(0, V, (T,), device="cuda", dtype=torch.int32, generator=torch.Generator(device="cuda").manual_seed(2))
    next_ids[59] = next_ids[T - 1] = -1
    names = dict(ctx=ctx, strp=strp, torch=torch, H=H0, T=T, heads=heads, kv_heads=heads, starts=torch.tensor(starts, dtype=torch.int32, device="cuda"), next_ids=next_ids,
                 qkv=[(w[n], b[n]) for n in "qkv"], **{n: w[n] for n in ("Wo", "W1", "W2", "E")}, **{n: b[n] for n in ("bo", "b1", "b2")}, **norms)
    exec(code, names)

    D = lambda t: t.double()
    norm = lambda x, i: (x - x.mean(0)) / torch.sqrt(x.var(0, unbiased=False) + 1e-5) * D(norms["gain" + i])[:, None] + D(norms["bias" + i])[:, None]
    x = D(H0)[:, :T]
    n = norm(x, "1")
    q, k, v = (D(w[m]) @ n + D(b[m])[:, None] for m in "qkv")
    c = torch.cat([attention_exact(q[:, a:e], k[:, a:e], v[:, a:e], heads, list(range(heads)), [0, e - a], (d // heads) ** -0.5, 0.0)[0] for a, e in zip(starts, starts[1:])], 1)
    x = x + D(w["Wo"]) @ c + D(b["bo"])[:, None]
    x = x + D(w["W2"]) @ (D(w["W1"]) @ norm(x, "2") + D(b["b1"])[:, None]).clamp_min(0) + D(b["b2"])[:, None]
    logp = torch.log_softmax(D(w["E"]) @ norm(x, "_f"), 0)
    scored = next_ids >= 0
    want = torch.where(scored, logp.gather(0, next_ids.clamp_min(0).long()[None])[0], 0.0)
    assert float((names["out"]["logp"].double() - want).norm() / want.norm()) <= 10 * 400 * U
    assert abs(float(names["perplexity"]) / math.exp(-float(want.sum()) / int(scored.sum())) - 1) <= 10 * 400 * U * float(want.abs().mean()) + 4 * U


# ---- every kernel that there is ----------------------------------------------------------------------------------------
FP32_TYPES = [(w, x, y) for w, x in ((F32, F32), (F32, BF16), (BF16, F32)) for y in (F32, BF16)]
IDS = lambda v: "x".join(map(str, v)) if isinstance(v[0], int) else "-".join(str(t)[6:] for t in v)


@pytest.mark.parametrize("types", [(BF16, BF16, BF16), (BF16, BF16, F32)], ids=IDS)
@pytest.mark.parametrize("size", sizes.LINEAR_BF16, ids=IDS)
def test_linear_in_every_tile_of_bf16(ctx, size, types):
    linear_case(ctx, *size, types, strp.ACT_RELU, True, True)
    linear_case(ctx, *size, types, strp.ACT_GELU, True, False)
    linear_as_a_whole(ctx, *size, types)


@pytest.mark.parametrize("types", FP32_TYPES, ids=IDS)
@pytest.mark.parametrize("size", sizes.LINEAR_F32, ids=IDS)
def test_linear_in_every_tile_of_fp32(ctx, size, types):
    linear_case(ctx, *size, types, strp.ACT_RELU, True, True)
    linear_as_a_whole(ctx, *size, types)


def linear_as_a_whole(c, M, K, T, types):
    """Relative to the result, in the 2-norm.  The K steps of a sum are off independently of each other, each by less than U of a partial sum that is no larger than the
    whole in the mean: sqrt(K) U together, and a rounding of the output.  (An operand of fp32 that met the products rounded to bf16 would be off by 1.6e-3.)"""
    wt, xt, yt = types
    W, X = padded(M, K, 11, wt, 0.05, ld8(K))[:, :K], padded(K, T, 12, xt)
    got = c.strp_linear(W, X, T, out=torch.empty((M, ld8(T)), dtype=yt, device="cuda"))[:, :T].double()
    want = W.double() @ X[:, :T].double()
    assert float((got - want).norm() / want.norm()) <= (math.sqrt(K) + 8) * U + H(yt), (M, K, T, types)


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("wide", sorted(sizes.NORM_TOKENS["f32"]))
def test_layer_norm_in_every_kernel(ctx, wide, dt):
    name = "bf16" if dt == BF16 else "f32"
    for d, T in sizes.NORM[name]:
        if T != sizes.NORM_TOKENS[name][wide]:
            continue
        Y = torch.full((d, ld8(T)), 7.0, dtype=dt, device="cuda")
        norm_check(ctx, padded(d, T, 5, dt), T, 1 + 0.1 * rand(d, 6), rand(d, 7), out=Y)
        assert (Y[:, T:] == 7.0).all()


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("d,T", sizes.NORM_TALL)
def test_layer_norm_of_more_channels_than_registers_hold(ctx, d, T, dt):
    Y = torch.full((d, ld8(T)), 7.0, dtype=dt, device="cuda")
    norm_check(ctx, padded(d, T, 5, dt), T, 1 + 0.1 * rand(d, 6), rand(d, 7), out=Y)
    assert (Y[:, T:] == 7.0).all()
    X = padded(d, T, 6, dt)
    assert norm_check(ctx, X, T, None, None, out=X) is X


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("V,T,n_top", sizes.LOGPROBS)
def test_token_logprobs_in_every_kernel(ctx, V, T, n_top, dt):
    X = padded(V, T, V + T, dt, 3.0)
    target = torch.randint(-2, V + 2, (T,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(torch.int32)
    logprobs_check(ctx, X, T, target, n_top)


# ---- offsets and maps that are wrong ------------------------------------------------------------------------------------
@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("starts", [[-100, 50, 300], [0, 5000, 300], [200, 100, 50], [7, 7, 7], [300, 0, 301], [-(2 ** 31), 2 ** 31 - 1, -5], [40, 260]], ids=str)
def test_attention_reads_and_writes_its_own_rows_and_tokens_whatever_the_offsets_say(ctx, fast, starts, dt):
    """Q, K, V and C lie inside larger buffers: NaN round K and V, 7 round C.  What is written is finite, so no key or value came from outside, and nothing is written outside."""
    T, dh, heads, kv, edge = 300, 40, 4, 3, 16
    big = {n: torch.full((rows * dh + 2 * edge, ld8(T) + 4 * edge), fill, dtype=dt, device="cuda") for n, rows, fill in
           (("Q", heads, 0.0), ("K", kv, float("nan")), ("V", kv, float("nan")), ("C", heads, 7.0))}
    inner = {n: b[edge:-edge, edge:-edge] for n, b in big.items()}
    for i, n in enumerate("QKV"):
        inner[n][:, :T] = rand((inner[n].shape[0], T), i, dt)
        inner[n][:, T:] = float("nan")
    kv_of = torch.tensor([-5, 900, 2 ** 31 - 1, -(2 ** 31)], dtype=torch.int32, device="cuda")
    for c in (ctx, fast):
        inner["C"][:] = 7.0
        c.strp_attention(inner["Q"], inner["K"], inner["V"], T, heads, kv, torch.tensor(starts, dtype=torch.int32, device="cuda"), kv_of_head=kv_of, out=inner["C"])
        inside = inner["C"][:, :T].clone()
        assert torch.isfinite(inside).all()
        inner["C"][:, :T] = 7.0
        assert (big["C"] == 7.0).all()
        if starts == [40, 260]:                    # right offsets: heads -5 and -2^31 have key-value head 0, the others the last
            right = torch.full((heads * dh, ld8(T)), 7.0, dtype=dt, device="cuda")
            c.strp_attention(inner["Q"], inner["K"], inner["V"], T, heads, kv, torch.tensor(starts, dtype=torch.int32, device="cuda"),
                             kv_of_head=torch.tensor([0, kv - 1, kv - 1, 0], dtype=torch.int32, device="cuda"), out=right)
            assert torch.equal(inside, right[:, :T]) and (inside[:, :40] == 7.0).all() and (inside[:, 260:] == 7.0).all() and not (inside[:, 40:260] == 7.0).any()
