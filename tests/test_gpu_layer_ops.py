"""The decoder layer's operators against their definitions in 64 bits: linear, layer norm, attention, token log probabilities.

U = 2^-23 bounds what one fp32 operation or one step of a matrix-core sum adds, relative to the magnitudes that meet there; H(t) is half a
step of an output of type t.  Every bound is the count of such steps times the sum of magnitudes, worked out beside its use."""
import math

import pytest
import torch

from paper_2510_03246_amd import strp

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


def rand(shape, seed, dt=F32, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dt)


def padded(rows, T, seed, dt, scale=1.0, ld=None, fill=float("nan")):
    """[rows x ld] with data in the first T columns and `fill` behind them."""
    x = torch.full((rows, ld or ld8(T)), fill, dtype=dt, device="cuda")
    x[:, :T] = rand((rows, T), seed, dt, scale)
    return x


def close(got, want, tol, what=""):
    got = got.double()
    bad = ~((got - want).abs() <= tol)
    assert not bad.any(), (what, int(bad.sum()), "worst", float(((got - want).abs() / tol.clamp_min(1e-300))[bad].max()), bad.nonzero()[:3].tolist())


# ---- linear ---------------------------------------------------------------------------------------------------------
def linear_reference(W, X, T, b, act, R, out_dtype):
    W, X = W.double(), X[:, :T].double()
    z, mag = W @ X, W.abs() @ X.abs()
    if b is not None:
        z, mag = z + b.double()[:, None], mag + b.double().abs()[:, None]
    # K products and sums and the bias; gelu has slope below 1.13 and is itself good to a few units, relative
    tol = (W.shape[1] + 4) * U * mag
    if act == strp.ACT_RELU:
        z = z.clamp_min(0)
    elif act == strp.ACT_GELU:
        z = z * 0.5 * torch.erfc(-z / math.sqrt(2))
        tol = 1.13 * tol + 16 * U * z.abs()
    if R is not None:
        z = z + R[:, :T].double()
        tol = tol + U * (z.abs() + R[:, :T].double().abs())
    return z, tol * (1 + H(out_dtype)) + H(out_dtype) * z.abs() + 1e-37


SIZES = [(1, 1, 1), (3, 5, 7), (64, 64, 64), (129, 257, 130), (200, 4915, 96), (768, 768, 1), (300, 1000, 17), (257, 8, 1025), (65, 33, 200), (512, 768, 4), (1000, 72, 33),
         (1013, 1000, 5), (40, 2000, 12), (33, 16, 3000)]
TYPES = [(BF16, BF16, BF16), (BF16, BF16, F32), (F32, F32, F32), (F32, BF16, BF16), (BF16, F32, F32)]


def linear_case(ctx, M, K, T, types, act, bias, res, seed=0, ldw=None, ldx=None):
    wt, xt, yt = types
    W = padded(M, K, seed + 1, wt, 0.05, ldw or ld8(K))[:, :K]        # NaN behind the rows
    X = padded(K, T, seed + 2, xt, ld=ldx)
    b = rand(M, seed + 3) if bias else None
    R = padded(M, T, seed + 4, yt) if res else None
    Y = torch.full((M, ld8(T)), 7.0, dtype=yt, device="cuda")
    got = ctx.strp_linear(W, X, T, bias=b, act=act, residual=R, out=Y)
    want, tol = linear_reference(W, X, T, b, act, R, yt)
    close(got[:, :T], want, tol, (M, K, T, types, act, bias, res))
    assert (got[:, T:] == 7.0).all()


@pytest.mark.parametrize("types", TYPES, ids=lambda t: "-".join(str(x)[6:] for x in t))
@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_linear(ctx, size, types):
    for act, bias, res in ((strp.ACT_NONE, False, False), (strp.ACT_RELU, True, True), (strp.ACT_GELU, True, False)):
        linear_case(ctx, *size, types, act, bias, res)


@pytest.mark.parametrize("types", [TYPES[0], TYPES[2]], ids=["bf16", "f32"])
@pytest.mark.parametrize("size", [(1536, 800, 1300), (2304, 264, 2049), (260, 1100, 4100), (4096, 40, 515)], ids=lambda s: "x".join(map(str, s)))
def test_linear_of_many_tiles(ctx, size, types):
    linear_case(ctx, *size, types, strp.ACT_NONE, True, True)


@pytest.mark.parametrize("T", [1, 5, 8, 9, 15, 16, 17, 31, 32, 33, 63, 64])
@pytest.mark.parametrize("M,K", [(70, 4101), (33, 2049), (5000, 3403), (2048, 2048)])
def test_linear_of_few_tokens(ctx, M, K, T):
    linear_case(ctx, M, K, T, TYPES[0], strp.ACT_RELU, True, True)
    linear_case(ctx, M, K, T, TYPES[1], strp.ACT_NONE, True, False)


def test_linear_into_its_residual(ctx):
    for T in (5, 300):
        W, X, R = rand((96, 64), 1, BF16, 0.1), rand((64, ld8(T)), 2, BF16), rand((96, ld8(T)), 3, BF16)
        want, tol = linear_reference(W, X, T, None, strp.ACT_NONE, R.clone(), BF16)
        assert ctx.strp_linear(W, X, T, residual=R, out=R) is R
        close(R[:, :T], want, tol)


def test_linear_with_wide_strides(ctx):
    linear_case(ctx, 70, 90, 50, TYPES[0], strp.ACT_RELU, True, False, ldw=160, ldx=1024)
    linear_case(ctx, 70, 90, 50, TYPES[2], strp.ACT_RELU, True, False, ldw=160, ldx=1024)


@pytest.mark.parametrize("T", [3, 200])
def test_linear_beyond_32_bit_offsets(ctx, T):
    """Rows 2^26 values apart: the last of 80 lies 5.3e9 values into X, and the result's the same."""
    ld = 1 << 26
    X, Y = torch.empty((80, ld), dtype=BF16, device="cuda"), torch.empty((80, ld), dtype=BF16, device="cuda")
    X[:, :T] = rand((80, T), 1, BF16)
    W = rand((80, 80), 2, BF16)
    ctx.strp_linear(W, X, T, out=Y)
    want, tol = linear_reference(W, X, T, None, strp.ACT_NONE, None, BF16)
    close(Y[:, :T], want, tol)


def test_linear_lets_what_is_not_finite_through(ctx):
    for T, dt in ((3, BF16), (200, BF16), (200, F32)):
        W, X = rand((40, 64), 1, dt), rand((64, ld8(T)), 2, dt)
        X[5, 1] = float("inf")
        X[9, 2] = float("nan")
        Y = ctx.strp_linear(W, X, T, act=strp.ACT_RELU)
        keep = [t for t in range(T) if t not in (1, 2)]
        want, tol = linear_reference(W, X, T, None, strp.ACT_RELU, None, dt)
        close(Y[:, keep], want[:, keep], tol[:, keep])
        assert torch.isnan(Y[:, 2]).all()
        up = W[:, 5] > 0
        assert (Y[up, 1] == float("inf")).all() and (Y[~up, 1] == 0).all()


# ---- layer norm -----------------------------------------------------------------------------------------------------
def norm_check(ctx, X, T, gain, bias, eps=1e-5, out=None):
    d = X.shape[0]
    x = X[:, :T].double().clone()
    Y = ctx.strp_layer_norm(X, T, gain=gain, bias=bias, eps=eps, out=out)
    mean = x.mean(0)
    c = x - mean
    r = 1 / torch.sqrt((c * c).mean(0) + eps)
    g, b = (v.double()[:, None] if v is not None else v0 for v, v0 in ((gain, 1.0), (bias, 0.0)))
    n = c * r * g
    # the mean is d sums of magnitudes; it moves every deviation, and the variance by its square and by d + 8 relative steps
    dm = (d + 2) * U * x.abs().mean(0)
    tol = (r * g * (dm + U * (x.abs() + mean.abs()))).abs() + n.abs() * ((d + 8) * U + (dm * r) ** 2 + 2 * dm * r) + 2 * U * (n.abs() + (n + b).abs())
    close(Y[:, :T], n + b, tol * (1 + H(X.dtype)) + H(X.dtype) * (n + b).abs() + 1e-37, (d, T, X.dtype))
    return Y


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("d,T", [(1, 1), (2, 9), (48, 1), (768, 5), (777, 130), (4096, 70), (64, 3001), (5000, 8), (9001, 33), (768, 2048), (130, 64), (2048, 40)])
def test_layer_norm(ctx, d, T, dt):
    X = padded(d, T, 5, dt)
    Y = torch.full((d, ld8(T)), 7.0, dtype=dt, device="cuda")
    norm_check(ctx, X, T, 1 + 0.1 * rand(d, 6), rand(d, 7), out=Y)
    assert (Y[:, T:] == 7.0).all()
    norm_check(ctx, X, T, None, None)


@pytest.mark.parametrize("dt", [BF16, F32])
def test_layer_norm_far_from_zero_and_in_place(ctx, dt):
    """Means a thousand times the spread, a token of equal values, one token not finite; the result in place of the input."""
    X = padded(512, 90, 1, dt)
    X[:, :40] += 1000.0
    X[:, 40] = 3.0
    clean = X.clone()
    X[7, 50] = float("inf")
    Z = ctx.strp_layer_norm(X, 90, gain=None, bias=None)
    assert torch.isnan(Z[:, 50]).any()
    Y = norm_check(ctx, clean, 90, None, rand(512, 2), out=clean)
    assert Y is clean
    keep = [t for t in range(90) if t != 50]
    Z2 = ctx.strp_layer_norm(torch.where(torch.isfinite(X), X, 0.0), 90)
    assert torch.equal(Z[:, keep], Z2[:, keep])


# ---- attention ------------------------------------------------------------------------------------------------------
def attention_reference(Q, K, V, heads, kv_of, starts, scale):
    """result and bound; NaN outside the sequences"""
    dt, dh = Q.dtype, Q.shape[0] // heads
    T = Q.shape[1]
    out = torch.full((heads * dh, T), float("nan"), dtype=torch.float64, device="cuda")
    tol = torch.zeros_like(out)
    for a, e in zip(starts, starts[1:]):
        if a == e:
            continue
        n = e - a
        seen = torch.ones((n, n), dtype=torch.bool, device="cuda").tril()
        for h in range(heads):
            r, rk = slice(h * dh, (h + 1) * dh), slice(kv_of[h] * dh, (kv_of[h] + 1) * dh)
            q, k, v = Q[r, a:e].double(), K[rk, a:e].double(), V[rk, a:e].double()
            s = torch.where(seen, scale * (q.t() @ k), -math.inf)
            p = torch.softmax(s, 1)
            o = v @ p.t()
            # a score is off by dh + 4 steps of its magnitudes, its probability by twice the largest of these of its row (the maximum's and its own), relative;
            # the probabilities may be rounded to bf16, the sums have n terms more
            mag = torch.where(seen, scale * (q.abs().t() @ k.abs()), 0.0).max(1).values
            rel = 2 * (dh + 4) * U * mag + 16 * U + n * U + (H(BF16) if dt == BF16 else 0.0)
            out[r, a:e] = o
            tol[r, a:e] = 2 * rel * (v.abs() @ p.t()) + H(dt) * o.abs() + 1e-37
    return out, tol


def attention_case(ctx, lens, heads, kv, dh, dt, first=0, behind=0, kv_of=None, scale=None, seed=0, spread=1.5):
    starts = [first]
    for n in lens:
        starts.append(starts[-1] + n)
    T = starts[-1] + behind
    Q, K, V = (padded((heads if i == 0 else kv) * dh, T, seed + i, dt, spread if i < 2 else 1.0) for i in range(3))
    for x in (Q, K, V):
        x[:, :first] = float("nan")               # tokens of no sequence hold what is not finite
        x[:, starts[-1]:] = float("inf")
    C = torch.full((heads * dh, ld8(T)), 7.0, dtype=dt, device="cuda")
    kvt = torch.tensor(kv_of, dtype=torch.int32, device="cuda") if kv_of else None
    whole = first == 0 and behind == 0 and len(lens) == 1 and seed % 2
    ctx.strp_attention(Q, K, V, T, heads, kv, None if whole else torch.tensor(starts, dtype=torch.int32, device="cuda"), kv_of_head=kvt, scale=scale, out=C)
    want, tol = attention_reference(Q[:, :T], K[:, :T], V[:, :T], heads, kv_of or [h // (heads // kv) for h in range(heads)], starts, scale or dh ** -0.5)
    inside = slice(first, starts[-1])
    close(C[:, inside], want[:, inside], tol[:, inside], (lens, heads, kv, dh, dt))
    assert (C[:, :first] == 7.0).all() and (C[:, starts[-1]:] == 7.0).all()


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("lens", [[1], [2], [31], [64], [65], [127], [129], [300], [1, 1, 1], [0, 5, 0, 0, 60, 0], [128, 128], [130, 1, 1, 1, 250, 63], [33] * 9], ids=str)
def test_attention_lengths(ctx, lens, dt):
    attention_case(ctx, lens, 3, 3, 64, dt)
    attention_case(ctx, lens, 2, 1, 80, dt, first=3, behind=5, seed=1)


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("dh", [1, 7, 8, 16, 31, 32, 33, 48, 63, 64, 65, 80, 96, 97, 100, 127, 128])
def test_attention_head_widths(ctx, dh, dt):
    attention_case(ctx, [70, 1, 140], 4, 2, dh, dt)


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("heads,kv,kv_of", [(8, 1, None), (6, 3, None), (5, 5, None), (7, 3, [0, 0, 0, 1, 2, 2, 2]), (3, 4, [3, 0, 3])])
def test_attention_heads_in_groups(ctx, heads, kv, kv_of, dt):
    attention_case(ctx, [90, 77], heads, kv, 64, dt, kv_of=kv_of)
    attention_case(ctx, [200], heads, kv, 128, dt, kv_of=kv_of, seed=1)


@pytest.mark.parametrize("dt,n", [(BF16, 5000), (F32, 3001)])
def test_attention_long(ctx, dt, n):
    attention_case(ctx, [n], 2, 1, 128, dt)
    attention_case(ctx, [700, n - 900, 200], 1, 1, 64, dt, first=1)


@pytest.mark.parametrize("dt", [BF16, F32])
def test_attention_scales_and_peaked_scores(ctx, dt):
    attention_case(ctx, [150], 2, 2, 64, dt, scale=1.0)              # scores of +- 50: one key takes almost all
    attention_case(ctx, [150], 2, 2, 64, dt, scale=1e-6)             # all keys alike
    attention_case(ctx, [150], 2, 2, 64, dt, spread=12.0)


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_what_a_token_does_not_see_has_no_part(ctx, dt, bad):
    """Token 100 of the second of three sequences holds what is not finite in K and V: the other sequences and the tokens before it are as they were, bit
    for bit; from it on, its head's results show it."""
    lens, dh = [70, 200, 90], 64
    starts = torch.tensor([0, 70, 270, 360], dtype=torch.int32, device="cuda")
    Q, K, V = (rand((2 * dh, 360), i, dt) for i in range(3))
    clean = ctx.strp_attention(Q, K, V, 360, 2, 2, starts).clone()
    V2, K2 = V.clone(), K.clone()
    V2[5, 170] = bad
    got = ctx.strp_attention(Q, K, V2, 360, 2, 2, starts)
    rows = torch.arange(2 * dh, device="cuda") != 5
    assert torch.equal(got[rows], clean[rows])
    assert torch.equal(got[5, :170], clean[5, :170]) and torch.equal(got[5, 270:], clean[5, 270:])
    assert not torch.isfinite(got[5, 170:270]).any()
    if bad == bad:
        assert (got[5, 170:200] == bad).all()
    K2[5, 170] = bad
    got = ctx.strp_attention(Q, K2, V, 360, 2, 2, starts)
    assert torch.equal(got[:, :170], clean[:, :170]) and torch.equal(got[:, 270:], clean[:, 270:]) and torch.equal(got[dh:], clean[dh:])
    Q2 = Q.clone()
    Q2[3, 100] = bad
    got = ctx.strp_attention(Q2, K, V, 360, 2, 2, starts)
    keep = [t for t in range(360) if t != 100]
    assert torch.equal(got[:, keep], clean[:, keep]) and torch.equal(got[dh:], clean[dh:])


def test_attention_lowest_values(ctx):
    """Values of the type's lowest magnitude and of its largest negative in tokens that are not seen."""
    for dt in (BF16, F32):
        low = torch.finfo(dt).min
        Q, K, V = (rand((64, 200), i, dt) for i in range(3))
        starts = torch.tensor([0, 90, 200], dtype=torch.int32, device="cuda")
        clean = ctx.strp_attention(Q, K, V, 200, 1, 1, starts).clone()
        V[:, 80:90] = low
        K[:, 80:90] = torch.finfo(dt).max
        got = ctx.strp_attention(Q, K, V, 200, 1, 1, starts)
        assert torch.equal(got[:, :80], clean[:, :80]) and torch.equal(got[:, 90:], clean[:, 90:])


def test_attention_beyond_32_bit_offsets(ctx):
    ld, T = 1 << 25, 150
    for dt in (BF16, F32):
        Q, K, V = (torch.empty((128, ld), dtype=dt, device="cuda") for _ in range(3))
        for i, x in enumerate((Q, K, V)):
            x[:, :T] = rand((128, T), i, dt)
        C = torch.empty((128, ld), dtype=dt, device="cuda")
        ctx.strp_attention(Q, K, V, T, 1, 1, None, out=C)
        want, tol = attention_reference(*(x[:, :T].contiguous() for x in (Q, K, V)), 1, [0], [0, T], 128 ** -0.5)
        close(C[:, :T], want, tol)


def test_attention_wrong_offsets_stay_in_bounds(ctx):
    """Offsets out of order or out of range give wrong results and nothing else: every read is held to the tokens there are."""
    Q, K, V = (rand((64, 304), i, BF16) for i in range(3))
    kv = torch.tensor([-5, 900], dtype=torch.int32, device="cuda")
    for starts in ([-100, 50, 300], [0, 5000, 300], [200, 100, 50], [7, 7, 7], [300, 0, 301]):
        ctx.strp_attention(Q, K[:32], V[:32], 300, 2, 1, torch.tensor(starts, dtype=torch.int32, device="cuda"), kv_of_head=kv)
    torch.cuda.synchronize()


# ---- token log probabilities ------------------------------------------------------------------------------------------
def logprobs_check(ctx, X, T, target, n_top, entropy=True):
    V = X.shape[0]
    x = X[:, :T].double()
    got = ctx.strp_token_logprobs(X, T, target, entropy=entropy, n_top=n_top)
    lse = torch.logsumexp(x, 0)
    p = torch.softmax(x, 0)
    logp = x - lse
    # log p: the two differences, the logarithm, and a sum of V terms whose chain is at most 32 entries, 8 merges of a workgroup and of a wavefront's, and
    # 2^16 slices at most: 128 + V / 8192 steps, relative, of a sum that is at least 1; the entropy's sum is of terms that add up to H / ln 2 + log2 of the sum
    steps = 128 + V / 8192
    tol = lambda v: U * (2 * v.abs() + 2 * lse.abs().clamp_min(1) + steps + (x.amax(0) - lse).abs())
    if target is not None:
        y = target.long()
        ok = (y >= 0) & (y < V)
        want = torch.where(ok, logp.gather(0, y.clamp(0, V - 1)[None])[0], 0.0)
        fin = torch.isfinite(want)
        close(got["logp"][fin], want[fin], tol(want)[fin], "logp")
        assert (got["logp"][~fin].double() == want[~fin]).all()
    if entropy:
        want = -torch.where(p > 0, p * logp, 0.0).sum(0)
        close(got["entropy"], want, U * (steps * (2 + 2 * want) + 4 * (x.amax(0) - lse).abs()), "entropy")
    if n_top:
        order = torch.sort(x, dim=0, descending=True, stable=True)
        assert torch.equal(got["top_ids"].long(), order.indices[:n_top])
        want = order.values[:n_top] - lse
        fin = torch.isfinite(want)
        close(got["top_logp"][fin], want[fin], tol(want)[fin], "top_logp")
        assert (got["top_logp"][~fin].double() == want[~fin]).all()
    return got


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("V,T", [(1, 1), (2, 3), (7, 9), (64, 64), (300, 65), (1000, 1), (1031, 513), (5000, 40), (50000, 1), (50001, 8), (50000, 17), (20000, 130), (130001, 3), (600, 4100)])
def test_token_logprobs(ctx, V, T, dt):
    X = padded(V, T, V + T, dt, 3.0)
    target = torch.randint(-2, V + 2, (T,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(torch.int32)
    logprobs_check(ctx, X, T, target, min(V, 5))
    logprobs_check(ctx, X, T, target, 0)
    logprobs_check(ctx, X, T, None, min(V, 16), entropy=False)
    logprobs_check(ctx, X, T, None, 0)


@pytest.mark.parametrize("dt", [BF16, F32])
@pytest.mark.parametrize("kind", ["equal", "few", "masked", "ascending", "descending", "far"])
@pytest.mark.parametrize("V,T", [(40, 5), (3000, 70), (40000, 2)])
def test_token_logprobs_edges(ctx, V, T, kind, dt):
    """Ties everywhere, masked entries, the best ones all in one stream at either end, logits far from zero."""
    g = torch.Generator(device="cuda").manual_seed(V)
    X = torch.zeros((V, ld8(T)), device="cuda")
    if kind == "few":
        X += torch.randint(-2, 3, X.shape, generator=g, device="cuda")
    elif kind == "masked":
        X += torch.randn(X.shape, generator=g, device="cuda")
        X[torch.rand(X.shape, generator=g, device="cuda") < 0.9] = -math.inf
        X[V // 2] = 1.0
        X[:, 0] = -math.inf
        X[min(V - 1, 17), 0] = -2.0
    elif kind == "ascending":
        X += torch.arange(V, device="cuda")[:, None] * (2.0 ** -10)
    elif kind == "descending":
        X -= torch.arange(V, device="cuda")[:, None] * (2.0 ** -10)
    elif kind == "far":
        X += 80000.0 * torch.randn(X.shape, generator=g, device="cuda")
    logprobs_check(ctx, X.to(dt), T, torch.full((T,), V - 1, dtype=torch.int32, device="cuda"), 16)


def test_token_logprobs_of_what_is_not_finite(ctx):
    for dt in (BF16, F32):
        X = rand((3000, 40), 3, dt)
        clean = ctx.strp_token_logprobs(X, 40, torch.zeros(40, dtype=torch.int32, device="cuda"), n_top=3)
        X[2000, 7] = float("nan")
        X[1500, 9] = float("inf")
        got = ctx.strp_token_logprobs(X, 40, torch.zeros(40, dtype=torch.int32, device="cuda"), n_top=3)
        keep = [t for t in range(40) if t not in (7, 9)]
        for name in clean:
            assert torch.equal(got[name][..., keep], clean[name][..., keep])
        assert torch.isnan(got["logp"][7]) and torch.isnan(got["entropy"][7]) and (got["top_ids"][:, 7] == -1).all() and torch.isnan(got["top_logp"][:, 7]).all()
        assert torch.isnan(got["entropy"][9]) and int(got["top_ids"][0, 9]) == 1500
    X = torch.full((50, 8), -math.inf, device="cuda")
    assert torch.isnan(ctx.strp_token_logprobs(X, 8, torch.zeros(8, dtype=torch.int32, device="cuda"))["logp"]).all()


def test_token_logprobs_beyond_32_bit_offsets(ctx):
    ld, V = 1 << 24, 330
    X = torch.empty((V, ld), dtype=BF16, device="cuda")
    X[:, :3] = rand((V, 3), 1, BF16, 3.0)
    logprobs_check(ctx, X, 3, torch.tensor([0, 329, 200], dtype=torch.int32, device="cuda"), 7)


# ---- together ---------------------------------------------------------------------------------------------------------
def layer_weights(d, f, V, dt):
    w = {n: rand((r, c), i, dt, c ** -0.5) for i, (n, r, c) in enumerate([("q", d, d), ("k", d, d), ("v", d, d), ("o", d, d), ("fc1", f, d), ("fc2", d, f), ("head", V, d)])}
    w.update({n + "_b": 0.1 * rand(r, 20 + i) for i, (n, r) in enumerate([("q", d), ("k", d), ("v", d), ("o", d), ("fc1", f), ("fc2", d)])})
    w.update({n: (1.0 if n[0] == "g" else 0.0) + 0.1 * rand(d, 30 + i) for i, n in enumerate(("g1", "b1", "g2", "b2"))})
    return w


def layer(ctx, w, X, T, heads, starts, target):
    """One decoder layer and the model's head: what the head module and the FFN module read, and the tokens' log probabilities."""
    n1 = ctx.strp_layer_norm(X, T, w["g1"], w["b1"])
    q, k, v = (ctx.strp_linear(w[n], n1, T, bias=w[n + "_b"]) for n in "qkv")
    c = ctx.strp_attention(q, k, v, T, heads, heads, starts)
    r = ctx.strp_linear(w["o"], c, T, bias=w["o_b"], residual=X)
    n2 = ctx.strp_layer_norm(r, T, w["g2"], w["b2"])
    a = ctx.strp_linear(w["fc1"], n2, T, bias=w["fc1_b"], act=strp.ACT_RELU)
    r = ctx.strp_linear(w["fc2"], a, T, bias=w["fc2_b"], residual=r, out=r)
    logits = ctx.strp_linear(w["head"], r, T)
    return dict(C=c, N2=n2, R=r, **ctx.strp_token_logprobs(logits, T, target, n_top=3))


def layer_reference(w, X, T, heads, starts, target):
    w = {n: t.double() for n, t in w.items()}
    X = X[:, :T].double()
    norm = lambda x, g, b: (x - x.mean(0)) / torch.sqrt(x.var(0, unbiased=False) + 1e-5) * g[:, None] + b[:, None]
    lin = lambda n, x: w[n] @ x + w[n + "_b"][:, None]
    n1 = norm(X, w["g1"], w["b1"])
    c, _ = attention_reference(lin("q", n1), lin("k", n1), lin("v", n1), heads, list(range(heads)), starts, (X.shape[0] // heads) ** -0.5)
    r = lin("o", c) + X
    n2 = norm(r, w["g2"], w["b2"])
    r = lin("fc2", lin("fc1", n2).clamp_min(0)) + r
    logits = w["head"] @ r
    logp = logits - torch.logsumexp(logits, 0)
    return dict(C=c, N2=n2, R=r, logp=logp.gather(0, target.long()[None])[0], entropy=-(logp.exp() * logp).sum(0))


@pytest.mark.parametrize("dt", [BF16, F32])
def test_a_decoder_layer(ctx, dt):
    """The operators one after the other as a calibration run calls them, then the head module's scores from what they made.  Relative errors of the whole:
    each of the seven results on the longest path is off by at most 10 half-steps of its type or 400 fp32 steps (sums of up to 512 terms, whose errors add up like
    their square root), and every one passes the earlier ones on with a factor of order one: 70 H(bf16), 2800 U."""
    d, f, V, heads, lens = 128, 512, 999, 4, [40, 1, 90, 200]
    T = sum(lens)
    starts = [0, 40, 41, 131, 331]
    w = layer_weights(d, f, V, dt)
    X = padded(d, T, 50, dt)
    target = torch.randint(0, V, (T,), device="cuda", dtype=torch.int32, generator=torch.Generator(device="cuda").manual_seed(2))
    got = layer(ctx, w, X, T, heads, torch.tensor(starts, dtype=torch.int32, device="cuda"), target)
    want = layer_reference(w, X, T, heads, starts, target)
    bound = 70 * H(BF16) if dt == BF16 else 2800 * U
    for name, ref in want.items():
        g = got[name][..., :T].double()
        assert float((g - ref).norm() / ref.norm()) <= bound, name
    energies, score = torch.zeros(1, dtype=torch.float64, device="cuda"), torch.empty(heads, device="cuda")
    ctx.ensure_workspace(1 << 20)
    ctx.strp_score_alloc(got["C"], T, strp.WANDA, score, energies, 0, 1, group=d // heads, What=w["o"])
    c, n2 = got["C"][:, :T].double(), (w["o"].double() ** 2).sum(0)
    ref = (n2 * (c * c).sum(1)).reshape(heads, -1).sum(1)
    assert torch.allclose(score.double(), ref, rtol=1e-5)


def test_captured_and_replayed(ctx):
    """The whole layer in a graph on new inputs: every replay has the bits of the eager run, with eager work between the replays."""
    d, f, V, heads, T = 128, 512, 4001, 4, 203
    w = layer_weights(d, f, V, BF16)
    starts = torch.tensor([0, 60, 203], dtype=torch.int32, device="cuda")
    target = torch.arange(T, device="cuda", dtype=torch.int32)
    X = rand((d, ld8(T)), 1, BF16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        own = strp.Context(0)
        own.set_workspace(1 << 26)
        layer(own, w, X, T, heads, starts, target)
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = layer(own, w, X, T, heads, starts, target)
    for seed in range(4):
        X.copy_(rand((d, ld8(T)), seed, BF16))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        kept = {n: t.clone() for n, t in got.items()}
        eager = layer(ctx, w, X, T, heads, starts, target)
        torch.cuda.synchronize()
        for n in kept:
            assert torch.equal(kept[n][..., :T], eager[n][..., :T]), (n, seed)


def test_a_graph_keeps_the_workspace_that_a_larger_call_replaces(ctx):
    W, X = rand((512, 4096), 1, BF16, 0.05), rand((4096, 128), 2, BF16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        own = strp.Context(0)
        want = own.strp_linear(W, X, 128)
        size = own.ws.numel()
        assert size >= own.lib.strp_linear_workspace_bytes(512, 4096, 128, strp.BF16, strp.BF16) > 0
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            got = own.strp_linear(W, X, 128)
        own.ensure_workspace(8 * size)
        others = [torch.full((size,), 7, dtype=torch.uint8, device="cuda") for _ in range(4)]
        for _ in range(3):
            got.zero_()
            graph.replay()
            assert torch.equal(own.strp_linear(W, X, 128), want) and torch.equal(got, want)
        assert all(bool((o == 7).all()) for o in others)
    torch.cuda.synchronize()


def test_outputs_come_from_the_memory_of_the_context_s_stream(ctx):
    """Called under another stream than its own, a context takes its outputs where its own stream's work is in order."""
    W, X = rand((64, 96), 1, BF16), rand((96, 200), 2, BF16)
    want = ctx.strp_linear(W, X, 200)
    tops = ctx.strp_token_logprobs(want, 200, n_top=3)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        y = ctx.strp_linear(W, X, 200)
        t = ctx.strp_token_logprobs(y, 200, n_top=3)
    torch.cuda.synchronize()
    assert torch.equal(y, want) and all(torch.equal(t[n], tops[n]) for n in tops)


def test_results_do_not_depend_on_the_workspace_or_the_run(ctx):
    d, f, V, heads, T = 128, 512, 4001, 4, 203
    w, X = layer_weights(d, f, V, BF16), rand((128, ld8(203)), 1, BF16)
    starts, target = torch.tensor([0, 60, 203], dtype=torch.int32, device="cuda"), torch.arange(203, device="cuda", dtype=torch.int32)
    first = layer(ctx, w, X, T, heads, starts, target)
    other = strp.Context(0)
    other.set_workspace(1 << 28)
    for c in (ctx, other):
        again = layer(c, w, X, T, heads, starts, target)
        for n in first:
            assert torch.equal(first[n][..., :T], again[n][..., :T]), n


def test_two_contexts_on_two_streams(ctx):
    """Two calls at once, each with its context and stream."""
    sides = [torch.cuda.Stream() for _ in range(2)]
    data = [(rand((512, 512), i, BF16, 0.05), rand((512, 2000), i + 5, BF16)) for i in range(2)]
    want = [ctx.strp_linear(w, x, 2000).clone() for w, x in data]
    tops = [ctx.strp_token_logprobs(x, 2000, n_top=4) for x in want]
    torch.cuda.synchronize()
    ctxs = []
    for s in sides:
        with torch.cuda.stream(s):
            ctxs.append(strp.Context(0))
            ctxs[-1].set_workspace(1 << 24)
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for s, c, (w, x) in zip(sides, ctxs, data):
            with torch.cuda.stream(s):
                y = c.strp_linear(w, x, 2000)
                got.append((y, c.strp_token_logprobs(y, 2000, n_top=4)))
        torch.cuda.synchronize()
        for (y, t), w, tw in zip(got, want, tops):
            assert torch.equal(y, w) and all(torch.equal(t[n], tw[n]) for n in tw)


def test_binding_refusals(ctx):
    W, X = rand((8, 16), 1), rand((16, 24), 2)
    with pytest.raises(ValueError):
        ctx.strp_linear(W, X[:15], 20)
    with pytest.raises(ValueError):
        ctx.strp_linear(W, X, 25)
    with pytest.raises(ValueError):
        ctx.strp_linear(W.cpu(), X, 20)
    with pytest.raises(TypeError):
        ctx.strp_linear(W.half(), X, 20)
    with pytest.raises(ValueError):
        ctx.strp_linear(W, X.t(), 16)
    with pytest.raises(TypeError):
        ctx.strp_linear(W, X, 20, bias=torch.zeros(8, dtype=BF16, device="cuda"))
    with pytest.raises(TypeError):
        ctx.strp_linear(W, X, 20, residual=torch.zeros((8, 24), dtype=BF16, device="cuda"))
    with pytest.raises(strp.StrpError):
        ctx.strp_linear(W, X, 0)
    with pytest.raises(strp.StrpError):
        ctx.strp_linear(rand((8, 19), 1)[:, :16], X, 20)          # rows that begin at odd places
    with pytest.raises(strp.StrpError):
        ctx.strp_linear(rand((1, 19), 1), rand((19, 24), 2), 20)  # one row without room for a whole eight
    with pytest.raises(ValueError):
        ctx.strp_layer_norm(X, 20, gain=torch.ones(15, device="cuda"))
    with pytest.raises(ValueError):
        ctx.strp_attention(X, X, X, 20, 3)
    with pytest.raises(ValueError):
        ctx.strp_attention(X, X[:4], X, 20, 4, 2)
    with pytest.raises(TypeError):
        ctx.strp_attention(X, X, X, 20, 4, seq_start=torch.tensor([0, 20], device="cuda"))
    with pytest.raises(ValueError):
        ctx.strp_token_logprobs(X, 20, n_top=17)
    with pytest.raises(TypeError):
        ctx.strp_token_logprobs(X, 20, target=torch.zeros(20, dtype=torch.int64, device="cuda"))
