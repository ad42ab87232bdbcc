"""The operators of generation together, as a program uses them: a model drafts with some of its units taken out, the whole one verifies, both on paged
caches, sequences of different lengths side by side.  At a low temperature the tokens are those of the whole model's largest logits."""
import math

import pytest
import torch

from paper_2510_03246_amd import strp

pytestmark = pytest.mark.gpu
F32, BF16, Q4 = torch.float32, torch.bfloat16, torch.uint8

D, HEADS, KV, DH, F, V, PAGE, LAYERS = 64, 4, 2, 16, 128, 96, 16, 2
TAU, K = 1e-3, 4


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def matrix(rows, cols, seed, scale):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn((rows, cols), generator=g, device="cuda") * scale


class Model:
    """One decoder: embedding, LAYERS layers (norm, attention with turned keys, norm, feed-forward), norm, head."""

    def __init__(self, ctx, keep=None, cache=F32, pages=40):
        self.ctx, self.cache_dt = ctx, cache
        self.E = matrix(V, D, 1, 1.0)
        self.layers = []
        for i in range(LAYERS):
            s = 100 * (i + 1)
            W1 = matrix(F, D, s + 5, D ** -0.5)
            if keep is not None:
                W1[keep:] = 0.0                      # units without input give nothing through a relu
            self.layers.append(dict(q=matrix(HEADS * DH, D, s + 1, D ** -0.5), k=matrix(KV * DH, D, s + 2, D ** -0.5), v=matrix(KV * DH, D, s + 3, D ** -0.5),
                                    o=matrix(D, HEADS * DH, s + 4, D ** -0.5), W1=W1, W2=matrix(D, F, s + 6, F ** -0.5)))
        self.head = matrix(V, D, 2, 1.0)
        self.one, self.zero = torch.ones(D, device="cuda"), torch.zeros(D, device="cuda")
        self.freq = 1e4 ** (-torch.arange(0, DH, 2, device="cuda", dtype=F32) / DH)
        self.caches = [strp.PagedCache.empty(ctx, pages, KV, DH, PAGE, cache) for _ in range(LAYERS)]

    def logits(self, tokens, table, past, starts):
        """tokens of all sequences, one behind the other: [V x ld]"""
        c, T = self.ctx, tokens.numel()
        H = torch.zeros((D, (T + 7) // 8 * 8), device="cuda")
        H[:, :T] = self.E[tokens.long()].t()
        for w, cache in zip(self.layers, self.caches):
            n = c.strp_layer_norm(H, T, self.one, self.zero)
            q, k, v = (c.strp_linear(w[x], n, T) for x in "qkv")
            c.strp_cache_append(k, v, T, cache, table, past, starts, self.freq, Q=q, q_out=q)
            H = c.strp_linear(w["o"], c.strp_cache_attention(q, T, HEADS, cache, table, past, starts), T, residual=H)
            n = c.strp_layer_norm(H, T, self.one, self.zero)
            H = c.strp_linear(w["W2"], c.strp_linear(w["W1"], n, T, act=strp.ACT_RELU), T, residual=H)
        return c.strp_linear(self.head, c.strp_layer_norm(H, T, self.one, self.zero), T)

    def whole(self, tokens):
        """The same for one sequence, in 64 bits: [T x V]"""
        T = len(tokens)
        norm = lambda x: (x - x.mean(1, keepdim=True)) / torch.sqrt(x.var(1, unbiased=False, keepdim=True) + 1e-5)
        x = self.E.double()[torch.tensor(tokens, device="cuda")]
        a = torch.arange(T, device="cuda", dtype=torch.float64)[:, None, None] * self.freq.double()
        cos, sin = torch.cos(a), torch.sin(a)

        def turn(y):
            l, r = y[..., :DH // 2], y[..., DH // 2:]
            return torch.cat([l * cos - r * sin, r * cos + l * sin], -1)

        mask = torch.ones((T, T), dtype=torch.bool, device="cuda").tril()
        for w in self.layers:
            n = norm(x)
            q, k, v = ((n @ w[y].double().t()).reshape(T, -1, DH) for y in "qkv")
            q, k = turn(q), turn(k)
            out = []
            for h in range(HEADS):
                s = (q[:, h] @ k[:, h // (HEADS // KV)].t()) / math.sqrt(DH)
                out.append(torch.softmax(s.masked_fill(~mask, -math.inf), 1) @ v[:, h // (HEADS // KV)])
            x = x + torch.cat(out, 1) @ w["o"].double().t()
            x = x + torch.relu(norm(x) @ w["W1"].double().t()) @ w["W2"].double().t()
        return norm(x) @ self.head.double().t()


@pytest.mark.parametrize("keep", [None, 80, 0], ids=["itself", "pruned", "none"])
def test_drafted_and_verified_tokens_are_the_model_s_own(keep):
    ctx = strp.Context(0)
    target, draft = Model(ctx), Model(ctx, keep)
    prompts = [[5, 17, 3], [90], [1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13, 14, 15, 16, 17, 18]]
    n = len(prompts)
    table = torch.randperm(n * 4, generator=torch.Generator().manual_seed(3)).to(torch.int32).reshape(n, 4).cuda()
    texts = [list(p) for p in prompts]
    # all of the prompts but their last tokens into both caches
    starts = [0]
    for p in prompts:
        starts.append(starts[-1] + len(p) - 1)
    packed = ints([t for p in prompts for t in p[:-1]])
    for m in (target, draft):
        m.logits(packed, table, ints([0] * n), ints(starts))
    past = ints([len(p) - 1 for p in prompts])
    last = ints([p[-1] for p in prompts])
    g = torch.Generator(device="cuda").manual_seed(9)
    kept = []
    for _ in range(6):
        # K tokens of the draft one by one, and one more step so that its cache has the last of them
        ids, logits, x = [], [], last
        for k in range(K + 1):
            out = draft.logits(x, table, past + k, ints(range(n + 1)))
            if k == K:
                break
            x = ctx.strp_verify_draft(out, None, None, None, torch.rand(n, generator=g, device="cuda"), temperature=TAU)["next_ids"]
            ids.append(x)
            logits.append(out[:, :n])
        drafted = torch.stack(ids, 1)                                                       # [n x K]
        D_logits = torch.zeros((V, (n * K + 7) // 8 * 8), device="cuda")
        D_logits[:, :n * K] = torch.stack(logits, 2).reshape(V, n * K)
        T_logits = target.logits(torch.cat([last[:, None], drafted], 1).reshape(-1), table, past, ints([(K + 1) * i for i in range(n + 1)]))
        res = ctx.strp_verify_draft(T_logits, D_logits, drafted.reshape(-1).contiguous(), torch.rand(n * K, generator=g, device="cuda"), torch.rand(n, generator=g, device="cuda"),
                                    ints([K * i for i in range(n + 1)]), TAU)
        for i in range(n):
            a = int(res["accepted"][i])
            kept.append(a)
            texts[i] += drafted[i, :a].tolist() + [int(res["next_ids"][i])]
        past = past + res["accepted"] + 1
        last = res["next_ids"].clone()
    assert past.tolist() == [len(t) - 1 for t in texts]
    for p, t in zip(prompts, texts):
        want = target.whole(t)[len(p) - 1:-1]
        top = want.topk(2, 1)
        # where the second is as near as the rounding of the logits and the temperature together let it be, either may follow
        sure = top.values[:, 0] - top.values[:, 1] > 40 * TAU
        assert sure.float().mean() > 0.5
        assert (top.indices[:, 0] == torch.tensor(t[len(p):], device="cuda"))[sure].all()
    if keep is None:
        assert min(kept) == K                        # the model drafts for itself: all of it is kept
    else:
        assert sum(kept) < K * len(kept)


@pytest.mark.parametrize("columns", [30, 2048])
@pytest.mark.parametrize("dt", [BF16, F32])
def test_many_sequences_beside_each_other(dt, columns):
    """More sequences than a workgroup keeps the lengths of, one of them with many new tokens: each as by itself."""
    ctx = strp.Context(0)
    n, kv, heads, dh, long = 700, 1, 2, 32, 650
    past = [(i * 37) % 90 for i in range(n)]
    cache = strp.PagedCache.empty(ctx, n * 6 + 30, kv, dh, 16, dt)
    g = torch.Generator(device="cuda").manual_seed(1)
    for x in (cache.K, cache.V):
        x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
    pages = torch.randperm(n * 6 + 30, generator=torch.Generator().manual_seed(2)).to(torch.int32)
    table = torch.full((n, columns), -1, dtype=torch.int32)
    table[:, :6] = pages[:n * 6].reshape(n, 6)
    table[long, :30] = pages[n * 6:]
    table = table.cuda()
    counts = [0 if i % 5 == 2 else 400 if i == long else 1 for i in range(n)]
    starts = [0]
    for c in counts:
        starts.append(starts[-1] + c)
    past[long] = 11
    T = starts[-1]
    Q = torch.randn((heads * dh, (T + 7) // 8 * 8), generator=g, device="cuda").to(dt)
    got = ctx.strp_cache_attention(Q, T, heads, cache, table, ints(past), ints(starts))
    for i in list(range(0, n, 13)) + [510, 511, 512, 513, 650, 698, 699]:
        a, c = starts[i], counts[i]
        if c == 0:
            continue
        one = torch.zeros((heads * dh, (c + 7) // 8 * 8), dtype=dt, device="cuda")
        one[:, :c] = Q[:, a:a + c]
        want = ctx.strp_cache_attention(one, c, heads, cache, table[i:i + 1].contiguous(), ints([past[i]]))[:, :c]
        # the keys may be divided otherwise: two roundings of the result, and of fp32 sums of at most 411 terms below the largest value of 5
        tol = 2 * torch.finfo(dt).eps * want.float().abs() + 2 * 500 * 2.0 ** -23 * 5 + (2.0 ** -15 * 5 if dt == BF16 else 0.0)
        assert ((got[:, a:a + c].float() - want.float()).abs() <= tol).all(), i
