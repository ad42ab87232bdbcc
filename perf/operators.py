"""Timing cases of the operators that carry calibration tokens through a decoder layer and score what a model answers.

Four operators, channel-major like every activation of the framework (rows are channels, tokens are contiguous):

  linear     Y = act(W X + b) + R: the projections of a layer, with bias, activation and residual in one pass
  attention  causal attention over whole prompts, packed one after the other along the tokens, heads in groups
  norm       layer normalisation over the channels of every token
  logprobs   log probability of each token's target under the logits, entropy, and the best alternatives

With `own` false the operators are computed in their plain form, elementary torch operations in 32 bits; with `own` true
through the entry points of the binding.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}

_context = None


def _ctx():
    """The one library context that a program keeps for its device."""
    global _context
    if _context is None:
        from paper_2510_03246_amd import strp
        _context = strp.Context(0)
    return _context


def listed():
    return [
        # One token through an output projection of the smallest model: nothing but launches and latency.
        dict(name="linear_d768_one_token", op="linear", M=768, K=768, T=1, w="bf16", x="bf16", y="bf16", act="none", bias=True, res=True),
        # fc1 of the 2048-wide model on one calibration segment of 2048 tokens.
        dict(name="linear_fc1_d2048", op="linear", M=8192, K=2048, T=2048, w="bf16", x="bf16", y="bf16", act="relu", bias=True, res=False),
        # fc2 of the 4096-wide model after pruning to 4915 of its units, on sixteen segments, added to the residual stream.
        dict(name="linear_fc2_kept4915", op="linear", M=4096, K=4915, T=32768, w="bf16", x="bf16", y="bf16", act="none", bias=True, res=True),
        # fp32 weights as a refit leaves them, no size a multiple of a tile.
        dict(name="linear_ragged_f32", op="linear", M=1013, K=1000, T=5003, w="f32", x="f32", y="f32", act="gelu", bias=True, res=False),
        # A batch of very short prompts, some of one token.
        dict(name="attention_short", op="attention", heads=12, kv=12, dh=64, lens="1 17 64 3 128 1 55 7", dtype="bf16"),
        # Eight calibration segments of 2048 tokens through the 32 x 64 heads of the 2048-wide model.
        dict(name="attention_8x2048", op="attention", heads=32, kv=32, dh=64, lens="2048 2048 2048 2048 2048 2048 2048 2048", dtype="bf16"),
        # Grouped heads and prompts of very different lengths, one of them long.
        dict(name="attention_grouped_ragged", op="attention", heads=32, kv=8, dh=128, lens="77 8191 1 300 1023 4096 33 2500", dtype="bf16"),
        # fp32 activations, a head width that is no power of two.
        dict(name="attention_f32", op="attention", heads=8, kv=8, dh=80, lens="1000 513 1 1500", dtype="f32"),
        # A segment of 2048 tokens of the smallest model.
        dict(name="norm_d768", op="norm", d=768, T=2048, dtype="bf16"),
        # Sixteen segments of the 4096-wide model.
        dict(name="norm_d4096", op="norm", d=4096, T=32768, dtype="bf16"),
        # The next token after one prompt: its distribution over the vocabulary with five alternatives.
        dict(name="logprobs_one_token", op="logprobs", V=50000, T=1, top=5, dtype="f32", masked=0),
        # Perplexity of one segment, with the vocabulary's padding rows masked.
        dict(name="logprobs_2048", op="logprobs", V=50000, T=2048, top=5, dtype="bf16", masked=16),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["linear", "attention", "norm", "logprobs"])
    if op == "linear":
        M, K = _log(rng, 64, 9000), _log(rng, 64, 9000)
        T = _log(rng, 1, max(1, min(32768, int(4.5e11 / (M * K)))))
        w, x = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("f32", "f32"), ("f32", "bf16")])
        if w == "f32":
            T = max(1, T // 8)
        return dict(op="linear", M=M, K=K, T=T, w=w, x=x, y=rng.choice([x, "f32"]), act=rng.choice(["none", "relu", "gelu"]),
                    bias=rng.random() < 0.7, res=rng.random() < 0.5)
    if op == "attention":
        dtype = rng.choice(["bf16", "bf16", "f32"])
        dh = rng.choice([32, 64, 64, 80, 96, 128, 128, rng.randint(8, 128)])
        kv = rng.randint(1, 12)
        heads = kv * rng.choice([1, 1, 2, 4])
        # the longest prompt so that the products stay below those of the largest listed case
        cap = 6.0e11 / (8.0 if dtype == "f32" else 1.0)
        lens, cost = [], 0.0
        for _ in range(_log(rng, 1, 24)):
            n = _log(rng, 1, 6000)
            c = 2.0 * heads * dh * n * (n + 1.0)
            if cost + c > cap:
                break
            lens.append(n)
            cost += c
        return dict(op="attention", heads=heads, kv=kv, dh=dh, lens=" ".join(map(str, lens or [17])), dtype=dtype)
    if op == "norm":
        d = _log(rng, 48, 9000)
        return dict(op="norm", d=d, T=_log(rng, 1, max(1, min(60000, int(1.2e8 / d)))), dtype=rng.choice(["bf16", "f32"]))
    V = _log(rng, 300, 130000)
    return dict(op="logprobs", V=V, T=_log(rng, 1, max(1, min(4096, int(1.0e8 / V)))), top=rng.choice([0, 1, 3, 5, 10, 16]),
                dtype=rng.choice(["bf16", "f32"]), masked=rng.choice([0, 0, 16]))


def _lens(case):
    return [int(n) for n in case["lens"].split()]


def _ld(T):
    return (T + 7) // 8 * 8


def _activations(rows, T, g, dtype, scale=1.0, heavy=True):
    """[rows x ld] with tokens contiguous: Gaussian, one channel in a hundred heavy-tailed."""
    x = torch.randn((rows, _ld(T)), generator=g, device="cuda") * scale
    if heavy:
        n = max(1, rows // 100)
        chi = sum(torch.randn((n, _ld(T)), generator=g, device="cuda") ** 2 for _ in range(3)) / 3.0
        x[:n] /= torch.sqrt(chi)
    return x.to(DTYPES[dtype])


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    st = dict(case=case)
    op = case["op"]
    if op == "linear":
        M, K, T = case["M"], case["K"], case["T"]
        # rows of the weights begin at multiples of eight values
        W = (torch.randn((M, _ld(K)), generator=g, device="cuda") * 0.02).to(DTYPES[case["w"]])
        st.update(W=W[:, :K], X=_activations(K, T, g, case["x"]),
                  b=0.1 * torch.randn(M, generator=g, device="cuda") if case["bias"] else None,
                  R=_activations(M, T, g, case["y"]) if case["res"] else None,
                  Y=torch.empty((M, _ld(T)), dtype=DTYPES[case["y"]], device="cuda"))
    elif op == "attention":
        T, dh = sum(_lens(case)), case["dh"]
        starts = [0]
        for n in _lens(case):
            starts.append(starts[-1] + n)
        dt = case["dtype"]
        st.update(Q=_activations(case["heads"] * dh, T, g, dt, 1.5, heavy=False), K=_activations(case["kv"] * dh, T, g, dt, 1.5, heavy=False),
                  V=_activations(case["kv"] * dh, T, g, dt), starts=torch.tensor(starts, dtype=torch.int32, device="cuda"),
                  C=torch.empty((case["heads"] * dh, _ld(T)), dtype=DTYPES[dt], device="cuda"))
    elif op == "norm":
        d, T = case["d"], case["T"]
        st.update(X=_activations(d, T, g, case["dtype"]), gain=1.0 + 0.1 * torch.randn(d, generator=g, device="cuda"),
                  b=0.1 * torch.randn(d, generator=g, device="cuda"), Y=torch.empty((d, _ld(T)), dtype=DTYPES[case["dtype"]], device="cuda"))
    else:
        V, T = case["V"], case["T"]
        x = torch.randn((V, _ld(T)), generator=g, device="cuda") * 2.5
        likely = torch.randint(0, V - case["masked"], (_ld(T),), generator=g, device="cuda")
        x[likely, torch.arange(_ld(T), device="cuda")] += 8.0
        if case["masked"]:
            x[V - case["masked"]:] = -math.inf
        other = torch.randint(0, V - case["masked"], (T,), generator=g, device="cuda")
        target = torch.where(torch.rand(T, generator=g, device="cuda") < 0.5, likely[:T], other).to(torch.int32)
        st.update(logits=x.to(DTYPES[case["dtype"]]), target=target)
    return st


def _own(st):
    from paper_2510_03246_amd import strp
    ctx, case = _ctx(), st["case"]
    op = case["op"]
    if op == "linear":
        T = case["T"]
        act = {"none": strp.ACT_NONE, "relu": strp.ACT_RELU, "gelu": strp.ACT_GELU}[case["act"]]
        return ctx.strp_linear(st["W"], st["X"], T, bias=st["b"], act=act, residual=st["R"], out=st["Y"])[:, :T]
    if op == "attention":
        T = sum(_lens(case))
        return ctx.strp_attention(st["Q"], st["K"], st["V"], T, case["heads"], case["kv"], st["starts"], out=st["C"])[:, :T]
    if op == "norm":
        T = case["T"]
        return ctx.strp_layer_norm(st["X"], T, gain=st["gain"], bias=st["b"], eps=1e-5, out=st["Y"])[:, :T]
    return ctx.strp_token_logprobs(st["logits"], case["T"], st["target"], n_top=case["top"])


def _plain_attention(st):
    case = st["case"]
    H, dh, rep = case["heads"], case["dh"], case["heads"] // case["kv"]
    T = sum(_lens(case))
    out = torch.empty((H * dh, T), dtype=st["Q"].dtype, device="cuda")
    a = 0
    for n in _lens(case):
        q = st["Q"][:, a:a + n].float().reshape(H, dh, n)
        k, v = (st[x][:, a:a + n].float().reshape(case["kv"], dh, n).repeat_interleave(rep, 0) for x in ("K", "V"))
        step = max(1, min(n, (1 << 28) // (H * n)))          # queries at a time, so that their scores take a GB at most
        for i in range(0, n, step):
            e = min(n, i + step)
            s = torch.matmul(q[:, :, i:e].transpose(1, 2).contiguous(), k[:, :, :e].contiguous()) / math.sqrt(dh)
            later = torch.arange(e, device="cuda")[None, :] > torch.arange(i, e, device="cuda")[:, None]
            s.masked_fill_(later, -math.inf)
            p = torch.exp(s - s.amax(-1, keepdim=True))
            p /= p.sum(-1, keepdim=True)
            o = torch.matmul(v[:, :, :e].contiguous(), p.transpose(1, 2).contiguous())
            out[:, a + i:a + e] = o.reshape(H * dh, e - i).to(out.dtype)
        a += n
    return out


def _plain(st):
    case = st["case"]
    op = case["op"]
    if op == "linear":
        T = case["T"]
        y = st["W"].float() @ st["X"][:, :T].float()
        if case["bias"]:
            y = y + st["b"][:, None]
        if case["act"] == "relu":
            y = torch.clamp_min(y, 0.0)
        elif case["act"] == "gelu":
            y = 0.5 * y * (1.0 + torch.erf(y / math.sqrt(2.0)))
        if case["res"]:
            y = y + st["R"][:, :T].float()
        return y.to(DTYPES[case["y"]])
    if op == "attention":
        return _plain_attention(st)
    if op == "norm":
        x = st["X"][:, :case["T"]].float()
        c = x - x.mean(0)
        y = c / torch.sqrt((c * c).mean(0) + 1e-5)
        return (y * st["gain"][:, None] + st["b"][:, None]).to(DTYPES[case["dtype"]])
    T, n_top = case["T"], case["top"]
    x = st["logits"][:, :T].float()
    c = x - x.amax(0)
    e = torch.exp(c)
    s = e.sum(0)
    log_s = torch.log(s)
    logp = c.gather(0, st["target"].long()[None, :])[0] - log_s
    entropy = log_s - torch.where(e > 0, e * c, 0.0).sum(0) / s
    rows = torch.arange(case["V"], device="cuda")[:, None]
    free = torch.ones_like(x, dtype=torch.bool) if n_top else None
    ids, tops = [], []
    for _ in range(n_top):
        best = torch.where(free, c, -math.inf).amax(0)
        at = torch.where(free & (c == best), rows, case["V"]).amin(0)
        free[at, torch.arange(T, device="cuda")] = False
        ids.append(at)
        tops.append(best - log_s)
    none = torch.empty((0, T), device="cuda")
    return dict(logp=logp, entropy=entropy, top_ids=torch.stack(ids).to(torch.int32) if ids else none.to(torch.int32),
                top_logp=torch.stack(tops) if tops else none)


def run(st):
    return _own(st) if own else _plain(st)


def work(case):
    b = {"bf16": 2.0, "f32": 4.0}
    op = case["op"]
    if op == "linear":
        M, K, T = case["M"], case["K"], case["T"]
        nbytes = b[case["w"]] * M * K + b[case["x"]] * K * T + b[case["y"]] * M * T * (2 if case["res"] else 1) + (4.0 * M if case["bias"] else 0.0)
        return {"bytes": nbytes, "flops": 2.0 * M * K * T}
    if op == "attention":
        T, dh = sum(_lens(case)), case["dh"]
        return {"bytes": b[case["dtype"]] * T * dh * 2.0 * (case["heads"] + case["kv"]),
                "flops": 2.0 * case["heads"] * dh * sum(n * (n + 1.0) for n in _lens(case))}
    if op == "norm":
        return {"bytes": 2.0 * b[case["dtype"]] * case["d"] * case["T"] + 8.0 * case["d"], "flops": 7.0 * case["d"] * case["T"]}
    return {"bytes": b[case["dtype"]] * case["V"] * case["T"] + case["T"] * (12.0 + 8.0 * case["top"]), "flops": 6.0 * case["V"] * case["T"]}


def exact(case, seed):
    """The same in 64 bits, from the definitions."""
    st = prepare(case, seed)
    op = case["op"]
    if op == "linear":
        T = case["T"]
        X, W = st["X"].double(), st["W"].double()
        y = torch.empty((case["M"], T), dtype=torch.float64, device="cuda")
        for t in range(0, T, 8192):
            z = torch.mm(W, X[:, t:min(T, t + 8192)].contiguous())
            if case["bias"]:
                z += st["b"].double().unsqueeze(1)
            if case["act"] == "relu":
                z = torch.where(z > 0, z, 0.0)
            if case["act"] == "gelu":
                z = z * 0.5 * torch.erfc(-z * math.sqrt(0.5))
            if case["res"]:
                z += st["R"][:, t:min(T, t + 8192)].double()
            y[:, t:t + z.shape[1]] = z
        return y
    if op == "attention":
        dh, group = case["dh"], case["heads"] // case["kv"]
        starts = st["starts"].tolist()
        out = torch.empty((case["heads"] * dh, starts[-1]), dtype=torch.float64, device="cuda")
        for a, e in zip(starts, starts[1:]):
            mask = torch.ones((e - a, e - a), dtype=torch.bool, device="cuda").tril()
            for h in range(case["heads"]):
                r, rk = slice(h * dh, (h + 1) * dh), slice(h // group * dh, (h // group + 1) * dh)
                w = torch.mm(st["Q"][r, a:e].double().t().contiguous(), st["K"][rk, a:e].double().contiguous()) * dh ** -0.5
                w = torch.exp(w - torch.where(mask, w, -math.inf).max(1, keepdim=True).values) * mask
                out[r, a:e] = torch.mm(w, st["V"][rk, a:e].double().t().contiguous()).div(w.sum(1, keepdim=True)).t()
        return out
    if op == "norm":
        x = st["X"][:, :case["T"]].double()
        mean = x.sum(0) / case["d"]
        var = ((x - mean) ** 2).sum(0) / case["d"]
        return (x - mean) * torch.rsqrt(var + 1e-5) * st["gain"].double().unsqueeze(1) + st["b"].double().unsqueeze(1)
    T, n = case["T"], case["top"]
    x = st["logits"][:, :T].double()
    lse = torch.logsumexp(x, 0)
    at = torch.arange(T, device="cuda")
    p = torch.exp(x - lse)
    entropy = -(p * torch.where(p > 0, x - lse, 0.0)).sum(0)
    order = torch.sort(x, dim=0, descending=True, stable=True)
    return dict(logp=x[st["target"].long(), at] - lse, entropy=entropy, top_ids=order.indices[:n].to(torch.int32), top_logp=order.values[:n] - lse)
