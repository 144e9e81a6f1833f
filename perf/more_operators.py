"""What the speed of the layers between a worker's linear layers is measured on: the root-mean-square norm with the residual's
addition, attention over packed sequences and for single tokens over a cache, and the loss on the head's logits, over the range of
sizes that the benchmark configurations, the paper's own architectures and the tests use.

A case is a dict with its kind and sizes:
  norm         h = x + residual, y = norm of h: serving
  norm_step    the same with y as 4-bit matrices both ways, and the backward pass: training
  attend       causal attention over packed sequences, forward
  attend_step  forward and backward
  token        one new token for each sequence, over its cache
  loss         loss of every token's logits and its gradient: negative log-likelihood, or (policy) clipped ratios with a KL term
Sequences: `sequences` of them, the longest of `longest` tokens, all of them (even) or a fixed mixture down to one token.
"""
import math
import random

import torch

own = False

EPS = 1e-5
CLIP_LOW, CLIP_HIGH, KL = 0.2, 0.28, 0.05
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _attend_case(kind, heads, kv_heads, dim, sequences, longest, even, name=None):
    c = {"kind": kind, "heads": heads, "kv_heads": kv_heads, "dim": dim, "sequences": sequences, "longest": longest, "even": even}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token before a layer of the 1.8B list: the smallest call, all latency
        {"name": "norm-token", "kind": "norm", "rows": 1, "cols": 2048, "x": "bf16", "residual": "f32"},
        # eight sequences of 2048 tokens through a norm of the 1.8B list, all in bf16
        {"name": "norm-1.8b", "kind": "norm", "rows": 16384, "cols": 2048, "x": "bf16", "residual": "bf16"},
        # a training step of a small ragged model (sizes of the ragged list of the tests)
        {"name": "norm-step-ragged", "kind": "norm_step", "rows": 1000, "cols": 200, "x": "f32", "residual": "f32"},
        # a training step of the 1.8B list with the residual in fp32, eight sequences of 2048 tokens
        {"name": "norm-step-1.8b", "kind": "norm_step", "rows": 16384, "cols": 2048, "x": "bf16", "residual": "f32"},
        # short prompts of very different lengths, five heads of 40 (a width of 200)
        _attend_case("attend", 5, 1, 40, 7, 203, False, "attend-ragged"),
        # one long prompt, heads of the paper's 2B architecture: 20 query heads, 5 for keys and values, of 128
        _attend_case("attend", 20, 5, 128, 1, 8192, True, "attend-long"),
        # a training step on packed documents, 16 heads of 64 (a width of 1024)
        _attend_case("attend_step", 16, 4, 64, 9, 1021, False, "attend-step-ragged"),
        # a training step of the 1.8B list: eight sequences of 2048 tokens, 16 heads of 128
        _attend_case("attend_step", 16, 16, 128, 8, 2048, True, "attend-step-1.8b"),
        # one sequence's next token: latency
        _attend_case("token", 16, 16, 128, 1, 2047, True, "token-one"),
        # a batch of 64 sequences with caches of up to 16,384 tokens, heads of the paper's 2B architecture
        _attend_case("token", 20, 5, 128, 64, 16384, False, "token-batch"),
        # a policy step on fp32 logits over the paper's vocabulary, an odd number of tokens
        {"name": "loss-policy", "kind": "loss", "rows": 517, "vocab": 32000, "type": "f32", "policy": True},
        # pre-training on the 1.8B list: the head's bf16 logits of four sequences of 2048 tokens, rows of odd length
        {"name": "loss-1.8b", "kind": "loss", "rows": 8192, "vocab": 50257, "type": "bf16", "policy": False},
    ]


def draw(rng):
    def spread(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    kind = rng.choice(["norm", "norm_step", "attend", "attend_step", "token", "loss"])
    if kind in ("norm", "norm_step"):
        return {"kind": kind, "rows": spread(1, 16384), "cols": spread(16, 2048), "x": rng.choice(["bf16", "f32"]),
                "residual": rng.choice(["bf16", "f32"])}
    if kind == "loss":
        return {"kind": kind, "rows": spread(1, 4096), "vocab": spread(64, 50257), "type": rng.choice(["bf16", "f32"]),
                "policy": rng.random() < 0.5}
    heads, kv_heads = rng.choice([(16, 16), (16, 4), (20, 5), (5, 1), (5, 5), (12, 4), (8, 1)])
    dim = rng.choice([40, 64, 80, 96, 128])
    if kind == "token":
        return _attend_case(kind, heads, kv_heads, dim, spread(1, 64), spread(1, 8192), rng.random() < 0.3)
    longest = spread(1, 4096)
    return _attend_case(kind, heads, kv_heads, dim, rng.randint(1, max(1, min(8, (1 << 25) // longest ** 2))), longest, rng.random() < 0.3)


# ---- inputs ----

def _lengths(c):
    """Tokens of each sequence; of an uneven list the first has the most and the last one."""
    n, longest = c["sequences"], c["longest"]
    if c["even"]:
        return [longest] * n
    rng = random.Random(1000 * longest + n)
    middle = [max(1, round(longest ** rng.uniform(0.5, 1.0))) for _ in range(n - 2)]
    return [longest] + middle + [1] * (n > 1)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    kind = case["kind"]
    s = {"case": case}

    def normal(*shape, std=1.0, dtype=torch.bfloat16):
        return torch.empty(*shape, device="cuda", dtype=dtype).normal_(0.0, std, generator=g)

    def like(t):
        return torch.zeros_like(t)

    if kind in ("norm", "norm_step"):
        shape = case["rows"], case["cols"]
        s["x"] = normal(*shape, std=0.5, dtype=DT[case["x"]])
        s["residual"] = normal(*shape, dtype=DT[case["residual"]])
        s["w"] = 1.0 + normal(case["cols"], std=0.1, dtype=torch.float32)
        s["h"], s["y"] = like(s["residual"]), torch.zeros(*shape, dtype=torch.bfloat16, device="cuda")
        if kind == "norm_step":
            s["dy"] = normal(*shape, std=1e-3)
            s["dh"] = normal(*shape, std=1e-3, dtype=DT[case["residual"]])
            s["rstd"], s["dx"], s["dw"] = torch.zeros(shape[0], device="cuda"), like(s["dh"]), like(s["w"])
            s["yt"] = torch.zeros(shape[1], shape[0], dtype=torch.bfloat16, device="cuda")
    elif kind == "loss":
        rows, vocab = case["rows"], case["vocab"]
        s["logits"] = normal(rows, vocab, std=2.0, dtype=DT[case["type"]])
        target = torch.randint(vocab, (rows,), device="cuda", generator=g)
        skipped = torch.rand(rows, device="cuda", generator=g) < 0.1                     # prompts and padding
        s["targets"] = torch.where(skipped, torch.full_like(target, -1), target)
        s["weights"] = torch.full((rows,), 1.0 / rows, device="cuda")
        s["logp"], s["loss"], s["dlogits"] = torch.zeros(rows, device="cuda"), torch.zeros(1, device="cuda"), like(s["logits"])
        if case["policy"]:
            now = s["logits"].gather(1, target[:, None])[:, 0].float() - torch.logsumexp(s["logits"].float(), 1)
            s["old"] = now + normal(rows, std=0.15, dtype=torch.float32)
            s["ref"] = now + normal(rows, std=0.3, dtype=torch.float32)
            s["advantages"] = normal(rows, dtype=torch.float32)
    else:
        lengths = _lengths(case)
        n, longest = case["sequences"], case["longest"]
        q_heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
        token = kind == "token"
        rows_q, rows_k = (n, n * longest) if token else (sum(lengths), sum(lengths))
        s["lengths"] = lengths
        s["q"] = normal(rows_q, q_heads, dim, std=1.5)
        s["k"], s["v"] = normal(rows_k, kv_heads, dim), normal(rows_k, kv_heads, dim)
        s["out"] = like(s["q"])
        ends = [0]
        for length in lengths:
            ends.append(ends[-1] + (longest if token else length))
        s["start"] = torch.tensor(ends, dtype=torch.int32, device="cuda")
        s["count"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        # where each sequence's tokens are in a batch that is filled up to the longest, and which of its places are real
        place = torch.arange(longest, device="cuda")
        s["real"] = place[None] < s["count"][:, None]
        s["at"] = torch.where(s["real"], s["start"][:-1, None] + place[None], torch.zeros_like(place))
        if kind == "attend_step":
            s["dout"] = normal(rows_q, q_heads, dim, std=1e-2)
            s["lse"] = torch.zeros(q_heads, rows_q, device="cuda")
            s["dq"], s["dk"], s["dv"] = like(s["q"]), like(s["k"]), like(s["v"])
    if own:
        from paper_2508_15706_amd import binding as sl
        s["sl"] = sl
        if kind == "norm_step":
            s["q4"], s["qt4"] = sl.alloc_mx4(*shape), sl.alloc_mx4(shape[1], shape[0])
            s["ws"] = sl.alloc_rms_norm_workspace(*shape)
        elif kind == "loss":
            s["ws"] = sl.alloc_token_loss_workspace(rows)
        elif kind == "attend_step":
            s["ws"] = sl.alloc_attention_workspace(rows_q, q_heads)
        elif kind == "token":
            s["ws"] = sl.alloc_attention_token_workspace(n, rows_k, q_heads, kv_heads, dim)
    return s


# ---- the plain forms ----

E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _mx4_values(x):
    """The values that the rows of `x` (fp32) have in 4 bits: blocks of 32 share the smallest power of two that leaves none
    of them above 6, elements go to the nearest of E2M1, ties to the even code."""
    rows, cols = x.shape
    b = torch.nn.functional.pad(x, (0, -cols % 32)).view(rows, -1, 32)
    top = b.abs().amax(-1, keepdim=True).view(torch.int32)
    e = (((top + 0x3FFFFF) >> 23) - 2).clamp(0, 253)
    y = (b * ((254 - e) << 23).view(torch.float32)).abs()
    code = ((y > 0.25).int() + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5.0))
    scale = torch.where(e == 0, torch.full_like(e, 0x400000), e << 23).view(torch.float32)
    return (torch.copysign(torch.tensor(E2M1, device=x.device)[code], b) * scale).view(rows, -1)[:, :cols]


def _norm_plain(s):
    step = s["case"]["kind"] == "norm_step"
    h = (s["x"].float() + s["residual"].float()).to(s["residual"].dtype)
    hf = h.float()
    rstd = (hf.double().square().mean(1) + EPS).rsqrt().float()[:, None]
    y = (hf * rstd * s["w"]).bfloat16()
    if not step:
        return {"h": h, "y": y}
    yf, dy = y.float(), s["dy"].float()
    g = dy * s["w"]
    unit = hf * rstd
    dx = s["dh"].float() + rstd * (g - unit * (g * unit).mean(1, keepdim=True))
    return {"h": h, "y": _mx4_values(yf).bfloat16(), "yt": _mx4_values(yf.t().contiguous()).bfloat16(),
            "dx": dx.to(s["dh"].dtype), "dw": (dy * unit).sum(0)}


def _filled(s, t):
    """(tokens, heads, dim) -> (sequences, heads, longest, dim) in fp32, zero where a sequence has ended."""
    return (t[s["at"]] * s["real"][:, :, None, None]).float().transpose(1, 2).contiguous()


def _packed(s, t):
    return t.transpose(1, 2)[s["real"]]


def _attend_plain(s):
    case = s["case"]
    group, dim, longest = case["heads"] // case["kv_heads"], case["dim"], case["longest"]
    scale = dim ** -0.5
    if case["kind"] == "token":
        q = s["q"].float().view(case["sequences"], case["kv_heads"], group, dim)
        k, v = _filled(s, s["k"]), _filled(s, s["v"])
        p = q @ k.transpose(2, 3) * scale
        p = p.masked_fill(~s["real"][:, None, None], -math.inf)
        p = (p - p.amax(-1, keepdim=True)).exp()
        return (p @ v / p.sum(-1, keepdim=True)).view_as(s["q"]).bfloat16()
    q = _filled(s, s["q"])
    k, v = (_filled(s, s[n]).repeat_interleave(group, 1) for n in "kv")
    p = q @ k.transpose(2, 3).contiguous() * scale
    later = torch.ones(longest, longest, dtype=torch.bool, device="cuda").triu(1)
    p = p.masked_fill_(later, -math.inf)
    p = p.sub_(p.amax(-1, keepdim=True)).exp_()
    p = p.div_(p.sum(-1, keepdim=True))
    out = p @ v
    if case["kind"] == "attend":
        return _packed(s, out).bfloat16()
    dout = _filled(s, s["dout"])
    ds = p * (dout @ v.transpose(2, 3).contiguous() - (dout * out).sum(-1, keepdim=True))
    shape = case["sequences"], case["kv_heads"], group, longest, dim
    dq = ds @ k * scale
    dk = (ds.transpose(2, 3).contiguous() @ q * scale).view(shape).sum(2)
    dv = (p.transpose(2, 3).contiguous() @ dout).view(shape).sum(2)
    return {"out": _packed(s, out).bfloat16(), "dq": _packed(s, dq).bfloat16(), "dk": _packed(s, dk).bfloat16(),
            "dv": _packed(s, dv).bfloat16()}


def _loss_plain(s):
    case = s["case"]
    z = s["logits"].float()
    used = s["targets"] >= 0
    at = s["targets"].clamp(min=0)[:, None]
    top = z.amax(1, keepdim=True)
    p = (z - top).exp()
    total = p.sum(1, keepdim=True)
    logp = (z.gather(1, at).double() - top - total.double().log())[:, 0]
    if case["policy"]:
        a = s["advantages"].double()
        r = (logp - s["old"]).exp()
        up = a >= 0
        kept = torch.where(up, r <= 1 + CLIP_HIGH, r >= 1 - CLIP_LOW)
        d = s["ref"] - logp
        each = -a * torch.where(up, r.clamp(max=1 + CLIP_HIGH), r.clamp(min=1 - CLIP_LOW)) + KL * (torch.expm1(d) - d)
        slope = -a * r * kept - KL * torch.expm1(d)
    else:
        each, slope = -logp, -torch.ones_like(logp)
    zero = torch.zeros_like(logp)
    loss = torch.where(used, s["weights"] * each, zero).sum().float().view(1)
    slope = torch.where(used, s["weights"] * slope, zero).float()[:, None]
    dz = p.div_(total).mul_(-slope)
    dz.scatter_add_(1, at, slope)
    return {"loss": loss, "logp": torch.where(used, logp, zero).float(), "dlogits": dz.to(s["logits"].dtype)}


# ---- one pass ----

def run(state):
    s = state
    case = s["case"]
    kind = case["kind"]
    if not own:
        return (_norm_plain if kind.startswith("norm") else _loss_plain if kind == "loss" else _attend_plain)(s)
    sl = s["sl"]
    if kind == "norm":
        sl.sl_rms_norm(s["x"], s["w"], s["y"], residual=s["residual"], h=s["h"], eps=EPS)
        return {"h": s["h"], "y": s["y"]}
    if kind == "norm_step":
        sl.sl_rms_norm(s["x"], s["w"], None, residual=s["residual"], h=s["h"], rstd=s["rstd"], q=s["q4"], qt=s["qt4"], eps=EPS)
        sl.sl_mx4_dequantize(s["q4"], s["y"])
        sl.sl_mx4_dequantize(s["qt4"], s["yt"])
        sl.sl_rms_norm_backward(s["h"], s["w"], s["rstd"], s["dy"], s["dx"], dh=s["dh"], dw=s["dw"], workspace=s["ws"])
        return {"h": s["h"], "y": s["y"], "yt": s["yt"], "dx": s["dx"], "dw": s["dw"]}
    if kind == "attend":
        sl.sl_attention(s["q"], s["k"], s["v"], s["out"], s["start"])
        return s["out"]
    if kind == "attend_step":
        sl.sl_attention(s["q"], s["k"], s["v"], s["out"], s["start"], lse=s["lse"])
        sl.sl_attention_backward(s["q"], s["k"], s["v"], s["out"], s["lse"], s["dout"], s["dq"], s["dk"], s["dv"], s["start"],
                                 workspace=s["ws"])
        return {"out": s["out"], "dq": s["dq"], "dk": s["dk"], "dv": s["dv"]}
    if kind == "token":
        sl.sl_attention_token(s["q"], s["k"], s["v"], s["out"], s["start"], s["count"], workspace=s["ws"])
        return s["out"]
    policy = None
    if case["policy"]:
        policy = sl.Policy(s["old"], s["advantages"], CLIP_LOW, CLIP_HIGH, s["ref"], KL)
    sl.sl_token_loss(s["logits"], s["targets"], s["weights"], s["loss"], logp=s["logp"], dlogits=s["dlogits"], policy=policy,
                     workspace=s["ws"])
    return {"loss": s["loss"], "logp": s["logp"], "dlogits": s["dlogits"]}


def work(case):
    kind = case["kind"]
    if kind in ("norm", "norm_step"):
        n, x, r = case["rows"] * case["cols"], 2 + 2 * (case["x"] == "f32"), 2 + 2 * (case["residual"] == "f32")
        # x and residual in, h and y out; a step: y twice, dy and dh in, dx out
        return {"bytes": n * (x + 2 * r + 2) + (n * (4 + 2 * r) if kind == "norm_step" else 0) + 4 * case["cols"],
                "flops": n * (4 if kind == "norm" else 14)}
    if kind == "loss":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * (4 if case["type"] == "bf16" else 8) + 16 * case["rows"], "flops": 5 * n}
    lengths = _lengths(case)
    row_q, row_k = 2 * case["heads"] * case["dim"], 2 * case["kv_heads"] * case["dim"]
    tokens = sum(lengths)
    if kind == "token":
        return {"bytes": 2 * tokens * row_k + 2 * len(lengths) * row_q, "flops": 4 * case["dim"] * case["heads"] * tokens}
    pairs = sum(n * (n + 1) // 2 for n in lengths)
    if kind == "attend":
        return {"bytes": tokens * (2 * row_q + 2 * row_k), "flops": 4 * case["dim"] * case["heads"] * pairs}
    return {"bytes": tokens * (4 * row_q + 4 * row_k), "flops": 14 * case["dim"] * case["heads"] * pairs}


# ---- the definitions in 64 bits ----

def _four_bits(x):
    """Rows of x in blocks of 32, each to the nearest multiple of its power of two among the eight magnitudes."""
    rows, cols = x.shape
    b = torch.nn.functional.pad(x, (0, -cols % 32)).view(rows, -1, 32)
    mant, e = torch.frexp(b.abs().amax(-1, keepdim=True) / 6)
    e = torch.where(mant == 0.5, e - 1, e).clamp(-127, 126)      # the smallest power of two that leaves the largest <= 6
    scale = ((e.long() + 1023) << 52).view(torch.float64)
    y = b / scale
    step = torch.where(y.abs() < 2, 0.5, torch.where(y.abs() < 4, 1.0, 2.0))
    return (torch.round(y / step) * step * scale).view(rows, -1)[:, :cols]


def _exact_attention(q, k, v, dout, group, scale):
    """One sequence, head by head: (tokens, heads, dim) in 64 bits."""
    n, heads, _ = q.shape
    shift = k.shape[0] - n
    ok = torch.arange(k.shape[0], device="cuda")[None] <= torch.arange(n, device="cuda")[:, None] + shift
    out, dq = torch.zeros_like(q), torch.zeros_like(q)
    dk, dv = torch.zeros_like(k), torch.zeros_like(v)
    for h in range(heads):
        qh, kh, vh = q[:, h], k[:, h // group], v[:, h // group]
        score = torch.where(ok, (qh @ kh.T) * scale, -math.inf)
        p = torch.softmax(score, 1)
        out[:, h] = p @ vh
        if dout is not None:
            do = dout[:, h]
            dp = do @ vh.T
            ds = p * (dp - (p * dp).sum(1, keepdim=True))
            dq[:, h] = scale * (ds @ kh)
            dk[:, h // group] += scale * (ds.T @ qh)
            dv[:, h // group] += p.T @ do
    return out, dq, dk, dv


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    kind = case["kind"]
    if kind in ("norm", "norm_step"):
        h = (s["x"].double() + s["residual"].double()).to(s["residual"].dtype)
        r = 1.0 / torch.sqrt(h.double().pow(2).sum(1, keepdim=True) / case["cols"] + EPS)
        y = h.double() * r * s["w"].double()
        if kind == "norm":
            return {"h": h.double(), "y": y}
        y16 = y.bfloat16().double()                              # (what is quantised is y in bf16)
        dy = s["dy"].double()
        n = h.double() * r
        a = dy * s["w"].double()
        dx = s["dh"].double() + r * a - r * n * (a * n).sum(1, keepdim=True) / case["cols"]
        return {"h": h.double(), "y": _four_bits(y16), "yt": _four_bits(y16.T.contiguous()), "dx": dx, "dw": (dy * n).sum(0)}
    if kind == "loss":
        out = {"loss": 0.0, "logp": [], "dlogits": []}
        for a in range(0, case["rows"], 1024):
            z = s["logits"][a:a + 1024].double()
            t, w = s["targets"][a:a + 1024], s["weights"][a:a + 1024].double()
            every = torch.log_softmax(z, 1)
            logp = every.gather(1, t.clamp(min=0)[:, None])[:, 0]
            slope, each = torch.full_like(logp, -1.0), -logp
            if case["policy"]:
                adv, old, ref = (s[n][a:a + 1024].double() for n in ("advantages", "old", "ref"))
                ratio = torch.exp(logp - old)
                clipped = ratio.clamp(1 - CLIP_LOW, 1 + CLIP_HIGH)
                each = -torch.minimum(ratio * adv, clipped * adv) + KL * (torch.exp(ref - logp) - (ref - logp) - 1)
                slope = torch.where(ratio * adv <= clipped * adv, -ratio * adv, torch.zeros_like(adv)) + KL * (1 - torch.exp(ref - logp))
            w = torch.where(t < 0, 0.0, w)
            out["loss"] = out["loss"] + (w * each).sum()
            out["logp"].append(torch.where(t < 0, 0.0, logp))
            hot = torch.zeros_like(z).scatter_(1, t.clamp(min=0)[:, None], 1.0)
            out["dlogits"].append((w * slope)[:, None] * (hot - every.exp()))
        return {"loss": out["loss"].view(1), "logp": torch.cat(out["logp"]), "dlogits": torch.cat(out["dlogits"])}
    group, scale = case["heads"] // case["kv_heads"], case["dim"] ** -0.5
    starts, parts = s["start"].tolist(), []
    for i, n in enumerate(s["lengths"]):
        keys = slice(starts[i], starts[i] + n)
        rows = slice(i, i + 1) if kind == "token" else keys
        dout = s["dout"][rows].double() if kind == "attend_step" else None
        parts.append(_exact_attention(s["q"][rows].double(), s["k"][keys].double(), s["v"][keys].double(), dout, group, scale))
    out, dq, dk, dv = (torch.cat(p) for p in zip(*parts))
    return {"out": out, "dq": dq, "dk": dk, "dv": dv} if kind == "attend_step" else out
