"""What the speed of a worker's inner step is measured on: linear layers on 4-bit microscaled operands (quantisation,
product, both gradients), the global gradient norm and the AdamW step with states in 32 and in 8 bits, over the range of
matrices and tensor lists that the benchmark configurations, the paper's own architectures and the tests use.

A case is a dict with its kind and sizes:
  quantize  a rows x cols matrix to 4 bits along its rows, and with both = True along its columns too
  linear    y = Q(x) W^T, x of m rows in bf16, W (n x k) laid out in 4 bits beforehand: serving
  train     one step through a linear layer: x, W and dy quantised, y, dx and dW
  norm      norm of all gradients of a list and the factor that clips it
  adamw     AdamW over a list, states in 32 bits
  adamw8    the same with states in 8 bits
Lists: vocab x d matrices at both ends, `layers` layers of seven matrices and two norm vectors; layers = 0: one vocab x d matrix.
"""
import math

import torch

own = False

BETA1, BETA2, EPS, DECAY, LR, STEP = 0.9, 0.95, 1e-8, 0.1, 3e-4, 100
MAX_NORM = 1.0
BLOCK = 256                       # elements that share a scale in the 8-bit states
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _list_case(name, kind, d, layers, ff, vocab, grad):
    return {"name": name, "kind": kind, "d": d, "layers": layers, "ff": ff, "vocab": vocab, "grad": grad}


def listed():
    return [
        # one token's activations before a layer of the 1.8B list: the smallest call, all latency
        {"name": "quantize-token", "kind": "quantize", "rows": 1, "cols": 2048, "both": False, "type": "bf16"},
        # the output head of the 1.8B list after an outer step: fp32 parameters, for the product and for its gradient
        {"name": "quantize-head", "kind": "quantize", "rows": 50257, "cols": 2048, "both": True, "type": "f32"},
        # one token through the gate projection of the 1.8B list
        {"name": "linear-token", "kind": "linear", "m": 1, "n": 8192, "k": 2048},
        # a prompt of odd length through the output head, whose width is odd
        {"name": "linear-prompt-head", "kind": "linear", "m": 517, "n": 50257, "k": 2048},
        # a step through a small ragged layer (the sizes of the ragged list of the tests)
        {"name": "train-ragged", "kind": "train", "m": 1000, "n": 530, "k": 200},
        # a step through the gate projection of the 1.8B list, eight sequences of 2048 tokens
        {"name": "train-1.8b", "kind": "train", "m": 16384, "n": 8192, "k": 2048},
        # gradients of one 1024 x 1024 matrix (configuration 1)
        _list_case("norm-1m", "norm", 1024, 0, 0, 1024, "bf16"),
        # gradients of the 1.8B list (configuration 4)
        _list_case("norm-1.8b", "norm", 2048, 24, 8192, 50257, "bf16"),
        # a small ragged model with fp32 gradients
        _list_case("adamw-ragged", "adamw", 200, 3, 530, 5003, "f32"),
        # the 1.8B list
        _list_case("adamw-1.8b", "adamw", 2048, 24, 8192, 50257, "bf16"),
        # one 1024 x 1024 matrix with 8-bit states: latency
        _list_case("adamw8-1m", "adamw8", 1024, 0, 0, 1024, "bf16"),
        # the 1.8B list with 8-bit states
        _list_case("adamw8-1.8b", "adamw8", 2048, 24, 8192, 50257, "bf16"),
    ]


def draw(rng):
    def spread(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    kind = rng.choice(["quantize", "linear", "train", "norm", "adamw", "adamw8"])
    if kind == "quantize":
        return {"kind": kind, "rows": spread(1, 50257), "cols": spread(16, 2048), "both": rng.random() < 0.5,
                "type": rng.choice(["bf16", "f32"])}
    if kind == "linear":
        return {"kind": kind, "m": spread(1, 517), "n": spread(16, 50257), "k": spread(16, 2048)}
    if kind == "train":
        return {"kind": kind, "m": spread(16, 16384), "n": spread(16, 8192), "k": spread(16, 2048)}
    d = spread(16, 2048)
    return {"kind": kind, "d": d, "layers": rng.randrange(0, 25), "ff": spread(d, 4 * d), "vocab": spread(64, 50257),
            "grad": rng.choice(["bf16", "f32"]) if d < 1024 else "bf16"}


# ---- lists and inputs ----

def _shapes(c):
    """(rows, cols) of each tensor of the list; norm vectors have one row."""
    d, ff, vocab = c["d"], c["ff"], c["vocab"]
    if not c["layers"]:
        return [(vocab, d)]
    layer = [(d, d)] * 4 + [(d, ff)] * 2 + [(ff, d)] + [(1, d)] * 2
    return [(vocab, d)] + layer * c["layers"] + [(1, d), (vocab, d)]


def _layout(c):
    """(rows, cols, offset, layout) of each tensor, the arena's length, and how many of its elements each tensor's part has.
    Tensors begin on multiples of 256 elements; what lies between them is zero."""
    descs, parts, off = [], [], 0
    for r, n in _shapes(c):
        descs.append((r, n, off, 1 if r > 1 else 0))
        parts.append(-(-r * n // BLOCK) * BLOCK)
        off += parts[-1]
    return descs, off, parts


def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _clear_gaps(descs, parts, tensors):
    gaps = []
    for (r, n, off, _), part in zip(descs, parts):
        if part > r * n:
            gaps.append((off + r * n, off + part))
    for a, b in gaps:
        for t in tensors:
            t[a:b] = 0


def prepare(case, seed):
    g = _generator(seed)
    kind = case["kind"]
    s = {"case": case}

    def normal(*shape, std=1.0, dtype=torch.bfloat16):
        return torch.empty(*shape, device="cuda", dtype=dtype).normal_(0.0, std, generator=g)

    if kind in ("quantize", "linear", "train"):
        if kind == "quantize":
            rows, cols = case["rows"], case["cols"]
            s["x"] = normal(rows, cols, std=0.02 if case["type"] == "f32" else 1.0, dtype=DT[case["type"]])
        elif kind == "linear":
            s["x"] = normal(case["m"], case["k"])
            w = normal(case["n"], case["k"], std=case["k"] ** -0.5)
            s["w"] = _mx4_values(w.float())
        else:
            s["x"] = normal(case["m"], case["k"])
            s["w"] = normal(case["n"], case["k"], std=case["k"] ** -0.5)
            s["dy"] = normal(case["m"], case["n"], std=1e-3)
        if own:
            from paper_2508_15706_amd import binding as sl
            s["sl"] = sl
            if kind == "quantize":
                s["q"] = sl.alloc_mx4(rows, cols)
                s["qt"] = sl.alloc_mx4(cols, rows) if case["both"] else None
                s["out"] = [torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda")]
                if case["both"]:
                    s["out"].append(torch.empty(cols, rows, dtype=torch.bfloat16, device="cuda"))
            elif kind == "linear":
                s["wq"] = sl.alloc_mx4(case["n"], case["k"])
                sl.sl_mx4_quantize(w, s["wq"])
                s["y"] = torch.empty(case["m"], case["n"], dtype=torch.bfloat16, device="cuda")
                s["ws"] = sl.alloc_mx4_workspace(case["m"], case["n"], case["k"])
            else:
                m, n, k = case["m"], case["n"], case["k"]
                s["q"] = {"x": sl.alloc_mx4(m, k), "xt": sl.alloc_mx4(k, m), "w": sl.alloc_mx4(n, k),
                          "wt": sl.alloc_mx4(k, n), "dy": sl.alloc_mx4(m, n), "dyt": sl.alloc_mx4(n, m)}
                s["y"] = torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
                s["dx"] = torch.empty(m, k, dtype=torch.bfloat16, device="cuda")
                s["dw"] = torch.empty(n, k, dtype=torch.float32, device="cuda")
                s["ws"] = [sl.alloc_mx4_workspace(*z) for z in ((m, n, k), (m, k, n), (n, k, m))]
        return s

    descs, arena, parts = _layout(case)
    s["grad"] = normal(arena, std=1e-3, dtype=DT[case["grad"]])
    decay = [1.0 if r > 1 else 0.0 for r, _, _, _ in descs]
    tensors = [s["grad"]]
    if kind != "norm":
        s["theta"] = normal(arena, std=0.02, dtype=torch.float32)
        s["theta16"] = torch.zeros(arena, dtype=torch.bfloat16, device="cuda")
        m = normal(arena, std=3e-4, dtype=torch.float32)
        v = torch.empty(arena, device="cuda").uniform_(1e-7, 2e-6, generator=g)
        tensors += [s["theta"], m, v]
        s["scale"] = torch.full((1,), 0.75, device="cuda")
        s["parts"] = torch.tensor(parts, device="cuda")
        s["decay"] = torch.tensor(decay, device="cuda")
        s["seed"] = seed & 0xFFFFFFFF
    _clear_gaps(descs, parts, tensors)
    if kind == "adamw":
        s["m"], s["v"] = m, v
    elif kind == "adamw8":
        half = torch.full((1,), 1 << 19, dtype=torch.int32, device="cuda")
        s["m"], s["m_scale"] = _encode8(m, half, True)
        s["v"], s["v_scale"] = _encode8(v, half, False)
        del m, v
    if own:
        from paper_2508_15706_amd import binding as sl
        s["sl"] = sl
        s["opt"] = sl.sl_adamw_create(descs, decay)
        s["result"] = torch.empty(2, device="cuda")
        s["ws"] = sl.alloc_norm_workspace(s["opt"])
        if kind == "adamw8":
            s["m_out"], s["v_out"] = torch.zeros(arena, device="cuda"), torch.zeros(arena, device="cuda")
    return s


# ---- the plain forms ----

E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _bits(x):
    return x.view(torch.int32)


def _mx4_values(x):
    """The values that the rows of `x` (fp32) have in 4 bits: blocks of 32 share the smallest power of two that leaves none
    of them above 6, elements go to the nearest of E2M1, ties to the even code."""
    rows, cols = x.shape
    pad = -cols % 32
    b = torch.nn.functional.pad(x, (0, pad)).view(rows, -1, 32)
    top = _bits(b.abs().amax(-1, keepdim=True))
    e = (((top + 0x3FFFFF) >> 23) - 2).clamp(0, 253)
    inv = ((254 - e) << 23).view(torch.float32)
    y = (b * inv).abs()
    code = ((y > 0.25).to(torch.uint8) + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5.0))
    table = torch.tensor(E2M1, device=x.device)
    scale = torch.where(e == 0, torch.full_like(e, 0x400000), e << 23).view(torch.float32)
    return (torch.copysign(table[code.int()], b) * scale).view(rows, -1)[:, :cols]


def _fmix(h):
    """MurmurHash3's 32-bit finalizer on int32 (products wrap, shifts are made logical)."""
    h = h ^ ((h >> 16) & 0xFFFF)
    h = h * -2048144789
    h = h ^ ((h >> 13) & 0x7FFFF)
    h = h * -1028477387
    return h ^ ((h >> 16) & 0xFFFF)


def _randoms(seed, n):
    """For each element of an arena of n, 32 random bits from the seed, its block and its place in it."""
    signed = torch.tensor([seed - (1 << 32) if seed >> 31 else seed], dtype=torch.int32, device="cuda")
    block = _fmix(_fmix(signed) ^ torch.arange(n // BLOCK, dtype=torch.int32, device="cuda"))
    return _fmix(block[:, None] ^ torch.arange(BLOCK, dtype=torch.int32, device="cuda")).view(-1)


def _encode8(x, rnd, signed):
    """Codes and block scales of a moment; rnd: 20 bits that are added below the last kept one."""
    b = x.view(-1, BLOCK)
    top = _bits(b.abs().amax(1, keepdim=True))
    e = ((top + 0xFFFFF) >> 23).clamp(1, 253)
    y = b.abs() * ((254 - e) << 23).view(torch.float32) * (2.0 ** -112 if signed else 2.0 ** -96)
    code = ((_bits(y.view(-1)) + rnd) >> 20).clamp(max=127 if signed else 255)
    if signed:
        code = code + 128 * (x < 0)
    else:
        code = torch.maximum(code, (x > 0).int())
    return code.to(torch.uint8), e.view(-1).to(torch.uint8)


def _decode8(codes, scales, signed):
    c = codes.int()
    x = ((c & 127) << 20 if signed else c << 20).view(torch.float32) * (2.0 ** 112 if signed else 2.0 ** 96)
    if signed:
        x = torch.where(c > 127, -x, x)
    return (x.view(-1, BLOCK) * (scales.int() << 23).view(torch.float32)[:, None]).view(-1)


def _adamw_plain(s, m, v):
    """The step in fp32, each operation rounded on its own; theta in place, the new moments returned."""
    g = s["grad"].float() * s["scale"]
    m1 = m * BETA1 + g * (1 - BETA1)
    v1 = v * BETA2 + (g * g) * (1 - BETA2)
    del g
    den = v1.sqrt() * (1 - BETA2 ** STEP) ** -0.5 + EPS
    shrink = torch.repeat_interleave(1 - s["decay"] * (LR * DECAY), s["parts"], output_size=m.numel())
    s["theta"].mul_(shrink).sub_((m1 * (LR / (1 - BETA1 ** STEP))) / den)
    s["theta16"].copy_(s["theta"])
    return m1, v1


def _plain(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "quantize":
        x = s["x"].float()
        out = [_mx4_values(x).bfloat16()]
        if case["both"]:
            out.append(_mx4_values(x.t().contiguous()).bfloat16())
        return out
    if kind == "linear":
        return (_mx4_values(s["x"].float()) @ s["w"].t()).bfloat16()
    if kind == "train":
        x, w, dy = s["x"].float(), s["w"].float(), s["dy"].float()
        y = _mx4_values(x) @ _mx4_values(w).t()
        dx = _mx4_values(dy) @ _mx4_values(w.t().contiguous()).t()
        dw = _mx4_values(dy.t().contiguous()) @ _mx4_values(x.t().contiguous()).t()
        return {"y": y.bfloat16(), "dx": dx.bfloat16(), "dw": dw}
    if kind == "norm":
        norm = s["grad"].float().square().sum().sqrt()
        return torch.stack([norm, torch.where(norm > MAX_NORM, MAX_NORM / norm, torch.ones_like(norm))])
    if kind == "adamw":
        s["m"], s["v"] = _adamw_plain(s, s["m"], s["v"])
        return {"theta": s["theta"], "theta16": s["theta16"], "m": s["m"], "v": s["v"]}
    m1, v1 = _adamw_plain(s, _decode8(s["m"], s["m_scale"], True), _decode8(s["v"], s["v_scale"], False))
    h = _randoms(s["seed"], m1.numel())
    s["m"], s["m_scale"] = _encode8(m1, (h & 0xFFFF) << 4 | 8, True)
    s["v"], s["v_scale"] = _encode8(v1, (h >> 16 & 0xFFFF) << 4 | 8, False)
    del h, m1, v1
    return {"theta": s["theta"], "theta16": s["theta16"], "m": _decode8(s["m"], s["m_scale"], True),
            "v": _decode8(s["v"], s["v_scale"], False)}


# ---- one pass ----

def run(state):
    s = state
    if not own:
        return _plain(s)
    sl, case = s["sl"], s["case"]
    kind = case["kind"]
    if kind == "quantize":
        sl.sl_mx4_quantize(s["x"], s["q"], s["qt"])
        sl.sl_mx4_dequantize(s["q"], s["out"][0])
        if case["both"]:
            sl.sl_mx4_dequantize(s["qt"], s["out"][1])
        return s["out"]
    if kind == "linear":
        sl.sl_mx4_linear(s["x"], s["wq"], s["y"], s["ws"])
        return s["y"]
    if kind == "train":
        q, ws = s["q"], s["ws"]
        sl.sl_mx4_quantize(s["x"], q["x"], q["xt"])
        sl.sl_mx4_quantize(s["w"], q["w"], q["wt"])
        sl.sl_mx4_product(q["x"], q["w"], s["y"], case["k"], ws[0])
        sl.sl_mx4_quantize(s["dy"], q["dy"], q["dyt"])
        sl.sl_mx4_product(q["dy"], q["wt"], s["dx"], case["n"], ws[1])
        sl.sl_mx4_product(q["dyt"], q["xt"], s["dw"], case["m"], ws[2])
        return {"y": s["y"], "dx": s["dx"], "dw": s["dw"]}
    if kind == "norm":
        sl.sl_grad_norm(s["opt"], s["grad"], MAX_NORM, s["result"], s["ws"])
        return s["result"]
    if kind == "adamw":
        sl.sl_adamw_step(s["opt"], s["theta"], s["grad"], s["m"], s["v"], lr=LR, beta1=BETA1, beta2=BETA2, eps=EPS,
                         weight_decay=DECAY, step=STEP, grad_scale=s["scale"], theta16=s["theta16"])
        return {"theta": s["theta"], "theta16": s["theta16"], "m": s["m"], "v": s["v"]}
    sl.sl_adamw_step8(s["opt"], s["theta"], s["grad"], s["m"], s["v"], s["m_scale"], s["v_scale"], s["seed"], lr=LR,
                      beta1=BETA1, beta2=BETA2, eps=EPS, weight_decay=DECAY, step=STEP, grad_scale=s["scale"],
                      theta16=s["theta16"])
    sl.sl_adamw_state_values(s["opt"], 1, s["m"], s["m_scale"], s["m_out"])
    sl.sl_adamw_state_values(s["opt"], 2, s["v"], s["v_scale"], s["v_out"])
    return {"theta": s["theta"], "theta16": s["theta16"], "m": s["m_out"], "v": s["v_out"]}


def work(case):
    kind = case["kind"]
    if kind == "quantize":
        n = case["rows"] * case["cols"]
        return {"bytes": n * ((2 if case["type"] == "bf16" else 4) + (4 if case["both"] else 2)), "flops": 0}
    if kind == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": 2 * m * k + n * k * 17 / 32 + 2 * m * n, "flops": 2 * m * n * k}
    if kind == "train":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": 4 * m * k + 4 * m * n + 6 * n * k, "flops": 6 * m * n * k}
    numel = sum(r * n for r, n in _shapes(case))
    grad = 2 if case["grad"] == "bf16" else 4
    if kind == "norm":
        return {"bytes": numel * grad, "flops": 2 * numel}
    # theta and both moments in and out, the gradient in, the bf16 copy out; 8 bits: the moments' values are written out besides
    return {"bytes": numel * (26 + grad if kind == "adamw" else 14 + 8 + grad), "flops": 12 * numel}


# ---- the definitions in 64 bits ----

def _pow2(e):
    """2^e in 64 bits (torch.ldexp rounds on some devices)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _mx4_exact(x):
    rows, cols = x.shape
    b = torch.nn.functional.pad(x.double(), (0, -cols % 32)).view(rows, -1, 32)
    top = b.abs().amax(-1, keepdim=True)
    mant, e = torch.frexp(top / 6)                               # top / 6 = mant * 2^e, mant in [0.5, 1)
    e = torch.where(mant == 0.5, e - 1, e).clamp(-127, 126)      # the smallest power of two that is not below it
    scale = _pow2(e)
    y = b / scale
    grid = torch.tensor(E2M1, dtype=torch.float64, device=x.device)
    step = torch.where(y.abs() < 2, 0.5, torch.where(y.abs() < 4, 1.0, 2.0))
    near = torch.round(y / step) * step                          # round() takes ties to the even multiple, which is the even code
    assert bool((near.abs() <= grid[-1]).all())
    return (near * scale).view(rows, -1)[:, :cols]


def _round8_exact(x, rnd, mantissa_min, signed):
    b = x.view(-1, BLOCK)
    mant, e = torch.frexp(b.abs().amax(1, keepdim=True))         # in [0.5, 1)
    e = torch.where(mant > 0.9375, e, e - 1).clamp(-126, 126)    # power of two of the largest code's binade
    y = b.abs() * _pow2(-e)
    _, own_e = torch.frexp(y)
    step = _pow2(torch.clamp(own_e - 1, min=mantissa_min) - 3)
    near = (torch.floor(y / step + rnd.view(-1, BLOCK)) * step).clamp(max=1.875)
    if not signed:
        near = torch.where((b > 0) & (near == 0), step, near)
    return torch.copysign(near * _pow2(e), b).view(-1)


def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    kind = case["kind"]
    if kind == "quantize":
        return [_mx4_exact(s["x"])] + ([_mx4_exact(s["x"].t().contiguous())] if case["both"] else [])
    if kind == "linear":
        return _mx4_exact(s["x"]) @ s["w"].double().t()
    if kind == "train":
        x, w, dy = s["x"], s["w"], s["dy"]
        return {"y": _mx4_exact(x) @ _mx4_exact(w).t(),
                "dx": _mx4_exact(dy) @ _mx4_exact(w.t().contiguous()).t(),
                "dw": _mx4_exact(dy.t().contiguous()) @ _mx4_exact(x.t().contiguous()).t()}
    if kind == "norm":
        total = sum(float(p.double().square().sum()) for p in s["grad"].split(1 << 28))
        norm = math.sqrt(total)
        return torch.tensor([norm, MAX_NORM / norm if norm > MAX_NORM else 1.0], dtype=torch.float64)
    n = s["theta"].numel()
    out = {k: torch.empty(n, dtype=torch.float64, device="cuda") for k in ("theta", "m", "v")}
    shrink = torch.repeat_interleave(1 - s["decay"].double() * (LR * DECAY), s["parts"], output_size=n)
    rnd = _randoms(s["seed"], n) if kind == "adamw8" else None
    for a in range(0, n, 1 << 26):
        z = slice(a, min(n, a + (1 << 26)))
        if kind == "adamw":
            m, v = s["m"][z].double(), s["v"][z].double()
        else:
            q = slice(z.start // BLOCK, z.stop // BLOCK)
            m = _decode8(s["m"][z], s["m_scale"][q], True).double()
            v = _decode8(s["v"][z], s["v_scale"][q], False).double()
        g = s["grad"][z].double() * s["scale"].double()
        m = BETA1 * m + (1 - BETA1) * g
        v = BETA2 * v + (1 - BETA2) * g * g
        den = torch.sqrt(v / (1 - BETA2 ** STEP)) + EPS
        out["theta"][z] = shrink[z] * s["theta"][z].double() - LR * (m / (1 - BETA1 ** STEP)) / den
        if kind == "adamw8":
            m = _round8_exact(m, ((rnd[z] & 0xFFFF).double() + 0.5) / 65536, -14, True)
            v = _round8_exact(v, ((rnd[z] >> 16 & 0xFFFF).double() + 0.5) / 65536, -30, False)
        out["m"][z], out["v"][z] = m, v
    out["theta16"] = out["theta"]
    return out
