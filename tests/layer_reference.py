"""Definitions in 64 bits of the layers between the linear ones - norm, attention, token loss - and how far fp32 and bf16 roundings can
take a result from them.  A rounding to nearest is off by at most half a step of the type."""
import math

import torch

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
F32 = HALF[torch.float32]


# ---- norm ----

def norm(x, residual, w, eps, h_type):
    """h (as its type holds it), s and y, in 64 bits."""
    h = (x.double() if residual is None else x.double() + residual.double().to(x.device)).to(h_type).double()
    s = 1.0 / torch.sqrt(h.square().mean(1) + eps)
    return h, s, h * s[:, None] * w.double()


def norm_backward(h, w, s, dy, dh):
    """dx, dw and their bounds without the last rounding: u, g, their mean, the difference and the sum are rounded once each on the way,
    s was before; nothing passes more than eight roundings."""
    h, w, dy, s = h.double(), w.double(), dy.double(), s.double()[:, None]
    n = h.shape[1]
    u, g = h * s, dy * w
    c = (g * u).sum(1, keepdim=True) / n
    dx = s * (g - u * c)
    off = 8 * F32 * (s * g.abs() + s * u.abs() * (c.abs() + (g * u).abs().sum(1, keepdim=True) / n))
    if dh is not None:
        dx = dx + dh.double()
        off = off + 8 * F32 * dh.double().abs()
    dw = (dy * u).sum(0)
    # rows are added in fp32 inside groups of them, the groups in 64 bits
    dw_off = (h.shape[0] / 512 + 16) * F32 * (dy * u).abs().sum(0)
    return dx, off, dw, dw_off


# ---- attention ----

def visible(n, m, causal, device):
    i, j = torch.arange(n, device=device)[:, None], torch.arange(m, device=device)[None]
    return (j <= i + m - n) if causal else torch.ones(n, m, dtype=torch.bool, device=device)


def attention(q, k, v, causal, scale, dout=None):
    """One head of one sequence, in 64 bits: q (n, d), k, v (m, d).  Returns a dict of values and of bounds ("..._off") for results whose
    probabilities and dS are rounded to bf16 and everything else to fp32, without the last rounding."""
    q, k, v = q.double(), k.double(), v.double()
    n, d = q.shape
    m = k.shape[0]
    see = visible(n, m, causal, q.device)
    s = torch.where(see, q @ k.T * scale, -math.inf)
    top = s.amax(1, keepdim=True) if m else torch.full((n, 1), -math.inf, dtype=torch.float64, device=q.device)
    e = torch.where(see, (s - torch.where(top == -math.inf, 0.0, top)).exp(), 0.0)
    total = e.sum(1, keepdim=True)
    some = total > 0
    p = e / torch.where(some, total, 1.0)
    lse = torch.where(some, top + torch.where(some, total, 1.0).log(), -math.inf)[:, 0]
    out = p @ v
    # a score is a sum of d products in fp32, then a product or two; an exponent of size z in base 2 is off by its own rounding
    size = (q.abs() @ k.abs().T * scale).amax() if n and m else torch.zeros((), dtype=torch.float64)
    score = (d + 4) * F32 * float(size) * 2
    rel = 2 * score + 16 * F32 * (1 + m ** 0.5)              # of a probability: score, exponential, the sum, its reciprocal
    half = HALF[torch.bfloat16]
    r = {"out": out, "lse": lse, "out_off": (half + rel) * (p @ v.abs()),
         "lse_off": 2 * score + 16 * F32 * (1 + lse.abs().nan_to_num(posinf=0.0))}
    if dout is not None:
        g = dout.double()
        dp = g @ v.T
        delta = (g * out).sum(1, keepdim=True)
        ds = p * (dp - delta)
        # what is given as `out` has its last rounding too
        delta_off = (g.abs() * (r["out_off"] + half * (out.abs() + r["out_off"]))).sum(1, keepdim=True) + (d + 4) * F32 * (g * out).abs().sum(1, keepdim=True)
        dp_off = (d + 4) * F32 * (g.abs() @ v.abs().T)
        p_rel = 2 * rel + r["lse_off"].amax() if n else 0.0
        ds_off = p * ((p_rel + 4 * F32) * (dp - delta).abs() + delta_off + dp_off) * (1 + half) + half * ds.abs()
        r.update(dq=scale * ds @ k, dk=scale * ds.T @ q, dv=p.T @ g,
                 dq_off=scale * ds_off @ k.abs() + (m + 8) * F32 * scale * (ds.abs() @ k.abs()),
                 dk_off=scale * ds_off.T @ q.abs() + (n + 8) * F32 * scale * (ds.abs().T @ q.abs()),
                 dv_off=(half + p_rel + (n + 8) * F32) * (p.T @ g.abs()))
    return r


# ---- token loss ----

def token_loss(z, targets, weights, policy=None):
    """loss, logp and dlogits in 64 bits; policy: (old, advantage, low, high, ref or None, kl)."""
    z = z.double()
    rows, vocab = z.shape
    ok = (targets >= 0) & (targets < vocab)
    w = torch.ones(rows, dtype=torch.float64, device=z.device) if weights is None else weights.double()
    loss = torch.zeros((), dtype=torch.float64, device=z.device)
    logp = torch.zeros(rows, dtype=torch.float64, device=z.device)
    dz = torch.zeros_like(z)
    for i in range(rows):
        if not bool(ok[i]):
            continue
        t = int(targets[i])
        every = z[i] - torch.logsumexp(z[i], 0)
        logp[i] = every[t]
        if float(w[i]) == 0.0:
            continue
        if policy is None:
            each, slope = -every[t], torch.tensor(-1.0, dtype=torch.float64, device=z.device)
        else:
            old, a, low, high, ref, kl = policy
            a = a[i].double()
            ratio = torch.exp(every[t] - old[i].double())
            inside = float(ratio) <= 1 + high if float(a) >= 0 else float(ratio) >= 1 - low
            c = ratio if inside else torch.tensor(1 + high if float(a) >= 0 else 1 - low, dtype=torch.float64, device=z.device)
            each = -a * c if float(a) != 0 else torch.zeros_like(a)
            slope = -a * ratio if inside and float(a) != 0 else torch.zeros_like(a)
            if kl:
                d = ref[i].double() - every[t]
                each, slope = each + kl * (torch.exp(d) - d - 1), slope + kl * (1 - torch.exp(d))
        loss = loss + w[i] * each
        hot = torch.zeros(vocab, dtype=torch.float64, device=z.device)
        hot[t] = 1.0
        dz[i] = w[i] * slope * (hot - every.exp())
    return loss, logp, dz
