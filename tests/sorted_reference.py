"""The operators of a layer without dropped tokens and of its optimizer, from their definitions in 64 bits (torch, any device)."""
import math

import torch

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}     # half a step, relative
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}   # and among the subnormals
E32 = 2.0 ** -24


def half_step(v, dtype):
    return v.abs() * HALF[dtype] + TINY[dtype]


def topk(logits, bias, k, normalize):
    """idx, weight, p (all N columns) and v"""
    v = logits.clone()
    if bias is not None:
        v = torch.where(bias == -math.inf, -math.inf, logits + bias)          # one addition in 32 bits
    vd = v.double()
    top = vd.amax(1, keepdim=True)
    e = torch.where(vd == -math.inf, 0.0, torch.exp(vd - torch.where(top == -math.inf, 0.0, top)))
    p = e / e.sum(1, keepdim=True).clamp_min(1e-300)
    order = torch.argsort(v, dim=1, descending=True, stable=True)[:, :k]
    none = v.gather(1, order) == -math.inf
    w = p.gather(1, order).masked_fill(none, 0.0)
    if normalize:
        w = w / w.sum(1, keepdim=True).clamp_min(1e-300)
    return torch.where(none, -1, order).to(torch.int32), w, p, v


def topk_backward(p, idx, weight, dweight, normalize, count, coef):
    """The Jacobian of the softmax applied to what reaches p, and the magnitudes of its terms (which cancel to zero in the columns that normalised weights leave
    alone: there the value is this computation's own rounding, 2^-53 of them for each of N terms)"""
    none = idx < 0
    at = idx.long().clamp_min(0)
    dw = dweight.double().masked_fill(none, 0.0)
    dp = torch.zeros_like(p) if count is None else (coef * count.double()).expand_as(p).clone()
    size = dw.abs()
    if normalize:
        total = p.gather(1, at).masked_fill(none, 0.0).sum(1, keepdim=True).clamp_min(1e-300)
        size = (size + (size * weight).sum(1, keepdim=True)) / total
        dw = ((dw - (dw * weight).sum(1, keepdim=True)) / total).masked_fill(none, 0.0)
    size = dp.abs().scatter_add(1, at, size.masked_fill(none, 0.0))
    dp = dp.scatter_add(1, at, dw)
    return p * (dp - (p * dp).sum(1, keepdim=True)), p * (size + (p * size).sum(1, keepdim=True))


def sort_experts(idx, N):
    """By hand, on the host: count, start, pos, source"""
    T, k = idx.shape
    rows = [[] for _ in range(N)]
    for pair, e in enumerate(idx.flatten().tolist()):
        if 0 <= e < N:
            rows[e].append(pair)
    source = [pair for group in rows for pair in group]
    pos = [-1] * (T * k)
    for r, pair in enumerate(source):
        pos[pair] = r
    count = [len(group) for group in rows]
    start = [sum(count[:e]) for e in range(N + 1)]
    as_int = lambda v: torch.tensor(v, dtype=torch.int32)                      # noqa: E731
    return as_int(count), as_int(start), as_int(pos).view(T, k), as_int(source + [-1] * (T * k - len(source)))


def act(v, name):
    return {"none": lambda: v, "relu": lambda: torch.where(v < 0, torch.zeros_like(v), v), "gelu": lambda: v * 0.5 * torch.special.erfc(-v / math.sqrt(2.0))}[name]()


def act_grad(v, name):
    if name == "gelu":
        return 0.5 * torch.special.erfc(-v / math.sqrt(2.0)) + v * torch.exp(-0.5 * v * v) / math.sqrt(2.0 * math.pi)
    return torch.ones_like(v) if name == "none" else (v > 0).double()


def groups(start, rows):
    return [(0, rows)] if start is None else list(zip(start.tolist()[:-1], start.tolist()[1:]))


def linear(x, w, bias, name, residual, start):
    """y, pre and the sum of the magnitudes of pre's terms; rows of no group are NaN"""
    rows, F = x.shape[0], w.shape[1]
    y, pre, size = (torch.full((rows, F), math.nan, dtype=torch.float64, device=x.device) for _ in range(3))
    for e, (lo, hi) in enumerate(groups(start, rows)):
        if lo == hi:
            continue
        a, b = x[lo:hi].double(), w[e].double()
        p, m = a @ b.T, a.abs() @ b.abs().T
        if bias is not None:
            p, m = p + bias[e].double(), m + bias[e].double().abs()
        pre[lo:hi], size[lo:hi] = p, m
        y[lo:hi] = act(p, name)
        if residual is not None:
            y[lo:hi] += residual[lo:hi].double()
    return y, pre, size


def linear_backward(dy, x, w, pre, name, start):
    """(value, sum of the magnitudes of its terms, the same with dy (1 + |pre|) in place of g = dy act'(pre)) of dx, dw, dbias; g is not rounded.  An error of act' is absolute,
    so that it counts with the third, not with the second (GELU's derivative passes zero at -0.75).  The fourth has ones for g: a rounding of g among the subnormals is
    absolute too."""
    N, F, K = w.shape
    rows, dev = x.shape[0], x.device
    zeros = lambda *s: torch.zeros(s, dtype=torch.float64, device=dev)         # noqa: E731
    out = {"dx": [zeros(rows, K) * math.nan for _ in range(4)], "dw": [zeros(N, F, K) for _ in range(4)], "dbias": [zeros(N, F) for _ in range(4)]}
    for e, (lo, hi) in enumerate(groups(start, rows)):
        if lo == hi:
            continue
        g = dy[lo:hi].double()
        wide = g.abs()
        if name != "none":
            wide = wide * (1 + pre[lo:hi].double().abs())
            g = g * act_grad(pre[lo:hi].double(), name)
        a, b = x[lo:hi].double(), w[e].double()
        for i, (ga, xa, wa) in enumerate(((g, a, b), (g.abs(), a.abs(), b.abs()), (wide, a.abs(), b.abs()), (torch.ones_like(g), a.abs(), b.abs()))):
            out["dx"][i][lo:hi] = ga @ wa
            out["dw"][i][e] = ga.T @ xa
            out["dbias"][i][e] = ga.sum(0)
    return out


# ------------------------------------------------------------------ AdamW

def mix(x):
    x = x ^ (x >> 16)
    x = (x * 0x7FEB352D) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0x846CA68B) & 0xFFFFFFFF
    return x ^ (x >> 16)


def random_bits(seed, t, tensor, n, device):
    key = mix(mix(mix(seed & 0xFFFFFFFF) ^ t) ^ tensor)
    return mix((torch.arange(n, dtype=torch.int64, device=device) + key) & 0xFFFFFFFF)


def m_value(code, scale):
    """e4m3 codes [n] times 2^(scale - 127) of blocks of 128"""
    c = code.long().view(-1, 128)
    e, f = (c >> 3) & 15, (c & 7).double()
    v = torch.where(e == 0, f * 2.0 ** -9, (8.0 + f) * torch.exp2(e.double() - 10.0))
    v = torch.where((c & 0x7F) == 0x7F, math.nan, v) * torch.where(c >= 128, -1.0, 1.0)
    return (v * torch.exp2(scale[:c.shape[0], None].double() - 127.0)).view(-1)


def v_value(code, scale):
    c = code.long().view(-1, 128)
    v = torch.where(c == 0, 0.0, (8.0 + (c & 7).double()) * torch.exp2((c >> 3).double() - 33.0))
    return (v * torch.exp2(scale[:c.shape[0], None].double() - 127.0)).view(-1)


def m_round(m, r, b):
    """m rounded to its code's value under the block bytes b, by the random bits r (both per element)"""
    scale = torch.exp2(b.double() - 127.0)
    u = m.abs() / scale
    x = torch.floor(torch.log2(u.clamp_min(2.0 ** -6)))
    x = torch.where(torch.exp2(x) > u.clamp_min(2.0 ** -6), x - 1, torch.where(torch.exp2(x + 1) <= u, x + 1, x))
    step = torch.exp2(x - 3.0)
    return torch.floor(u / step + r.double() / 65536.0) * step * scale * torch.sign(m)


def v_round(v, r, b):
    scale = torch.exp2(b.double() - 127.0)
    u = v / scale
    safe = u.clamp_min(2.0 ** -200)
    x = torch.floor(torch.log2(safe))
    x = torch.where(torch.exp2(x) > safe, x - 1, torch.where(torch.exp2(x + 1) <= safe, x + 1, x))
    step = torch.exp2(x - 3.0)
    q = torch.floor(u / step + r.double() / 65536.0) * step
    return torch.where(v == 0, torch.zeros_like(v), q.clamp_min(1.125 * 2.0 ** -30) * scale)


def m_byte(largest):
    """least byte >= 1 whose power of two brings `largest` to 448 or less"""
    return torch.tensor([max(1, next(b for b in range(1, 255) if v <= 448.0 * 2.0 ** (b - 127))) for v in largest.tolist()])


def v_byte(largest):
    return torch.tensor([max(1, math.frexp(v)[1] - 1 + 127) if v > 0 else 1 for v in largest.tolist()])


def adamw(p, g, m, v, t, lr, decay, beta1, beta2, eps):
    m = beta1 * m + (1.0 - beta1) * g
    v = beta2 * v + (1.0 - beta2) * g * g
    update = m / (1.0 - beta1 ** t) / (torch.sqrt(v / (1.0 - beta2 ** t)) + eps)
    return p - lr * (decay * p + update), m, v, update
