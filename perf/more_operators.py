"""The operators of a layer without dropped tokens and of its optimizer, what they are timed on and how their inputs are made.

Operators: the choice of k experts for a token with its weights and gradient, tokens sorted by expert and returned with their
weights (and the gradients), the matrix product of sorted or dense rows with bias, activation and residual in its epilogue (and its
gradients), and an AdamW step over many tensors with states in 32 or 8 bits.  A case is one of

  route     k experts of N for each of T tokens: indices, weights, the sum of the probabilities over the tokens;
  routes    the same as a training step: with the gradient of the logits, of the weights and of the balance term;
  sort      the (token, choice) pairs sorted by expert, and the tokens' rows moved there;
  back      the sorted rows returned: a weighted sum of k rows for each token, added to the residual stream;
  backs     the same as a training step: gradients of the sorted rows and of the weights, and of the tokens' rows;
  linear    y = act(x w^T + bias) + residual, dense or for each expert's rows;
  linears   the same as a training step: gradients of x, w and bias;
  adamw     one optimizer step over the tensors of a model's layers.

prepare() makes everything that a program holds: inputs, output buffers, workspaces.  run() computes the plain form, or calls the
library.
"""
from __future__ import annotations

import math

import torch

own = False
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BETA1, BETA2, ADAM_EPS, LR, DECAY = 0.9, 0.99, 1e-8, 1e-3, 0.1


def _route(name, op, T, N, k, normalize=True, bias=False, masked=0):
    return dict(name=name, op=op, T=T, N=N, k=k, normalize=normalize, bias=bias, masked=masked)


def _move(name, op, T, N, k, d, dtype="bf16", drop=0.0, skew=False, residual=False):
    return dict(name=name, op=op, T=T, N=N, k=k, d=d, dtype=dtype, drop=drop, skew=skew, residual=residual)


def _linear(name, op, N, M, K, F, dtype="bf16", act="none", bias=False, residual=False, skew=False, behind=0):
    return dict(name=name, op=op, N=N, M=M, K=K, F=F, dtype=dtype, act=act, bias=bias, residual=residual, skew=skew, behind=behind)


def _adamw(name, layers, N, d, F, dtype="bf16", states=32, master=False, grad="same"):
    return dict(name=name, op="adamw", layers=layers, N=N, d=d, F=F, dtype=dtype, states=states, master=master, grad=grad)


def listed():
    return [
        # One token while text is generated: nothing but latency.
        _route("route_one_token", "route", 1, 64, 2),
        # Training, the largest batch, many choices, a bias for each expert and some experts shut off by it.
        _route("route_train_large", "routes", 65536, 128, 8, normalize=False, bias=True, masked=5),
        # A last batch that divides by nothing, half precision, a few choices without an expert.
        _move("sort_ragged_f16", "sort", 5003, 15, 2, 960, "f16", drop=0.1),
        # The large model's micro-batch, four experts a token, a skewed router.
        _move("sort_large", "sort", 16384, 64, 4, 1024, skew=True),
        # A handful of sequences that generate together.
        _move("back_generate", "back", 16, 64, 2, 1024, residual=True),
        # Training, the large model's micro-batch.
        _move("back_train_large", "backs", 16384, 64, 4, 1024, residual=True),
        # A dense projection of a handful of sequences that generate together: every weight read for 16 rows.
        _linear("linear_generate", "linear", 1, 16, 1024, 4096, act="gelu", bias=True),
        # 64 experts of the large model, two experts a token.
        _linear("linear_experts", "linear", 64, 32768, 1024, 4096, act="gelu", bias=True),
        # Training, a dense down-projection that returns to the residual stream.
        _linear("linear_train_dense", "linears", 1, 16384, 4096, 1024, bias=True, residual=True),
        # Training, 15 experts of odd widths in half precision, rows behind the last expert's.
        _linear("linear_train_ragged_f16", "linears", 15, 10006, 960, 3840, "f16", act="gelu", bias=True, behind=37),
        # Fine-tuning of the small tensors of 12 layers: norms, biases and routers, in 32 bits.
        _adamw("adamw_small_tensors", 12, 16, 768, 0, "f32", 32, grad="f32"),
        # 16 experts of the large model with 8-bit states and 32-bit master weights.
        _adamw("adamw_experts_8bit", 1, 16, 1024, 4096, "bf16", 8, master=True),
    ]


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _cost(c):
    w = work(c)
    return w["bytes"] / 5e12 + w["flops"] / (1e15 if c.get("dtype") != "f32" else 1e14)


def _width(rng, lo, hi):
    d = max(8, round(_log_uniform(rng, lo, hi) / 8) * 8)
    return max(64, d // 64 * 64) if rng.random() < 0.6 else d


def draw(rng):
    most = {}
    for c in listed():
        most[c["op"]] = max(most.get(c["op"], 0.0), _cost(c))
    while True:
        op = rng.choice(("route", "routes", "sort", "back", "backs", "linear", "linear", "linears", "linears", "adamw", "adamw"))
        dtype = rng.choices(("bf16", "f16", "f32"), (60, 25, 15))[0]
        N = round(_log_uniform(rng, 1, 256))
        k = min(N, rng.choice((1, 2, 2, 3, 4, 6, 8)))
        T = round(_log_uniform(rng, 1, 65536))
        if op in ("route", "routes"):
            bias = rng.random() < 0.5
            c = _route("", op, T, N, k, rng.random() < 0.5, bias, rng.randrange(0, N // 4 + 1) if bias else 0)
        elif op in ("sort", "back", "backs"):
            c = _move("", op, T, N, k, _width(rng, 64, 2048), dtype, rng.choice((0.0, 0.0, 0.1, 0.5)), rng.random() < 0.3, rng.random() < 0.5)
        elif op in ("linear", "linears"):
            N = rng.choice((1, N))
            K = _width(rng, 32, 4096)
            F = max(64, round(K * rng.choice((0.25, 0.5, 1, 2, 3, 4)) / 8) * 8)
            # (no ReLU's derivative in 32 bits: the side of zero of a sum next to it goes by the order of its terms)
            act = rng.choice(("none", "gelu", "relu" if op == "linear" or dtype != "f32" else "gelu"))
            c = _linear("", op, N, round(_log_uniform(rng, 1, 32768)), K, F, dtype, act, rng.random() < 0.6,
                        rng.random() < 0.4, N > 1 and rng.random() < 0.4, rng.choice((0, 0, 1, 100)) if N > 1 else 0)
        else:
            d = _width(rng, 64, 1600)
            c = _adamw("", rng.randrange(1, 13), N, d, d * rng.choice((0, 0, 1, 2, 4)), dtype, rng.choice((32, 8)), dtype != "f32" and rng.random() < 0.6,
                       rng.choice(("same", "f32")))
        del c["name"]
        w = work(c)
        # (the smaller cases of a kind stand for the larger ones of its other direction too)
        if _cost(c) <= max(most.get(op, 0.0), 2e-4 if op in ("linear",) else 0.0) and w["bytes"] < 8e9:
            if op != "route" or c["T"] > 1:
                return c
        if op in ("route", "back") and c["T"] <= 4096:
            return c


# ---- inputs

def _generator(seed):
    return torch.Generator(device="cuda:0").manual_seed(int(seed))


def _normal(g, *shape, std=1.0, dtype=torch.float32):
    return torch.empty(shape, dtype=torch.float32, device="cuda:0").normal_(0.0, std, generator=g).to(dtype)


def _choose(g, T, N, k, skew, drop):
    """k different experts for each token, some of them left out (-1)."""
    score = torch.empty((T, N), device="cuda:0").exponential_(generator=g).log_().neg_()      # Gumbel
    if skew:          # Zipf ranking over the experts
        score += torch.log((torch.randperm(N, device="cuda:0", generator=g).float() + 1.0) ** -1.2)
    idx = torch.argsort(score, 1, descending=True)[:, :k].to(torch.int32)
    if drop:
        idx = torch.where(torch.rand((T, k), device="cuda:0", generator=g) < drop, -1, idx)
    return idx.contiguous()


def _sorted(idx, N):
    """counts, first rows, each pair's row (-1: none) and each row's pair, sorted by expert and then by the pair's place."""
    flat = idx.reshape(-1).long()
    some = (flat >= 0) & (flat < N)
    key = torch.where(some, flat, N)
    order = torch.sort(key, stable=True).indices
    count = (key[:, None] == torch.arange(N, device=key.device)).sum(0) if key.numel() * N < 1 << 24 else torch.zeros(
        N + 1, dtype=torch.int64, device=key.device).index_add_(0, key, torch.ones_like(key))[:N]
    start = torch.cat([torch.zeros(1, dtype=torch.int64, device=key.device), torch.cumsum(count, 0)])
    row = torch.empty_like(key)
    row[order] = torch.arange(key.numel(), device=key.device)
    pos = torch.where(some, row, -1).view(idx.shape)
    source = torch.where(torch.arange(key.numel(), device=key.device) < start[N], order, -1)
    return {"count": count.to(torch.int32), "start": start.to(torch.int32), "pos": pos.to(torch.int32), "source": source.to(torch.int32)}


def _tensors(case):
    """(elements, whether weight decay applies) of the tensors of a layer, as many times as there are layers."""
    N, d, F = case["N"], case["d"], case["F"]
    one = [(d, False), (N * d, True), (N, False), (d + 3, False)]
    if F:
        one += [(N * F * d, True), (N * F, False), (N * d * F, True), (N * d, False)]
    return one * case["layers"]


def prepare(case, seed):
    dev = "cuda:0"
    g = _generator(seed)
    s = dict(case)
    st = s["st"] = TYPES[case.get("dtype", "f32")]
    op = case["op"]
    if op in ("route", "routes"):
        T, N, k = case["T"], case["N"], case["k"]
        s["logits"] = _normal(g, T, N, std=2.0)
        s["bias"] = None
        if case["bias"]:
            s["bias"] = _normal(g, N, std=0.5)
            s["bias"][torch.randperm(N, device=dev, generator=g)[:case["masked"]]] = -math.inf
        s["idx"], s["weight"] = torch.zeros((T, k), dtype=torch.int32, device=dev), torch.zeros((T, k), device=dev)
        s["p_sum"] = torch.zeros(N, device=dev)
        if op == "routes":
            s["dweight"] = _normal(g, T, k)
            s["count"] = torch.full((N,), T * k // N, dtype=torch.int32, device=dev) + torch.randint(0, 7, (N,), device=dev, generator=g, dtype=torch.int32)
            s["dlogits"] = torch.zeros((T, N), device=dev)
            s["coef"] = 0.01 * N / (float(T) * T * k)
        return s
    if op in ("sort", "back", "backs"):
        T, N, k, d = (case[n] for n in ("T", "N", "k", "d"))
        s["idx"] = _choose(g, T, N, k, case["skew"], case["drop"])
        if op == "sort":
            s["x"] = _normal(g, T, d, dtype=st)
            s["count"], s["start"] = (torch.zeros(n, dtype=torch.int32, device=dev) for n in (N, N + 1))
            s["pos"], s["source"] = torch.full((T, k), -1, dtype=torch.int32, device=dev), torch.full((T * k,), -1, dtype=torch.int32, device=dev)
            s["xs"] = torch.zeros((T * k, d), dtype=st, device=dev)
            return s
        s["pos"] = _sorted(s["idx"], N)["pos"]
        s["weight"] = torch.softmax(_normal(g, T, k), 1)
        s["ys"] = _normal(g, T * k, d, dtype=st)
        s["residual"] = _normal(g, T, d, std=3.0, dtype=st) if case["residual"] else None
        s["y"] = torch.zeros((T, d), dtype=st, device=dev)
        if op == "backs":
            s["dy"], s["dxs"] = _normal(g, T, d, dtype=st), _normal(g, T * k, d, dtype=st)
            s["dys"], s["dweight"] = torch.zeros((T * k, d), dtype=st, device=dev), torch.zeros((T, k), device=dev)
            s["dx"] = torch.zeros((T, d), dtype=st, device=dev)
        return s
    if op in ("linear", "linears"):
        N, M, K, F = (case[n] for n in ("N", "M", "K", "F"))
        rows = M + case["behind"]
        s["start"] = None
        s["most"] = M
        if N > 1:
            idx = _choose(g, M, N, 1, case["skew"], 0.0)
            s["start"] = _sorted(idx, N)["start"]
            s["most"] = max(1, int((s["start"][1:] - s["start"][:-1]).max()))
        s["x"] = _normal(g, rows, K, dtype=st)
        s["w"] = _normal(g, N, F, K, std=K ** -0.5, dtype=st)
        s["bias"] = _normal(g, N, F, std=0.1, dtype=st) if case["bias"] else None
        s["residual"] = _normal(g, rows, F, std=2.0, dtype=st) if case["residual"] else None
        s["y"] = torch.zeros((rows, F), dtype=st, device=dev)
        if op == "linears":
            s["pre"] = torch.zeros((rows, F), dtype=st, device=dev) if case["act"] != "none" else None
            s["dy"] = _normal(g, rows, F, dtype=st)
            s["dx"], s["dw"] = torch.zeros((rows, K), dtype=st, device=dev), torch.zeros((N, F, K), dtype=st, device=dev)
            s["dbias"] = torch.zeros((N, F), dtype=st, device=dev) if case["bias"] else None
        return s
    # One buffer of each kind for all tensors, as a program holds them; a tensor begins at a multiple of 2048 elements (16 scales).
    sizes = _tensors(case)
    s["tensors"], at = [], 0
    for n, decay in sizes:
        s["tensors"].append((at, n, DECAY if decay else 0.0))
        at += -(-n // 2048) * 2048
    live = torch.zeros(at, dtype=torch.bool, device=dev)
    for first, n, _ in s["tensors"]:
        live[first:first + n] = True
    p = _normal(g, at, std=0.02) * live
    s["param"], s["master"] = p.to(st), p if case["master"] else None
    s["grad"] = (_normal(g, at, std=1e-3) * live).to(torch.float32 if case["grad"] == "f32" else st)
    # states of a run that has gone on for a while: magnitudes that differ from element to element
    m, v = _normal(g, at, std=3e-4) * live, (_normal(g, at, std=1e-3) * live).square_()
    if case["states"] == 8:
        half = torch.full((1,), 0x8000, device=dev).expand(at)
        s["m"], s["m_scale"] = _pack_m(m, half)
        s["v"], s["v_scale"] = _pack_v(v, half)
        s["m_value"], s["v_value"] = (torch.zeros((at // 128, 128), dtype=torch.bfloat16, device=dev) for _ in range(2))
    else:
        s["m"], s["v"], s["m_scale"], s["v_scale"] = m, v, None, None
    s["lr"], s["step"] = torch.full((1,), LR, device=dev), torch.full((1,), 100, dtype=torch.int32, device=dev)
    s["seed"] = int(seed) & 0x7FFFFFFF
    return s


# ---- plain forms

def _act(v, act):
    return v if act == "none" else torch.relu(v) if act == "relu" else 0.5 * v * (1.0 + torch.erf(v * math.sqrt(0.5)))


def _act_grad(v, act):
    if act == "none":
        return torch.ones_like(v)
    if act == "relu":
        return (v > 0).float()
    return 0.5 * (1.0 + torch.erf(v * math.sqrt(0.5))) + v * torch.exp(-0.5 * v * v) * (1.0 / math.sqrt(2.0 * math.pi))


def _plain_route(s):
    v = s["logits"]
    if s["bias"] is not None:
        v = torch.where(torch.isinf(s["bias"]), -math.inf, v + s["bias"])
    top = v.amax(1, keepdim=True)
    e = torch.where(torch.isinf(v), 0.0, torch.exp(v - torch.where(torch.isinf(top), 0.0, top)))
    p = e / e.sum(1, keepdim=True).clamp_min(1e-30)
    idx = torch.sort(v, dim=1, descending=True, stable=True).indices[:, :s["k"]]
    none = torch.isinf(v.gather(1, idx))
    w = p.gather(1, idx)
    if s["normalize"]:
        w = w / w.sum(1, keepdim=True).clamp_min(1e-30)
    out = {"idx": torch.where(none, -1, idx).to(torch.int32), "weight": w, "p_sum": p.double().sum(0).float()}
    if s["op"] == "route":
        return out
    u = (s["coef"] * s["count"].float()).expand_as(p)
    if s["normalize"]:
        dw = s["dweight"] * ~none
        chosen = torch.zeros_like(p).scatter_(1, idx, w * (dw - (w * dw).sum(1, keepdim=True)))
    else:
        u = u.scatter_add(1, idx, s["dweight"] * ~none)
        chosen = 0.0
    out["dlogits"] = p * (u - (p * u).sum(1, keepdim=True)) + chosen
    return out


def _plain_sort(s):
    out = _sorted(s["idx"], s["N"])
    source = out["source"].long()
    live = (source >= 0)[:, None]
    out["xs"] = s["x"][torch.div(source.clamp_min(0), s["k"], rounding_mode="floor")] * live
    return out


def _plain_back(s):
    T, k, d, st = s["T"], s["k"], s["d"], s["st"]
    pos = s["pos"].long()
    live = pos >= 0
    at = pos.clamp_min(0)
    rows = s["ys"].float()[at.view(-1)].view(T, k, d) * live[..., None]
    w = s["weight"] * live
    y = (rows * w[..., None]).sum(1)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    if s["op"] == "back":
        return {"y": y.to(st)}
    dy = s["dy"].float()
    dys = torch.zeros((T * k + 1, d), dtype=torch.float32, device=y.device)
    dys[torch.where(live, pos, T * k).view(-1)] = (dy[:, None] * w[..., None]).reshape(T * k, d)
    dx = (s["dxs"].float()[at.view(-1)].view(T, k, d) * live[..., None]).sum(1)
    return {"y": y.to(st), "dys": dys[:T * k].to(st), "dweight": (dy[:, None] * rows).sum(2), "dx": dx.to(st)}


def _plain_linear(s):
    N, M, K, F, st, act = s["N"], s["M"], s["K"], s["F"], s["st"], s["act"]
    dev = s["x"].device
    # each expert's rows as a batch of `most`: row i of expert e is x[start[e] + i]
    if s["start"] is None:
        row = torch.arange(M, device=dev)[None]
        live = torch.ones((1, M), dtype=torch.bool, device=dev)
    else:
        start = s["start"].long()
        i = torch.arange(s["most"], device=dev)
        row, live = start[:-1, None] + i, i < (start[1:] - start[:-1])[:, None]
    take = torch.where(live, row, 0)
    put = torch.where(live, row, s["x"].shape[0]).view(-1)
    back = lambda v: torch.zeros((s["x"].shape[0] + 1, v.shape[-1]), dtype=torch.float32, device=dev).index_copy_(  # noqa: E731
        0, put[live.view(-1)], v.reshape(-1, v.shape[-1])[live.view(-1)])[:-1]
    x, w = s["x"].float()[take] * live[..., None], s["w"].float()
    pre = torch.bmm(x, w.transpose(1, 2))
    if s["bias"] is not None:
        pre = pre + s["bias"].float()[:, None]
    y = _act(pre, act)
    if s["residual"] is not None:
        y = y + s["residual"].float()[take]
    out = {"y": back(y).to(st)}
    if s["op"] == "linear":
        return out
    # what is kept for the backward pass is the pre-activation in the storage type
    kept = pre.to(st)
    g = s["dy"].float()[take] * _act_grad(kept.float(), act) * live[..., None]
    if s["pre"] is not None:
        out["pre"] = back(kept.float()).to(st)
    out["dx"] = back(torch.bmm(g, w)).to(st)
    out["dw"] = torch.bmm(g.transpose(1, 2), x).to(st)
    if s["bias"] is not None:
        out["dbias"] = g.double().sum(1).to(st)
    return out


# 8-bit states.  Blocks of 128 neighbouring elements share a power of two 2^(b - 127).  The first moment: e4m3 codes, b the least
# byte >= 1 with which the block's largest magnitude is at most 448.  The second moment: unsigned codes c of 5 exponent and 3 fraction
# bits, (1 + (c & 7) / 8) 2^((c >> 3) - 30) times the power of two of the block's largest value, 0 for c = 0, at least c = 1 for
# what is not 0.  Both round up or down by 16 random bits R: up where the part cut off is at least 1 - R / 65536 of a step.

def _blocks(v):
    n = v.numel()
    return torch.nn.functional.pad(v, (0, -n % 128)).view(-1, 128)


def _scale_bytes(b):
    r = b.numel()
    return torch.nn.functional.pad(b.to(torch.uint8), (0, -r % 16))


def _floor_random(u, r):
    """floor(u + R / 65536) in 64 bits."""
    return torch.floor(u.double() + r.double() / 65536.0)


def _pack_m(m, r):
    a, r = _blocks(m), _blocks(r)
    f, p = torch.frexp(a.abs().amax(1, keepdim=True))                  # f in [0.5, 1): 448 = 0.875 * 2^9
    e = torch.where(f == 0, -126, torch.clamp(p - 9 + (f > 0.875).int(), min=-126))
    u = torch.ldexp(a.abs().double(), -e)
    step = torch.exp2(torch.clamp(torch.frexp(u)[1] - 1, min=-6).double() - 3.0)
    q = _floor_random(u / step, r) * step
    codes = torch.where(a < 0, -q, q).float().to(torch.float8_e4m3fn).view(torch.uint8)
    return codes.contiguous().view(-1), _scale_bytes((e + 127).view(-1))


def _m_values(codes, scales):
    v = codes.view(torch.float8_e4m3fn).float().view(-1, 128)
    return v * torch.exp2(scales[:v.shape[0], None].double() - 127.0).float()


def _pack_v(v, r):
    a, r = _blocks(v), _blocks(r)
    e = torch.clamp(torch.frexp(a.amax(1, keepdim=True))[1] - 1, min=-126)
    u = torch.ldexp(a.double(), -e)                                    # at most 2
    x = torch.frexp(u)[1] - 1
    q = _floor_random(torch.ldexp(u, 3 - x), r).long()                 # 8 .. 16, eighths of 2^x
    code = (x.long() + 30) * 8 + q - 8
    code = torch.where(u == 0, 0, code.clamp(min=1))
    return code.to(torch.uint8).view(-1), _scale_bytes((e + 127).view(-1))


def _v_values(codes, scales):
    c = codes.view(-1, 128).long()
    v = torch.ldexp(1.0 + (c & 7).double() / 8.0, (c >> 3) - 30) * torch.exp2(scales[:c.shape[0], None].double() - 127.0)
    return torch.where(c == 0, 0.0, v).float()


def _mix(x):
    """A 32-bit integer hash: two rounds of xor-shift and multiplication."""
    x = x ^ (x >> 16)
    x = (x * 0x7FEB352D) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0x846CA68B) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _random_bits(seed, step, tensor, n, dev):
    """32 random bits of every element: low half for the first moment, high half for the second."""
    key = _mix(_mix(_mix(torch.tensor(seed, dtype=torch.int64, device=dev)) ^ step.long()) ^ tensor)
    return _mix((torch.arange(n, dtype=torch.int64, device=dev) + key) & 0xFFFFFFFF)


def _plain_adamw_tensor(s, i, first, n, decay):
    part = lambda name: s[name][first:first + n]                       # noqa: E731
    step = s["step"][0] + 1
    eight = s["states"] == 8
    c1, c2 = (1.0 - torch.pow(torch.tensor(b, dtype=torch.float64, device=step.device), step) for b in (BETA1, BETA2))
    grad = part("grad").float()
    blocks, to_block = slice(first // 128, (first + n + 127) // 128), (n + 127) // 128 * 128
    if eight:
        m = _m_values(s["m"][first:first + to_block], s["m_scale"][blocks]).view(-1)[:n]
        v = _v_values(s["v"][first:first + to_block], s["v_scale"][blocks]).view(-1)[:n]
    else:
        m, v = part("m"), part("v")
    p = part("master" if s["master"] is not None else "param").float()
    m = BETA1 * m + (1.0 - BETA1) * grad
    v = BETA2 * v + (1.0 - BETA2) * grad * grad
    lr = s["lr"][0]
    p = p - lr * (decay * p + (m / c1.float()) / (torch.sqrt(v / c2.float()) + ADAM_EPS))
    part("param").copy_(p)
    if s["master"] is not None:
        part("master").copy_(p)
    if not eight:
        part("m").copy_(m)
        part("v").copy_(v)
        return
    r = _random_bits(s["seed"], step, i, n, p.device)
    for name, (codes, scales) in (("m", _pack_m(m, r & 0xFFFF)), ("v", _pack_v(v, r >> 16))):
        s[name][first:first + to_block] = codes
        s[name + "_scale"][blocks] = scales[:to_block // 128]


def _plain_adamw(s):
    """A step in place, as an optimizer makes it."""
    for i, (first, n, decay) in enumerate(s["tensors"]):
        _plain_adamw_tensor(s, i, first, n, decay)
    s["step"] += 1
    if s["states"] == 8:
        return _adamw_outputs(s, _m_values(s["m"], s["m_scale"]).bfloat16(), _v_values(s["v"], s["v_scale"]).bfloat16())
    return _adamw_outputs(s, s["m"], s["v"])


def _adamw_outputs(s, m, v):
    out = {"param": s["param"], "m": m.view(-1), "v": v.view(-1), "step": s["step"]}
    return out if s["master"] is None else {**out, "master": s["master"]}


def _plain(s):
    op = s["op"]
    if op in ("route", "routes"):
        return _plain_route(s)
    if op == "sort":
        return _plain_sort(s)
    if op in ("back", "backs"):
        return _plain_back(s)
    return _plain_linear(s) if op in ("linear", "linears") else _plain_adamw(s)


# ---- the library's calls

def _library(s):
    from paper_2212_05191_amd import binding as B

    op = s["op"]
    dev = "cuda:0"
    scratch = lambda nbytes: torch.empty(nbytes, dtype=torch.uint8, device=dev)      # noqa: E731
    if op in ("route", "routes"):
        if "workspace" not in s:
            s["workspace"] = scratch(B.smile_topk_workspace_bytes(s["T"], s["N"]))
        B.smile_topk(s["logits"], s["idx"], s["weight"], bias=s["bias"], normalize=s["normalize"], p_sum=s["p_sum"], workspace=s["workspace"])
        out = {"idx": s["idx"], "weight": s["weight"], "p_sum": s["p_sum"]}
        if op == "routes":
            B.smile_topk_backward(s["logits"], s["idx"], s["dweight"], s["dlogits"], bias=s["bias"], normalize=s["normalize"], count=s["count"],
                                  coef=s["coef"])
            out["dlogits"] = s["dlogits"]
        return out
    if op == "sort":
        if "workspace" not in s:
            s["workspace"] = scratch(B.smile_sort_experts_workspace_bytes(s["T"], s["k"], s["N"]))
        B.smile_sort_experts(s["idx"], s["count"], s["start"], s["pos"], s["source"], s["workspace"])
        B.smile_sorted_dispatch(s["x"], s["pos"], s["xs"])
        return {n: s[n] for n in ("count", "start", "pos", "source", "xs")}
    if op in ("back", "backs"):
        B.smile_sorted_combine(s["ys"], s["pos"], s["y"], weight=s["weight"], residual=s["residual"])
        if op == "back":
            return {"y": s["y"]}
        B.smile_sorted_combine_backward(s["dy"], s["ys"], s["pos"], s["weight"], s["dys"], s["dweight"])
        B.smile_sorted_combine(s["dxs"], s["pos"], s["dx"])
        return {n: s[n] for n in ("y", "dys", "dweight", "dx")}
    if op in ("linear", "linears"):
        if "args" not in s:       # the argument blocks, built once as a program would
            s["args"] = B.make_linear_args(s["x"], s["w"], s["y"], bias=s["bias"], act=s["act"], residual=s["residual"], start=s["start"],
                                           pre=s.get("pre"))
            if op == "linears":
                s["bargs"] = B.make_linear_backward_args(s["dy"], s["x"], s["w"], dx=s["dx"], dw=s["dw"], dbias=s["dbias"], pre=s["pre"],
                                                         act=s["act"], start=s["start"])
                s["workspace"] = scratch(B.smile_linear_backward_workspace_bytes(s["bargs"]))
        B.smile_linear(s["args"])
        if op == "linear":
            return {"y": s["y"]}
        B.smile_linear_backward(s["bargs"], s["workspace"])
        return {n: s[n] for n in ("y", "pre", "dx", "dw", "dbias") if s[n] is not None}
    return _library_adamw(B, s)


def _library_adamw(B, s):
    eight = s["states"] == 8
    if "opt" not in s:
        cut = lambda name, lo, hi: None if s[name] is None else s[name][lo:hi]      # noqa: E731
        tensors = []
        for first, n, decay in s["tensors"]:
            b0, b1 = first // 128, first // 128 + -(-n // 2048) * 16
            end = first + (-(-n // 128) * 128 if eight else n)
            tensors.append(dict(param=cut("param", first, first + n), grad=cut("grad", first, first + n), master=cut("master", first, first + n),
                                m=cut("m", first, end), v=cut("v", first, end), m_scale=cut("m_scale", b0, b1), v_scale=cut("v_scale", b0, b1),
                                weight_decay=decay))
        s["opt"] = B.AdamW(tensors, beta1=BETA1, beta2=BETA2, eps=ADAM_EPS, seed=s["seed"])
    B.smile_adamw(s["opt"], s["lr"], s["step"])
    if not eight:
        return _adamw_outputs(s, s["m"], s["v"])
    B.smile_adamw_unpack_states(s["m"], s["m_scale"], s["v"], s["v_scale"], s["m_value"], s["v_value"])
    return _adamw_outputs(s, s["m_value"], s["v_value"])


def run(s):
    return _library(s) if own else _plain(s)


# ---- the definition in 64 bits

def _exact_act(v, act):
    return {"none": lambda: v, "relu": lambda: v.clamp_min(0.0), "gelu": lambda: v * 0.5 * torch.special.erfc(-v / math.sqrt(2.0))}[act]()


def _exact_slope(v, act):
    if act == "gelu":
        return 0.5 * torch.special.erfc(-v / math.sqrt(2.0)) + v * torch.exp(-v * v / 2.0) / math.sqrt(2.0 * math.pi)
    return torch.ones_like(v) if act == "none" else (v > 0).double()


def _exact_route(s, case):
    T, N, k = case["T"], case["N"], case["k"]
    v = s["logits"]
    if s["bias"] is not None:
        v = v + s["bias"]                                              # one addition in 32 bits decides, as in the definition
    left, idx = v.clone(), []
    for _ in range(k):                                                 # the largest that is left, the lowest index of equal ones
        best = left.max(1, keepdim=True).values
        e = torch.where(left == best, torch.arange(N, device=v.device), N).min(1, keepdim=True).values
        idx.append(torch.where(best == -math.inf, -1, e))
        left = left.scatter(1, e, -math.inf)
    idx = torch.cat(idx, 1)
    none = idx < 0
    p = torch.softmax(v.double(), 1).nan_to_num(0.0)                   # (a token without any expert)
    w = p.gather(1, idx.clamp_min(0)).masked_fill(none, 0.0)
    total = w.sum(1, keepdim=True)
    if case["normalize"]:
        w = torch.where(total > 0, w / total, 0.0)
    out = {"idx": idx.to(torch.int32), "weight": w, "p_sum": p.sum(0)}
    if case["op"] == "route":
        return out
    # L = sum of dweight * weight + coef * sum of count * p_sum, differentiated through the softmax
    dw = s["dweight"].double().masked_fill(none, 0.0)
    if case["normalize"]:
        dw = torch.where(total > 0, (dw - (dw * w).sum(1, keepdim=True)) / total, 0.0)
    dp = (s["coef"] * s["count"].double()).expand(T, N).scatter_add(1, idx.clamp_min(0), dw.masked_fill(none, 0.0))
    return {**out, "dlogits": p * (dp - (p * dp).sum(1, keepdim=True))}


def _exact_moves(s, case):
    T, N, k, d = (case[n] for n in ("T", "N", "k", "d"))
    if case["op"] == "sort":
        flat = s["idx"].reshape(-1).long()
        parts = [torch.nonzero(flat == e).view(-1) for e in range(N)]
        order = torch.cat(parts)
        count = torch.tensor([p.numel() for p in parts], dtype=torch.int32, device=flat.device)
        pos, source = s["pos"].clone().view(-1), s["source"].clone()
        pos[order] = torch.arange(order.numel(), dtype=torch.int32, device=flat.device)
        source[:order.numel()] = order.to(torch.int32)
        xs = s["xs"].double()
        xs[:order.numel()] = s["x"].double()[order // k]
        start = torch.tensor([0] + [p.numel() for p in parts], device=flat.device).cumsum(0).to(torch.int32)
        return {"count": count, "start": start, "pos": pos.view(T, k), "source": source, "xs": xs}
    y = s["y"].double() if s["residual"] is None else s["residual"].double()
    dx, dys, dweight = torch.zeros_like(y), torch.zeros(T * k, d, dtype=torch.float64, device=y.device), s["weight"].double() * 0.0
    for j in range(k):
        t = torch.nonzero(s["pos"][:, j] >= 0).view(-1)
        r, w = s["pos"][t, j].long(), s["weight"][t, j].double()[:, None]
        y = y.index_add(0, t, w * s["ys"][r].double())
        if case["op"] == "backs":
            dx.index_add_(0, t, s["dxs"][r].double())
            dys[r] = w * s["dy"][t].double()
            dweight[t, j] = (s["dy"][t].double() * s["ys"][r].double()).sum(1)
    return {"y": y} if case["op"] == "back" else {"y": y, "dys": dys, "dweight": dweight, "dx": dx}


def _exact_linear(s, case):
    N, M = case["N"], case["M"]
    start = [0, M] if s["start"] is None else s["start"].tolist()
    names = ("y", "pre", "dx", "dw", "dbias") if case["op"] == "linears" else ("y",)
    out = {n: torch.zeros(s[n].shape, dtype=torch.float64, device="cuda:0") for n in names if s[n] is not None}
    for e in range(N):
        at = slice(start[e], start[e + 1])
        if start[e] == start[e + 1]:
            continue
        x, w = s["x"][at].double(), s["w"][e].double()
        pre = x @ w.mT
        if s["bias"] is not None:
            pre = pre + s["bias"][e].double()
        y = _exact_act(pre, case["act"])
        out["y"][at] = y if s["residual"] is None else y + s["residual"][at].double()
        if case["op"] == "linears":
            if "pre" in out:
                out["pre"][at] = pre
            g = s["dy"][at].double() * _exact_slope(pre.to(s["st"]).double(), case["act"])
            out["dx"][at] = g @ w
            out["dw"][e] = g.mT @ x
            if "dbias" in out:
                out["dbias"][e] = g.sum(0)
    return out


def _exact_adamw(s, case):
    out = {"param": torch.zeros(s["param"].shape, dtype=torch.float64, device="cuda:0")}
    out["m"], out["v"] = torch.zeros_like(out["param"]), torch.zeros_like(out["param"])
    t = int(s["step"][0]) + 1
    for i, (first, n, decay) in enumerate(s["tensors"]):
        at, padded = slice(first, first + n), slice(first, first + -(-n // 2048) * 2048)
        blocks = slice(first // 128, first // 128 + -(-n // 2048) * 16)
        g, p = s["grad"][at].double(), (s["param"] if s["master"] is None else s["master"])[at].double()
        if case["states"] == 8:
            c = s["m"][padded].long().view(-1, 128)
            f = torch.where(((c >> 3) & 15) == 0, (c & 7) * 2.0 ** -9, (8.0 + (c & 7)) * torch.exp2(((c >> 3) & 15).double() - 10.0))
            m = (f * (1.0 - 2.0 * (c >> 7)) * torch.exp2(s["m_scale"][blocks].double() - 127.0)[:, None]).view(-1)[:n]
            c = s["v"][padded].long().view(-1, 128)
            f = torch.where(c == 0, 0.0, (8.0 + (c & 7)) * torch.exp2((c >> 3).double() - 33.0))
            v = (f * torch.exp2(s["v_scale"][blocks].double() - 127.0)[:, None]).view(-1)[:n]
        else:
            m, v = s["m"][at].double(), s["v"][at].double()
        m, v = m + (1.0 - BETA1) * (g - m), v + (1.0 - BETA2) * (g * g - v)
        update = m / (1.0 - BETA1 ** t) / (torch.sqrt(v / (1.0 - BETA2 ** t)) + ADAM_EPS)
        out["param"][at] = p - LR * (update + decay * p)
        if case["states"] == 8:
            r = _random_bits(s["seed"], torch.tensor(t, device="cuda:0"), i, n, "cuda:0")
            m, v = _exact_states(m, v, (r & 0xFFFF).double() / 65536.0, (r >> 16).double() / 65536.0)
        out["m"][at], out["v"][at] = m, v
    return {**out, "step": s["step"] + 1, **({} if s["master"] is None else {"master": out["param"]})}


def _exact_states(m, v, rm, rv):
    """Both moments rounded to the values of their codes; what a step of the code is follows from the value's own power of two."""
    n = m.numel()
    pad = lambda x: torch.nn.functional.pad(x, (0, -n % 128)).view(-1, 128)          # noqa: E731
    m, v, rm, rv = pad(m), pad(v), pad(rm), pad(rv)
    scale = torch.exp2(torch.ceil(torch.log2(m.abs().amax(1, keepdim=True).clamp_min(448.0 * 2.0 ** -126) / 448.0)))
    step = torch.exp2(torch.floor(torch.log2((m.abs() / scale).clamp_min(2.0 ** -6))) - 3.0) * scale
    m = torch.floor(m.abs() / step + rm) * step * torch.sign(m)
    least = torch.exp2(torch.floor(torch.log2(v.amax(1, keepdim=True).clamp_min(2.0 ** -126))) - 30.0) * 1.125
    step = torch.exp2(torch.floor(torch.log2(v.clamp_min(2.0 ** -300))) - 3.0)
    v = torch.where(v == 0, 0.0, torch.maximum(torch.floor(v / step + rv) * step, least))
    return m.view(-1)[:n], v.view(-1)[:n]


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op in ("route", "routes"):
        return _exact_route(s, case)
    if op in ("sort", "back", "backs"):
        return _exact_moves(s, case)
    return _exact_linear(s, case) if op in ("linear", "linears") else _exact_adamw(s, case)


def work(case):
    op = case["op"]
    if op in ("route", "routes"):         # logits in; indices and weights out; backward: logits, indices, dweight in, dlogits out
        T, N, k = case["T"], case["N"], case["k"]
        b = T * (4.0 * N + 8.0 * k) + 4.0 * N
        return {"bytes": b + (T * (4.0 * N + 4.0 * k) if op == "routes" else 0.0), "flops": 6.0 * T * N * (2 if op == "routes" else 1)}
    b = 4.0 if case["dtype"] == "f32" else 2.0
    if op in ("sort", "back", "backs"):
        T, k, d = case["T"], case["k"], case["d"]
        pairs = T * k * (1.0 - case["drop"])
        if op == "sort":                  # the tokens read once, each pair's row written
            return {"bytes": T * d * b + pairs * d * b + 12.0 * T * k, "flops": 1.0 * T * k}
        nbytes = pairs * d * b + T * d * b * (2 if case["residual"] else 1) + 8.0 * T * k
        if op == "backs":                 # dy in, dys out (ys is the forward's); dxs in, dx out
            nbytes += T * d * b + pairs * d * b + pairs * d * b + T * d * b + 4.0 * T * k
        return {"bytes": nbytes, "flops": pairs * d * (2.0 if op == "back" else 6.0)}
    if op in ("linear", "linears"):
        N, M, K, F = (case[n] for n in ("N", "M", "K", "F"))
        nbytes = b * (M * K + M * F + min(N, M) * float(F) * K + (M * F if case["residual"] else 0))
        if op == "linears":               # pre out, dy in, dx and dw out
            nbytes += b * (M * F * (1 if case["act"] == "none" else 2) + M * K + N * float(F) * K)
        return {"bytes": nbytes, "flops": 2.0 * M * K * F * (3 if op == "linears" else 1)}
    n = float(sum(n for n, _ in _tensors(case)))
    state = 8.0 if case["states"] == 32 else 2.0 + 2.0 / 128
    nbytes = n * ((4.0 if case["grad"] == "f32" else b) + 2 * state + (8.0 + b if case["master"] else 2 * b))
    return {"bytes": nbytes + (n * 4.0 if case["states"] == 8 else 0.0), "flops": 20.0 * n}
