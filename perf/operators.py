"""The 8-bit operators of a layer, what they are timed on and how their inputs are made.

Operators: the root-mean-square norm with the residual's addition (16-bit and 8-bit outputs, backward pass), the matrix
product of 8-bit operands with a scale for each block of 128 (dense and grouped by expert), and activation checkpoints in 8
bits with their use in the backward pass.  A case is one of

  norm    s = x + residual, y = rms_norm(s) in the storage type and in 8 bits (unpacked here, so that it can be compared);
  back    a training step of the norm: forward in the storage type, then the gradients;
  proj    norm with 8-bit output, then a dense product with 8-bit weights: what stands in front of every projection;
  ffn     the expert FFN on 8-bit rows of every expert's buffer: up, activation, 8-bit hidden rows, down;
  train   a training step of the expert FFN: the forward pass keeps its hidden rows and pre-activations in 8 bits, the
          backward pass reads them: gradients of the rows and of both weights.

8-bit rows are e4m3 codes [N][C][K up to a multiple of 128] and power-of-two scales [N][K / 128][C up to a multiple of 16],
byte b standing for 2^(b - 127); weights have a scale for each 128 x 128 block.  prepare() makes everything that a program
holds: inputs, packed weights, output buffers and workspaces.  run() computes the plain form, or calls the library.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False
EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _norm(name, op, T, d, dtype="bf16"):
    return dict(name=name, op=op, T=T, d=d, dtype=dtype)


def _proj(name, T, d, F, dtype="bf16", act="none"):
    return dict(name=name, op="proj", T=T, d=d, F=F, dtype=dtype, act=act)


def _ffn(name, op, N, C, tokens, d, F, dtype="bf16", act="gelu", bias=False, skew=False):
    return dict(name=name, op=op, N=N, C=C, tokens=tokens, d=d, F=F, dtype=dtype, act=act, bias=bias, skew=skew)


def listed():
    return [
        # One token in front of a layer while text is generated: nothing but latency.
        _norm("norm_one_token", "norm", 1, 1024),
        # The large model's micro-batch.
        _norm("norm_batch", "norm", 16384, 1024),
        # Training, a last batch that divides by nothing, in half precision and of a width that ends inside a block.
        _norm("back_ragged_f16", "back", 5003, 960, "f16"),
        # Training, the largest batch.
        _norm("back_large", "back", 65536, 1024),
        # A dense projection of a handful of sequences that generate together: every weight read for 16 rows.
        _proj("proj_generate", 16, 1024, 4096),
        # The same projection over a batch.
        _proj("proj_batch", 16384, 1024, 4096, act="gelu"),
        # One sequence of 128 tokens through 16 experts of the base width: eight rows an expert.
        _ffn("ffn_one_sequence", "ffn", 16, 16, 128, 768, 3072),
        # Odd buffers, odd widths, half precision, ReLU and biases.
        _ffn("ffn_ragged_f16", "ffn", 15, 417, 5003, 960, 3840, "f16", "relu", bias=True),
        # 64 experts of the large model.
        _ffn("ffn_large", "ffn", 64, 320, 16384, 1024, 4096),
        # 128 experts behind a skewed router: full buffers, nearly empty and empty ones.
        _ffn("ffn_skewed", "ffn", 128, 512, 32768, 768, 3072, skew=True),
        # Training steps: the base layer on its micro-batch, ...
        _ffn("train_base", "train", 16, 512, 8192, 768, 3072),
        # ... and the large model.
        _ffn("train_large", "train", 64, 320, 16384, 1024, 4096),
    ]


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _cost(c):
    w = work(c)
    return w["bytes"] / 6e12 + w["flops"] / 1e15


def draw(rng):
    most = {}
    for c in listed():
        most[c["op"]] = max(most.get(c["op"], 0.0), _cost(c))
    while True:
        op = rng.choice(("norm", "back", "proj", "ffn", "ffn", "train", "train"))
        # 32 bits for the norm alone: what follows an 8-bit rounding is no nearer than that
        dtype = rng.choices(("bf16", "f16", "f32"), (65, 20, 15 if op in ("norm", "back") else 0))[0]
        d = max(8, round(_log_uniform(rng, 64, 2048) / 8) * 8)
        if rng.random() < 0.6:
            d = max(64, d // 64 * 64)
        if op in ("norm", "back"):
            c = _norm("", op, round(_log_uniform(rng, 1, 65536)), d, dtype)
        elif op == "proj":
            c = _proj("", round(_log_uniform(rng, 1, 32768)), d, max(64, round(d * rng.choice((1, 2, 3, 4)) / 8) * 8), dtype,
                      rng.choice(("none", "relu", "gelu")))
        else:
            d = max(64, d // 64 * 64)
            N, tokens = round(_log_uniform(rng, 1, 128)), round(_log_uniform(rng, 16, 32768))
            C = max(1, math.ceil(rng.choice((1.0, 1.25, 2.0)) * tokens / N))
            c = _ffn("", op, N, C, tokens, d, d * rng.choice((2, 3, 4, 4)), dtype, rng.choice(("gelu", "gelu", "relu")),
                     bias=op == "ffn" and rng.random() < 0.3, skew=rng.random() < 0.3)
        del c["name"]
        if _cost(c) <= most[op]:
            return c


def _up(v, q):
    return (v + q - 1) // q * q


# ---- inputs

def _pack(v, square=False):
    """8-bit rows of v[N][R][K] (square: one scale for each 128 x 128 block): codes, scales."""
    N, R, K = v.shape
    Kp, KB = _up(K, 128), _up(K, 128) // 128
    Rp = _up(R, 128) if square else R
    a = torch.zeros((N, Rp, Kp), dtype=torch.float32, device=v.device)
    a[:, :R, :K] = v
    b = a.view(N, Rp // 128, 128, KB, 128) if square else a.view(N, Rp, 1, KB, 128)
    # the smallest power of two that brings the largest magnitude to 448 or less
    m, p = torch.frexp(b.abs().amax((2, 4), keepdim=True))                   # m in [0.5, 1): 448 = 0.875 * 2^9
    e = torch.where(m == 0, -126, torch.clamp(p - 9 + (m > 0.875).int(), min=-126))
    codes = torch.ldexp(b, -e).to(torch.float8_e4m3fn).view(N, Rp, Kp)[:, :R].contiguous()
    e = (e + 127).to(torch.uint8)[:, :, 0, :, 0]
    scales = torch.zeros((N, KB, _up(e.shape[1], 16)), dtype=torch.uint8, device=v.device)
    scales[:, :, :e.shape[1]] = e.transpose(1, 2)
    return codes.view(torch.uint8), scales


def _rows8(N, C, K, dev):
    return (torch.zeros((N, C, _up(K, 128)), dtype=torch.uint8, device=dev),
            torch.zeros((N, _up(K, 128) // 128, _up(C, 16)), dtype=torch.uint8, device=dev))


def prepare(case, seed):
    dev = "cuda:0"
    st = TYPES[case["dtype"]]
    g = torch.Generator(device=dev).manual_seed(int(seed))

    def normal(*shape, std=1.0, dtype=st):
        return torch.empty(shape, dtype=torch.float32, device=dev).normal_(0.0, std, generator=g).to(dtype)

    s = dict(case)
    s["st"] = st
    if case["op"] in ("norm", "back", "proj"):
        T, d = case["T"], case["d"]
        # a stream that has grown with depth, with a few channels far larger than the others
        s["x"], s["residual"] = normal(T, d), normal(T, d, std=3.0)
        s["residual"][:, ::97] *= 20
        s["weight"] = (1.0 + normal(d, std=0.1, dtype=torch.float32)).to(st)
        s["sum"], s["y"] = torch.zeros_like(s["x"]), torch.zeros_like(s["x"])
        s["rstd"] = torch.zeros(T, dtype=torch.float32, device=dev)
        s["y8"], s["y8_scale"] = _rows8(1, T, d, dev)
        s["unpacked"] = torch.zeros((T, d), dtype=torch.bfloat16, device=dev)
        if case["op"] == "back":
            s["dy"], s["dsum"] = normal(T, d), normal(T, d)
            s["ds"], s["dweight"] = torch.zeros_like(s["x"]), torch.zeros(d, dtype=torch.float32, device=dev)
        if case["op"] == "proj":
            s["w8"], s["w8_scale"] = _pack(normal(1, case["F"], d, std=0.02, dtype=torch.float32), True)
            s["out"] = torch.zeros((T, case["F"]), dtype=st, device=dev)
        return s
    N, C, d, F = (case[k] for k in ("N", "C", "d", "F"))
    p = torch.ones(N, device=dev)
    if case["skew"]:          # Zipf ranking over the experts
        p = (torch.randperm(N, device=dev, generator=g).float() + 1.0) ** -1.2
    expert = torch.multinomial(p, case["tokens"], replacement=True, generator=g)
    s["rows"] = torch.bincount(expert, minlength=N).clamp(max=C).to(torch.int32)
    live = (torch.arange(C, device=dev) < s["rows"][:, None])[:, :, None]
    s["xe8"], s["xe_scale"] = _pack(normal(N, C, d, dtype=torch.float32) * live)
    w1, w2 = normal(N, F, d, std=0.02, dtype=torch.float32), normal(N, d, F, std=0.02, dtype=torch.float32)
    s["w1"], s["w1_scale"] = _pack(w1, True)
    s["w2"], s["w2_scale"] = _pack(w2, True)
    s["b1"] = normal(N, F, std=0.02) if case["bias"] else None
    s["b2"] = normal(N, d, std=0.02) if case["bias"] else None
    s["h8"], s["h_scale"] = _rows8(N, C, F, dev)
    s["ye"] = torch.zeros((N, C, d), dtype=st, device=dev)
    if case["op"] == "train":
        s["w1t"], s["w1t_scale"] = _pack(w1.transpose(1, 2), True)
        s["w2t"], s["w2t_scale"] = _pack(w2.transpose(1, 2), True)
        s["dye"] = normal(N, C, d) * live
        s["pre8"], s["pre_scale"] = _rows8(N, C, F, dev)
        s["dye8"], s["dye_scale"] = _rows8(N, C, d, dev)
        s["dpre8"], s["dpre_scale"] = _rows8(N, C, F, dev)
        s["dpre"] = torch.zeros((N, C, F), dtype=st, device=dev)
        s["dxe"] = torch.zeros((N, C, d), dtype=st, device=dev)
        s["dw1"] = torch.zeros((N, F, d), dtype=st, device=dev)
        s["dw2"] = torch.zeros((N, d, F), dtype=st, device=dev)
        # the weight gradient's scratch memory: the 8-bit operand widened to 16 bits
        s["workspace"] = torch.empty(N * C * max(d, F) * 2 + 4096, dtype=torch.uint8, device=dev)
    return s


# ---- plain forms

def _values(codes, scales, R, K, square=False):
    """What 8-bit rows stand for, in 32 bits."""
    v = codes.view(torch.float8_e4m3fn).float()
    f = torch.ldexp(torch.ones_like(scales, dtype=torch.float32), scales.int() - 127).transpose(1, 2)
    if square:
        f = f.repeat_interleave(128, 1)
    return (v * f[:, :R].repeat_interleave(128, 2))[:, :, :K]


def _round8(v):
    """v rounded to 8-bit rows, as the 32-bit values that they stand for."""
    codes, scales = _pack(v)
    return _values(codes, scales, v.shape[1], v.shape[2])


def _act(v, act):
    return v if act == "none" else torch.relu(v) if act == "relu" else 0.5 * v * (1.0 + torch.erf(v * math.sqrt(0.5)))


def _act_grad(v, act):
    if act == "relu":
        return (v > 0).float()
    return 0.5 * (1.0 + torch.erf(v * math.sqrt(0.5))) + v * torch.exp(-0.5 * v * v) * (1.0 / math.sqrt(2.0 * math.pi))


def _plain_norm(s):
    total = (s["x"].float() + s["residual"].float()).to(s["st"])
    v = total.float()
    rstd = torch.rsqrt(v.square().mean(1, keepdim=True) + EPS)
    return total, v, rstd, v * rstd * s["weight"].float()


def _plain(s):
    op, st = s["op"], s["st"]
    if op in ("norm", "back", "proj"):
        total, v, rstd, y = _plain_norm(s)
        if op == "norm":
            return {"sum": total, "y": y.to(st), "y8": _round8(y[None])[0].bfloat16()}
        if op == "proj":
            w = _values(s["w8"], s["w8_scale"], s["F"], s["d"], True)[0]
            return {"sum": total, "out": _act(_round8(y[None])[0] @ w.T, s["act"]).to(st)}
        dy, xh = s["dy"].float(), v * rstd
        gw = dy * s["weight"].float()
        ds = s["dsum"].float() + rstd * (gw - xh * (gw * xh).mean(1, keepdim=True))
        return {"sum": total, "y": y.to(st), "ds": ds.to(st), "dweight": (dy * xh).double().sum(0).float()}
    C, d, F, act = s["C"], s["d"], s["F"], s["act"]
    live = (torch.arange(C, device=s["rows"].device) < s["rows"][:, None])[:, :, None].float()
    xe = _values(s["xe8"], s["xe_scale"], C, d)
    w1, w2 = _values(s["w1"], s["w1_scale"], F, d, True), _values(s["w2"], s["w2_scale"], d, F, True)
    pre = torch.bmm(xe, w1.transpose(1, 2))
    if s["b1"] is not None:
        pre = pre + s["b1"].float()[:, None]
    h = _round8(_act(pre, act)) * live
    ye = torch.bmm(h, w2.transpose(1, 2))
    if s["b2"] is not None:
        ye = (ye + s["b2"].float()[:, None]) * live
    if op == "ffn":
        return {"ye": ye.to(st)}
    dye = s["dye"].float()
    dpre = torch.bmm(_round8(dye), w2) * _act_grad(_round8(pre), act) * live
    dxe = torch.bmm(_round8(dpre), w1)
    dw2 = torch.bmm(dye.transpose(1, 2), h)
    dw1 = torch.bmm(dpre.to(st).float().transpose(1, 2), xe)
    return {"ye": ye.to(st), "dxe": dxe.to(st), "dw1": dw1.to(st), "dw2": dw2.to(st)}


# ---- the library's calls

def _library(s):
    from paper_2212_05191_amd import binding as B

    op = s["op"]
    if op == "norm":
        B.smile_rms_norm(s["x"], s["residual"], s["weight"], EPS, sum=s["sum"], y=s["y"], y8=s["y8"], y8_scale=s["y8_scale"])
        B.smile_fp8_unpack_rows(s["y8"], s["y8_scale"], s["unpacked"])
        return {"sum": s["sum"], "y": s["y"], "y8": s["unpacked"]}
    if op == "back":
        if "workspace" not in s:
            s["workspace"] = torch.empty(B.smile_rms_norm_backward_workspace_bytes(s["T"], s["d"]), dtype=torch.uint8,
                                         device=s["x"].device)
        B.smile_rms_norm(s["x"], s["residual"], s["weight"], EPS, sum=s["sum"], y=s["y"], rstd=s["rstd"])
        B.smile_rms_norm_backward(s["dy"], s["sum"], s["weight"], s["rstd"], s["ds"], s["dweight"], s["workspace"],
                                  dsum=s["dsum"])
        return {"sum": s["sum"], "y": s["y"], "ds": s["ds"], "dweight": s["dweight"]}
    if op == "proj":
        if "args" not in s:       # the argument block, built once as a program would
            s["args"] = B.make_fp8_gemm_args(s["y8"], s["y8_scale"], s["w8"], s["w8_scale"], s["d"], s["F"], act=s["act"],
                                             y=s["out"])
        B.smile_rms_norm(s["x"], s["residual"], s["weight"], EPS, sum=s["sum"], y8=s["y8"], y8_scale=s["y8_scale"])
        B.smile_fp8_gemm(s["args"])
        return {"sum": s["sum"], "out": s["out"]}
    d, F, act, rows = s["d"], s["F"], s["act"], s["rows"]
    train = op == "train"
    if "up" not in s:
        pre = dict(pre8=s["pre8"], pre_scale=s["pre_scale"]) if train else {}
        s["up"] = B.make_fp8_gemm_args(s["xe8"], s["xe_scale"], s["w1"], s["w1_scale"], d, F, rows=rows, act=act, bias=s["b1"],
                                       y8=s["h8"], y_scale=s["h_scale"], dtype=s["dtype"], **pre)
        s["down"] = B.make_fp8_gemm_args(s["h8"], s["h_scale"], s["w2"], s["w2_scale"], F, d, rows=rows, bias=s["b2"], y=s["ye"])
        if train:
            s["dup"] = B.make_fp8_gemm_args(s["dye8"], s["dye_scale"], s["w2t"], s["w2t_scale"], d, F, rows=rows, act=act,
                                            y=s["dpre"], y8=s["dpre8"], y_scale=s["dpre_scale"], grad8=s["pre8"],
                                            grad_scale=s["pre_scale"])
            s["ddown"] = B.make_fp8_gemm_args(s["dpre8"], s["dpre_scale"], s["w1t"], s["w1t_scale"], F, d, rows=rows, y=s["dxe"])
    B.smile_fp8_gemm(s["up"])
    B.smile_fp8_gemm(s["down"])
    if not train:
        return {"ye": s["ye"]}
    B.smile_fp8_pack_rows(s["dye"], s["dye8"], s["dye_scale"], rows=rows)
    B.smile_fp8_gemm(s["dup"])
    B.smile_fp8_gemm(s["ddown"])
    B.smile_fp8_weight_grad(s["dye"], s["h8"], s["h_scale"], s["dw2"], s["workspace"], rows=rows)
    B.smile_fp8_weight_grad(s["dpre"], s["xe8"], s["xe_scale"], s["dw1"], s["workspace"], rows=rows)
    return {"ye": s["ye"], "dxe": s["dxe"], "dw1": s["dw1"], "dw2": s["dw2"]}


def run(s):
    return _library(s) if own else _plain(s)


# ---- the definition in 64 bits

def _exact8(v):
    """The nearest values of 8-bit rows along the last axis: three fraction bits, normal down to 2^-6 of the block's scale."""
    K = v.shape[-1]
    b = torch.nn.functional.pad(v, (0, -K % 128)).unflatten(-1, (-1, 128))
    top = b.abs().amax(-1, keepdim=True).clamp_min(448.0 * 2.0 ** -126)
    scale = torch.exp2(torch.ceil(torch.log2(top / 448.0)))
    u = b / scale
    step = torch.exp2(torch.floor(torch.log2(u.abs().clamp_min(2.0 ** -6))) - 3.0)
    return (torch.round(u / step) * step * scale).flatten(-2)[..., :K]


def _exact_operand(codes, scales, R, K, rows_per_scale):
    c = codes.to(torch.int64)
    sign, exponent, fraction = 1.0 - 2.0 * (c >> 7).double(), (c >> 3) & 15, (c & 7).double()
    v = sign * torch.where(exponent == 0, fraction * 2.0 ** -9, (8.0 + fraction) * torch.exp2(exponent.double() - 10.0))
    N, _, Kp = v.shape
    at_row = torch.arange(R, device=v.device) // rows_per_scale
    f = torch.exp2(scales.double() - 127.0)[:, :, at_row]                    # [N][K / 128][R]
    return (v.view(N, R, Kp // 128, 128) * f.transpose(1, 2)[..., None]).view(N, R, Kp)[:, :, :K]


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    phi = lambda v: 0.5 * torch.special.erfc(-v / math.sqrt(2.0))            # noqa: E731
    f = {"none": lambda v: v, "relu": lambda v: v.clamp_min(0.0), "gelu": lambda v: v * phi(v)}[case.get("act", "none")]
    if op in ("norm", "back", "proj"):
        total = s["x"].double() + s["residual"].double()
        kept = total.to(s["st"]).double()
        var = (kept * kept).sum(1, keepdim=True) / case["d"]
        unit = kept / torch.sqrt(var + EPS)
        y = unit * s["weight"].double()
        if op == "norm":
            return {"sum": kept, "y": y, "y8": _exact8(y)}
        if op == "proj":
            w = _exact_operand(s["w8"], s["w8_scale"], case["F"], case["d"], 128)[0]
            return {"sum": kept, "out": f(torch.matmul(_exact8(y), w.t()))}
        up = s["dy"].double() * s["weight"].double()
        ds = s["dsum"].double() + (up - unit * (up * unit).sum(1, keepdim=True) / case["d"]) / torch.sqrt(var + EPS)
        return {"sum": kept, "y": y, "ds": ds, "dweight": (s["dy"].double() * unit).sum(0)}
    C, d, F = case["C"], case["d"], case["F"]
    x = _exact_operand(s["xe8"], s["xe_scale"], C, d, 1)
    w1 = _exact_operand(s["w1"], s["w1_scale"], F, d, 128)
    w2 = _exact_operand(s["w2"], s["w2_scale"], d, F, 128)
    dead = torch.arange(C, device=x.device)[None, :] >= s["rows"][:, None]
    pre = torch.matmul(x, w1.mT)
    pre = pre if s["b1"] is None else pre + s["b1"].double().unsqueeze(1)
    h = _exact8(f(pre)).masked_fill(dead[..., None], 0.0)
    ye = torch.matmul(h, w2.mT)
    ye = ye if s["b2"] is None else (ye + s["b2"].double().unsqueeze(1)).masked_fill(dead[..., None], 0.0)
    if op == "ffn":
        return {"ye": ye}
    kept = _exact8(pre)
    slope = (kept > 0).double() if case["act"] == "relu" else phi(kept) + kept * torch.exp(-kept * kept / 2.0) / math.sqrt(2.0 * math.pi)
    dye = s["dye"].double()
    dpre = (torch.matmul(_exact8(dye), w2) * slope).masked_fill(dead[..., None], 0.0)
    return {"ye": ye, "dxe": torch.matmul(_exact8(dpre), w1), "dw1": torch.matmul(dpre.mT, x), "dw2": torch.matmul(dye.mT, h)}


def work(case):
    b = 4 if case["dtype"] == "f32" else 2
    d = case["d"]
    if case["op"] in ("norm", "back", "proj"):
        T = case["T"]
        if case["op"] == "norm":        # x, residual in; sum, y and its 8-bit form out
            return {"bytes": T * d * (4.0 * b + 1 + 1 / 128) + d * b, "flops": 8.0 * T * d}
        if case["op"] == "back":        # x, residual, dy, dsum in; sum, y, ds out; dweight
            return {"bytes": T * d * 7.0 * b + d * (b + 4.0), "flops": 16.0 * T * d}
        F = case["F"]
        return {"bytes": T * d * 3.0 * b + float(F) * d + T * F * float(b), "flops": 2.0 * T * d * F}
    N, C, F = case["N"], case["C"], case["F"]
    p = np.ones(N) if not case["skew"] else np.arange(1.0, N + 1.0) ** -1.2
    count = np.minimum(np.random.default_rng(3).multinomial(case["tokens"], p / p.sum()), C)
    kept, live = float(count.sum()), float((count > 0).sum())
    nbytes, flops = kept * d * (1 + 1 / 128 + b) + live * 2.0 * d * F, 4.0 * kept * d * F
    if case["op"] == "train":           # dye in; the transposed weights, dxe, dw1, dw2
        nbytes += kept * d * 2.0 * b + live * 2.0 * d * F + N * 2.0 * d * F * b
        flops *= 3
    return {"bytes": nbytes, "flops": flops}
