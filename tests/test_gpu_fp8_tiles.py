"""The loops of the 8-bit operators' kernels: workgroups that take several tiles, contractions of every number of slabs that has a path of its own,
both tile widths, and norms, checkpoints whose waves take several rows.  Everything is compared with the definition in 64 bits, computed on the GPU by
elementary torch operations in float64; which kernel a shape reaches is asserted through the library's own rule.

Tolerances as in test_gpu_fp8.py: half a step for each rounding, 4e-7 (1 + |v|) for GELU and its derivative, 64 additions of 2^-24 for the norm's sums.
The matrix cores add 16 products at a time to 2^-16 of the largest of them, each of which may lose that: 2^-12 of the sum of magnitudes at most, which
is what contractions of less than 256 are held to (a single large product in 128 comes near: 2^-14.6 in 20 million sums); K 2^-23 of it for longer ones.
fp32 results are held to 2^-15 normwise too, twice what the entry point states."""
import math

import numpy as np
import pytest
import torch

import fp8_reference as R
from paper_2212_05191_amd import binding as B

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5
CHAIN = 2.0 ** -18      # 64 additions
FEW_Y, FEW_CODES, RING128, RING256 = range(4)
CUS = 256


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    global CUS
    CUS = torch.cuda.get_device_properties(0).multi_processor_count


def generator(seed):
    return torch.Generator(device="cuda:0").manual_seed(seed)


def normal(g, *shape, dtype="f32"):
    return torch.empty(shape, dtype=torch.float32, device="cuda:0").normal_(generator=g).to(TYPES[dtype])


def code_values(codes):
    return torch.from_numpy(R.CODES).to(codes.device)[codes.long()]


def row_scales(scales, C, K):
    """2^(byte - 127) of every value of rows [..., C, K]"""
    return torch.exp2(scales[..., :C].double() - 127.0).transpose(-1, -2).repeat_interleave(128, -1)[..., :K]


def row_values(codes, scales, K):
    return code_values(codes[..., :K]) * row_scales(scales, codes.shape[-2], K)


def weight_values(codes, scales, K):
    s = torch.exp2(scales.double() - 127.0).transpose(-1, -2).repeat_interleave(128, -2)[..., :codes.shape[-2], :]
    return code_values(codes[..., :K]) * s.repeat_interleave(128, -1)[..., :K]


def near(got, want, tol, what):
    off = torch.where(got == want, torch.zeros_like(want), (got - want).abs() - tol)
    off = torch.where(off.isnan(), torch.full_like(off, math.inf), off)
    if off.numel() and float(off.max()) > 0:
        at = np.unravel_index(int(off.argmax()), tuple(off.shape))
        raise AssertionError((what, at, float(got[at]), float(want[at]), float(tol.expand_as(want)[at]), int((off > 0).sum())))


def half(v, dtype):
    return v.abs() * R.HALF[dtype] + R.TINY[dtype]


def act(v, name):
    return v if name == "none" else v.clamp_min(0.0) if name == "relu" else 0.5 * v * torch.special.erfc(-v / math.sqrt(2.0))


def slope(v, name):
    if name == "relu":
        return (v > 0).double()
    return 0.5 * torch.special.erfc(-v / math.sqrt(2.0)) + v * torch.exp(-0.5 * v * v) / math.sqrt(2.0 * math.pi)


def check_rows8(codes, scales, value, slack, what):
    """codes[k, pitch], scales[blocks, >= k] of one group against value[k, Nout] known to +-slack"""
    k, Nout = value.shape
    s = row_scales(scales, k, Nout)
    step = s * torch.exp2(torch.floor(torch.log2((value.abs() / s).clamp_min(2.0 ** -6))) - 4.0)
    near(code_values(codes[:, :Nout]) * s, value, step * (1 + 2.0 ** -10) + slack, what)
    assert bool((codes[:, Nout:] == 0).all()), what
    blocks = lambda a: torch.nn.functional.pad(a, (0, -Nout % 128)).view(k, -(-Nout // 128), 128).amax(2)     # noqa: E731
    byte = scales[:, :k].t()
    sv = torch.exp2(byte.double() - 127.0)
    assert bool((blocks(value.abs() - slack) <= 448 * sv).all()), what
    assert bool(((blocks(value.abs() + slack) >= 224 * sv) | (byte == 1)).all()), what


def live_tiles(rows, BM, Nout, BN):
    return sum(-(-r // BM) for r in rows) * -(-Nout // BN)


def gemm_case(kernel, N, C, K, Nout, rows, dtype="bf16", activation="none", bias=False, y=True, y8=False, pre8=False, grad=False):
    assert R.kernel_of(CUS, N, C, K, Nout, y8 or pre8 or grad, activation) == kernel
    tile, slots = ((128, 128), 2 * CUS) if kernel == RING128 else ((128, 256), CUS)
    assert live_tiles(rows, tile[0], Nout, tile[1]) > slots, "a workgroup takes several tiles"
    g = generator(N + C + K + Nout)
    x8, xs = B.alloc_fp8_rows(N, C, K)
    w8, ws = B.alloc_fp8_weights(N, Nout, K)
    spread = lambda n, r: torch.exp(torch.rand((n, r, 1), device="cuda:0", generator=g) * 2 - 1)      # noqa: E731
    B.smile_fp8_pack_rows(normal(g, N, C, K) * spread(N, C) ** 2, x8, xs)
    B.smile_fp8_pack_weights(normal(g, N, Nout, K) * 0.05 * spread(N, Nout), w8, ws)
    b = 0.5 * normal(g, N, Nout) if bias else None
    b = None if b is None else b.to(TYPES[dtype])
    counts = torch.tensor(rows, dtype=torch.int32, device="cuda:0")
    for e in range(N):             # what lies beyond the valid rows must not matter
        x8[e, rows[e]:] = 0x7f
        xs[e, :, rows[e]:] = 0xff
    out = torch.full((N, C, Nout), 77.0, dtype=TYPES[dtype], device="cuda:0") if y else None
    o8, p8, g8 = ((*(t.fill_(0xAA) for t in B.alloc_fp8_rows(N, C, Nout)),) if want else (None, None) for want in (y8, pre8, False))
    if grad:
        g8 = B.alloc_fp8_rows(N, C, Nout)
        B.smile_fp8_pack_rows(2.0 * normal(g, N, C, Nout), *g8)
    B.smile_fp8_gemm(B.make_fp8_gemm_args(x8, xs, w8, ws, K, Nout, rows=counts, act=activation, bias=b, y=out, y8=o8[0], y_scale=o8[1],
                                          pre8=p8[0], pre_scale=p8[1], grad8=g8[0], grad_scale=g8[1], dtype=dtype))
    for e in range(N):
        k = rows[e]
        x, w = row_values(x8[e, :k], xs[e], K), weight_values(w8[e], ws[e], K)
        p, size = x @ w.T, x.abs() @ w.abs().T
        if b is not None:
            p, size = p + b[e].double(), size + b[e].double().abs()
        err = (K * 2.0 ** -23 if K >= 256 else 2.0 ** -12) * size
        if grad:
            kept = row_values(g8[0][e, :k], g8[1][e], Nout)
            v = p * slope(kept, activation)
            verr = err * slope(kept, activation).abs() + p.abs() * 4e-7 * (1 + kept.abs())
        else:
            v = act(p, activation)
            verr = err * 1.13 + (4e-7 * (1 + p.abs()) if activation == "gelu" else 0.0)
        if y:
            near(out[e, :k].double(), v, half(v, dtype) * (1 + 2.0 ** -10) + verr, ("y", e))
            if dtype == "f32":
                assert float((out[e, :k].double() - v).norm()) <= 2.0 ** -15 * float(v.norm()), ("y normwise", e)
            assert bool((out[e, k:] == 77.0).all()), ("y beyond the rows", e)
        for name, (codes, scales), value, slack in (("y8", o8, v, verr), ("pre8", p8, p, err)):
            if codes is not None:
                check_rows8(codes[e, :k], scales[e], value, slack, (name, e))
                assert bool((codes[e, k:] == 0xAA).all()) and bool((scales[e, :, k:C] == 0xAA).all()), (name, e)


EPILOGUES = {
    "y, bias": dict(bias=True), "y f16 gelu": dict(dtype="f16", activation="gelu"), "y f32 relu, bias": dict(dtype="f32", activation="relu", bias=True),
    "8 bits gelu, bias, kept": dict(activation="gelu", bias=True, y=False, y8=True, pre8=True),
    "8 bits relu, y f32, kept": dict(dtype="f32", activation="relu", y8=True, pre8=True),
    "8 bits, y f16": dict(dtype="f16", y8=True), "y gelu, kept": dict(activation="gelu", pre8=True),
    "slope gelu": dict(activation="gelu", y8=True, grad=True), "slope relu f32": dict(dtype="f32", activation="relu", grad=True),
    "slope gelu, 8 bits": dict(activation="gelu", y=False, y8=True, grad=True),
}
CYCLE = (290, 0, 129, 128, 1, 257, 40)


@pytest.mark.parametrize("epilogue", EPILOGUES)
@pytest.mark.parametrize("K", (128, 256, 384, 512, 1032))      # one, two, three, four and nine slabs
def test_ring_from_tile_to_tile(K, epilogue):
    rows = [CYCLE[e % 7] for e in range(70)]
    gemm_case(RING128, 70, 290, K, 1160, rows, **EPILOGUES[epilogue])


@pytest.mark.parametrize("epilogue", ("y, bias", "8 bits gelu, bias, kept", "slope gelu"))
def test_ring_bands_of_row_tiles(epilogue):
    gemm_case(RING128, 2, 1500, 384, 3400, [1500, 1100], **EPILOGUES[epilogue])       # twelve and nine row tiles


@pytest.mark.parametrize("dtype", ("bf16", "f16", "f32"))
@pytest.mark.parametrize("K,Nout,bias", [(1928, 1352, True), (2048, 1536, False), (2176, 1304, False)])      # an odd last block; whole tiles
def test_wide_ring_from_tile_to_tile(dtype, K, Nout, bias):
    rows = [(300, 0, 129, 256, 1, 33)[e % 6] for e in range(64)]
    gemm_case(RING256, 64, 300, K, Nout, rows, dtype=dtype, bias=bias)


def test_checkpoint_of_relu_of_many_rows():
    """Waves of the pass over codes next to zero that take several rows; columns of zero weights, whose sums are zero."""
    N, C, K, Nout = 30, 300, 128, 1160
    g = generator(5)
    x8, xs = B.alloc_fp8_rows(N, C, K)
    w8, ws = B.alloc_fp8_weights(N, Nout, K)
    w = 0.05 * normal(g, N, Nout, K)
    w[:, 5::61] = 0.0
    B.smile_fp8_pack_rows(normal(g, N, C, K), x8, xs)
    B.smile_fp8_pack_weights(w, w8, ws)
    rows = [(300, 0, 7, 299, 150)[e % 5] for e in range(N)]
    p8, ps = (t.fill_(0xAA) for t in B.alloc_fp8_rows(N, C, Nout))
    out = torch.zeros((N, C, Nout), dtype=torch.bfloat16, device="cuda:0")
    B.smile_fp8_gemm(B.make_fp8_gemm_args(x8, xs, w8, ws, K, Nout, rows=torch.tensor(rows, dtype=torch.int32, device="cuda:0"), act="relu",
                                          y=out, pre8=p8, pre_scale=ps))
    for e in range(N):
        k = rows[e]
        exact = row_values(x8[e, :k], xs[e], K) @ weight_values(w8[e], ws[e], K).T
        got = p8[e, :k, :Nout]
        wrong = ((got > 0) & (got < 0x80)) != (exact > 2.0 ** -10 * row_scales(ps[e], k, Nout))
        assert not bool(wrong.any()), (e, int(wrong.sum()))
        assert bool((p8[e, k:] == 0xAA).all()) and bool((p8[e, :k, Nout:] == 0).all())
        size = row_values(x8[e, :k], xs[e], K).abs() @ weight_values(w8[e], ws[e], K).abs().T
        check_rows8(p8[e, :k], ps[e], exact, 2.0 ** -12 * size, ("pre8", e))


# ------------------------------------------------------------------ norm

@pytest.mark.parametrize("dtype", ("bf16", "f16", "f32"))
@pytest.mark.parametrize("T,d,lanes", [(33000, 72, 16), (17003, 200, 32), (9001, 512, 64), (13005, 1024, 64), (8300, 1600, 64), (4099, 1032, 64),
                                       (1000, 1600, 256), (2100, 2056, 256), (1101, 4096, 256), (2500, 8192, 256), (1030, 8200, 256), (1100, 16384, 256)])
def test_norm_of_several_rows_a_lane_group(dtype, T, d, lanes):
    assert T > 768 * (256 // lanes)      # at most 768 workgroups backward, 1024 forward
    g = generator(T + d)
    x, res = normal(g, T, d, dtype=dtype), (3.0 * normal(g, T, d)).to(TYPES[dtype])
    w = (1.0 + 0.1 * normal(g, d)).to(TYPES[dtype])
    dy, extra = normal(g, T, d, dtype=dtype), normal(g, T, d, dtype=dtype)
    total, y, ds = (torch.full_like(x, 9.0) for _ in range(3))
    rstd, dw = torch.zeros(T, device="cuda:0"), torch.full((d,), 9.0, device="cuda:0")
    y8, y8s = B.alloc_fp8_rows(1, T, d)
    y8.fill_(0xAA)
    B.smile_rms_norm(x, res, w, EPS, sum=total, y=y, y8=y8, y8_scale=y8s, rstd=rstd)
    s, weight = total.double(), w.double()
    both = x.double() + res.double()
    near(s, both, half(both, dtype) + both.abs() * 2.0 ** -24, "sum")
    want_rstd = torch.rsqrt(s.square().mean(1) + EPS)
    near(rstd.double(), want_rstd, want_rstd * CHAIN, "rstd")
    u = s * want_rstd[:, None]
    want = u * weight
    near(y.double(), want, half(want, dtype) + want.abs() * CHAIN, "y")
    check_rows8(y8[0], y8s[0], want, want.abs() * CHAIN, "y8")
    alone = torch.full_like(x, 9.0)
    B.smile_rms_norm(total, None, w, EPS, y=alone)
    assert torch.equal(alone, y)

    ws = torch.full((B.smile_rms_norm_backward_workspace_bytes(T, d),), 0x5A, dtype=torch.uint8, device="cuda:0")
    B.smile_rms_norm_backward(dy, total, w, rstd, ds, dw, ws, dsum=extra)
    gw = dy.double() * weight
    mean = (gw * u).mean(1, keepdim=True)
    want_ds = extra.double() + want_rstd[:, None] * (gw - u * mean)
    slack = want_rstd[:, None] * (gw.abs() + u.abs() * (gw * u).abs().mean(1, keepdim=True)) * 2 * CHAIN
    near(ds.double(), want_ds, half(want_ds, dtype) + slack + extra.double().abs() * 2.0 ** -23, "ds")
    terms = dy.double() * u
    near(dw.double(), terms.sum(0), 2 * CHAIN * terms.abs().sum(0) + 1e-30, "dweight")
