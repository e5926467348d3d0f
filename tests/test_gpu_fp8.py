"""GPU parity of the 8-bit operators with their definition in 64 bits (fp8_reference.py).

Tolerances.  A rounding to a storage type is off by half a step (R.HALF relative, R.TINY among the subnormals), one to 8 bits by half the
distance of the codes (R.row_step).  fp32 sums: each of the n additions of a chain rounds by at most 2^-24 of the sum of
magnitudes, so n 2^-24 sum |terms| bounds the sum; the norm's chains are at most 64 long (eight columns a piece, a butterfly, a few waves).
The matrix cores add 16 products of 8-bit values at a time to 2^-16 of the largest of them, at most 2^-12 of the sum of magnitudes
(MFMA below, for values whose exponents are spread widely); of the normally distributed rows of the other tests they lose a few 2^-17, which
K 2^-23 sum |terms| covers from K = 256 on and the half steps of the 16-bit results below.  GELU and its derivative: 4e-7 (1 + |v|), from
the erfc approximation's 1.5e-7."""
import numpy as np
import pytest
import torch

import fp8_reference as R
from paper_2212_05191_amd import binding as B

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5
CHAIN = 2.0 ** -18      # 64 additions


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    B.load()


def dev(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a)).to("cuda:0")
    return t if dtype is None else t.to(TYPES[dtype])


def host(t):
    return t.detach().cpu().double().numpy() if t.is_floating_point() else t.detach().cpu().numpy()


def stored(a, dtype):
    """a rounded to a storage type, as float64"""
    return torch.from_numpy(np.asarray(a, np.float32)).to(TYPES[dtype]).double().numpy()


def near(got, want, tol, what):
    got, want, tol = np.broadcast_arrays(got, want, tol)
    if not got.size:
        return
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    with np.errstate(invalid="ignore"):
        off = np.where(same, 0.0, np.abs(got - want) - tol)
    worst = np.unravel_index(np.argmax(np.where(np.isnan(off), np.inf, off)), off.shape)
    assert not np.any(np.isnan(off)) and off[worst] <= 0, (what, worst, got[worst], want[worst], tol[worst])


def half(v, dtype):
    return np.abs(v) * R.HALF[dtype] + R.TINY[dtype]


# ------------------------------------------------------------------ packing

def check_packed(codes, scales, v, rows=None):
    want_c, want_s = R.pack_rows(v)
    codes, scales = host(codes), host(scales)
    for e in range(v.shape[0]):
        n = v.shape[1] if rows is None else min(max(int(rows[e]), 0), v.shape[1])
        nan = (want_c[e, :n] & 0x7f) == 0x7f
        assert np.array_equal((codes[e, :n] & 0x7f) == 0x7f, nan)
        assert np.array_equal(codes[e, :n][~nan], want_c[e, :n][~nan])
        assert np.array_equal(scales[e, :, :n], want_s[e, :, :n])
        assert np.all(codes[e, n:] == 0xAA) and np.all(scales[e, :, n:v.shape[1]] == 0xAA)


@pytest.mark.parametrize("dtype", ("bf16", "f16", "f32"))
@pytest.mark.parametrize("N,C,K,rows", [(1, 1, 8, None), (1, 1, 128, None), (3, 17, 136, (17, 0, 5)), (2, 33, 960, (40, -3)),
                                        (1, 70, 1600, None), (5, 16, 64, (1, 2, 3, 15, 16)), (1, 3, 4104, None)])
def test_pack_and_unpack_rows(dtype, N, C, K, rows):
    r = np.random.default_rng(N * C + K)
    v = r.standard_normal((N, C, K)) * np.exp(r.uniform(-12, 6, (N, C, 1)))
    v[r.random(v.shape) < 0.05] *= 300.0
    v[r.random(v.shape) < 0.05] = 0.0
    v[:, 0, : K // 2] = 0.0
    v = stored(v, dtype)
    src = dev(v, dtype)
    codes, scales = B.alloc_fp8_rows(N, C, K)
    codes.fill_(0xAA), scales.fill_(0xAA)
    counts = None if rows is None else dev(np.array(rows, np.int32))
    B.smile_fp8_pack_rows(src, codes, scales, rows=counts)
    check_packed(codes, scales, v, rows)
    out = torch.full((N, C, K), 77.0, dtype=TYPES[dtype], device="cuda:0")
    B.smile_fp8_unpack_rows(codes, scales, out, rows=counts)
    want = R.unpack_rows(host(codes), host(scales), K)
    got = host(out)
    for e in range(N):
        n = C if rows is None else min(max(rows[e], 0), C)
        near(got[e, :n], want[e, :n], 0.0 if dtype == "bf16" else half(want[e, :n], dtype) * (dtype == "f16"), "unpacked")
        assert np.all(got[e, n:] == 77.0)


def test_every_bfloat16_packs_to_the_nearest_code():
    bits = np.arange(65536, dtype=np.uint32)
    v = (bits << 16).view(np.float32).astype(np.float64)
    # neighbours in magnitude share a block with its largest, and, in a second copy, with a value 2^9 above
    order = np.argsort(np.where(np.isfinite(v), np.abs(v), np.inf), kind="stable")
    a = v[order].reshape(1, 512, 128)
    b = a.copy()
    with np.errstate(invalid="ignore", over="ignore"):
        b[:, :, 0] = stored(np.minimum(np.nanmax(np.where(np.isfinite(a), np.abs(a), 0), axis=2) * 512.0, 3e38), "bf16")
    v = np.concatenate([a, b], axis=1)
    src = torch.from_numpy(v.astype(np.float32)).to(torch.bfloat16).cuda()
    codes, scales = B.alloc_fp8_rows(1, 1024, 128)
    B.smile_fp8_pack_rows(src, codes, scales)
    check_packed(codes, scales, v)


@pytest.mark.parametrize("dtype", ("bf16", "f16", "f32"))
@pytest.mark.parametrize("N,Nout,K", [(1, 8, 8), (2, 128, 128), (3, 200, 136), (1, 960, 320), (2, 72, 1032)])
def test_pack_weights(dtype, N, Nout, K):
    r = np.random.default_rng(Nout + K)
    w = stored(0.02 * r.standard_normal((N, Nout, K)) * np.exp(r.uniform(-3, 3, (N, Nout, 1))), dtype)
    w[0, : Nout // 2, : K // 2] = 0.0
    w[-1, 1, 3] = np.nan
    w[-1, Nout - 1, K - 1] = np.inf
    codes, scales = B.alloc_fp8_weights(N, Nout, K)
    codes_t, scales_t = B.alloc_fp8_weights(N, K, Nout)
    for t in (codes, codes_t):
        t.fill_(0xAA)
    B.smile_fp8_pack_weights(dev(w, dtype), codes, scales, codes_t, scales_t)
    for c, s, v in ((codes, scales, w), (codes_t, scales_t, w.transpose(0, 2, 1))):
        want_c, want_s = R.pack_weights(v)
        c, s = host(c), host(s)
        nan = (want_c & 0x7f) == 0x7f
        assert np.array_equal((c & 0x7f) == 0x7f, nan) and np.array_equal(c[~nan], want_c[~nan])
        assert np.array_equal(s, want_s)
    only, only_s = B.alloc_fp8_weights(N, Nout, K)
    B.smile_fp8_pack_weights(dev(w, dtype), only, only_s)
    assert torch.equal(only, codes) and torch.equal(only_s, scales)


@pytest.mark.parametrize("T,d,n,m,cap", [(1, 64, 2, 2, 1), (300, 192, 2, 4, 30), (1000, 1600, 3, 5, 50)])
def test_dispatch_of_packed_rows(T, d, n, m, cap):
    r = np.random.default_rng(T)
    desc = B.make_desc(T, d, 128, n, m, cap, "bf16", "relu")
    ctx = B.Ctx(desc)
    g, l = r.integers(n, size=T), r.integers(m, size=T)
    seen, slot = {}, np.empty(T, np.int64)
    for t in range(T):
        k = seen.get((g[t], l[t]), 0)
        seen[g[t], l[t]] = k + 1
        slot[t] = k if k < cap else -1
    x8, xs = B.alloc_fp8_rows(1, T, d)
    x8.copy_(dev(r.integers(0, 256, x8.shape).astype(np.uint8)))
    xs.copy_(dev(r.integers(0, 256, xs.shape).astype(np.uint8)))
    xe8, xes = B.alloc_fp8_rows(n * m, cap, d)
    xe8.fill_(0xAA), xes.fill_(0xAA)
    i32 = lambda a: dev(a.astype(np.int32))      # noqa: E731
    B.smile_fp8_dispatch(ctx, x8, xs, i32(g), i32(l), i32(slot), xe8, xes)
    want_c, want_s = np.full(tuple(xe8.shape), 0xAA, np.uint8), np.full(tuple(xes.shape), 0xAA, np.uint8)
    c, s = host(x8), host(xs)
    for t in range(T):
        if slot[t] >= 0:
            want_c[g[t] * m + l[t], slot[t]] = c[0, t]
            want_s[g[t] * m + l[t], :, slot[t]] = s[0, :, t]
    assert np.array_equal(host(xe8), want_c) and np.array_equal(host(xes), want_s)
    ctx.close()


# ------------------------------------------------------------------ norm

NORMS = [(1, 8), (3, 64), (5, 136), (2, 960), (700, 200), (1030, 512), (1, 1024), (257, 1600), (1100, 2048), (9, 2056), (2, 4096),
         (3, 8200), (2, 16384), (5000, 72)]


@pytest.mark.parametrize("dtype", ("bf16", "f16", "f32"))
@pytest.mark.parametrize("T,d", NORMS)
def test_norm_and_its_gradient(dtype, T, d):
    r = np.random.default_rng(T * 7 + d)
    x, res = r.standard_normal((T, d)), 3.0 * r.standard_normal((T, d))
    res[:, ::97] *= 20.0
    x[T // 2], res[T // 2] = 0.0, 0.0                 # a row of nothing
    w, dy, extra = 1.0 + 0.1 * r.standard_normal(d), r.standard_normal((T, d)), r.standard_normal((T, d))
    x, res, w, dy, extra = (stored(a, dtype) for a in (x, res, w, dy, extra))
    X, W = dev(x, dtype), dev(w, dtype)
    total, y = torch.full_like(X, 9.0), torch.full_like(X, 9.0)
    rstd = torch.zeros(T, device="cuda:0")
    y8, y8s = B.alloc_fp8_rows(1, T, d)
    y8.fill_(0xAA)
    B.smile_rms_norm(X, dev(res, dtype), W, EPS, sum=total, y=y, y8=y8, y8_scale=y8s, rstd=rstd)
    s = host(total)
    near(s, x + res, half(x + res, dtype) + np.abs(x + res) * 2.0 ** -24, "sum")
    want_rstd, want = R.rms_norm(s, w, EPS)
    near(host(rstd), want_rstd, want_rstd * CHAIN, "rstd")
    near(host(y), want, half(want, dtype) + np.abs(want) * CHAIN, "y")
    got8, scales = R.unpack_rows(host(y8), host(y8s), d), host(y8s)
    near(got8[0], want, R.row_step(want[None], scales)[0] + np.abs(want) * CHAIN, "y8")
    assert np.all(host(y8)[:, :, d:] == 0)
    blocks = np.pad(np.abs(want), ((0, 0), (0, -d % 128))).reshape(T, -1, 128).max(2)
    sv = 2.0 ** (scales[0, :, :T].T.astype(np.float64) - 127)
    assert np.all(blocks <= 448 * sv * (1 + CHAIN)) and np.all((blocks >= 224 * sv * (1 - CHAIN)) | (scales[0, :, :T].T == 1))

    # without residual, one output at a time, in place
    y2 = dev(s, dtype)
    B.smile_rms_norm(y2, None, W, EPS, y=y2)
    assert torch.equal(y2, y)
    z8, z8s = B.alloc_fp8_rows(1, T, d)
    acc = dev(res, dtype)
    B.smile_rms_norm(X, acc, W, EPS, sum=acc, y8=z8, y8_scale=z8s)
    assert torch.equal(acc, total) and torch.equal(z8, y8) and torch.equal(z8s[:, :, :T], y8s[:, :, :T])

    for with_sum in (True, False):
        want_ds, want_dw = R.rms_norm_backward(dy, s, w, EPS, extra if with_sum else None)
        ds, dw = torch.full_like(X, 9.0), torch.full((d,), 9.0, device="cuda:0")
        ws = torch.full((B.smile_rms_norm_backward_workspace_bytes(T, d),), 0x5A, dtype=torch.uint8, device="cuda:0")
        B.smile_rms_norm_backward(dev(dy, dtype), total, W, rstd, ds, dw, ws, dsum=dev(extra, dtype) if with_sum else None)
        u = s * want_rstd[:, None]
        g = dy * w
        slack = want_rstd[:, None] * (np.abs(g) + np.abs(u) * np.mean(np.abs(g * u), axis=1)[:, None]) * 2 * CHAIN
        near(host(ds), want_ds, half(want_ds, dtype) + slack + np.abs(extra) * 2.0 ** -23, "ds")
        near(host(dw), want_dw, 2 * CHAIN * np.sum(np.abs(dy * u), axis=0) + 1e-30, "dweight")
        in_place = dev(dy, dtype)
        B.smile_rms_norm_backward(in_place, total, W, rstd, in_place, dw, ws, dsum=dev(extra, dtype) if with_sum else None)
        assert torch.equal(in_place, ds)


def test_norm_of_large_and_small_rows():
    d = 256
    x = np.stack([np.full(d, 1e15), np.full(d, 1e-15), np.where(np.arange(d) == 3, 3e4, 0.0), np.full(d, 1.5)])
    X = dev(x, "f32")
    y, rstd = torch.zeros_like(X), torch.zeros(4, device="cuda:0")
    y8, y8s = B.alloc_fp8_rows(1, 4, d)
    B.smile_rms_norm(X, None, torch.ones(d, device="cuda:0"), 1e-6, y=y, y8=y8, y8_scale=y8s, rstd=rstd)
    s = stored(x, "f32")
    _, want = R.rms_norm(s, np.ones(d), 1e-6)
    near(host(y), want, np.abs(want) * 2 * CHAIN, "y")
    near(R.unpack_rows(host(y8), host(y8s), d)[0], want, R.row_step(want[None], host(y8s))[0] + np.abs(want) * CHAIN, "y8")


# ------------------------------------------------------------------ product

def packed(v, weights=False):
    c, s = R.pack_weights(v) if weights else R.pack_rows(v)
    return (dev(c), dev(s)), (R.unpack_weights(c, s, v.shape[2]) if weights else R.unpack_rows(c, s, v.shape[2]))


def gemm_case(N, C, K, Nout, dtype="bf16", act="none", bias=False, rows=None, y=True, y8=False, pre8=False, grad=False, seed=0):
    r = np.random.default_rng(seed + N + C + K + Nout)
    (x8, xs), x = packed(r.standard_normal((N, C, K)) * np.exp(r.uniform(-2, 2, (N, C, 1))))
    (w8, wsc), w = packed(0.05 * r.standard_normal((N, Nout, K)) * np.exp(r.uniform(-1, 1, (N, Nout, 1))), True)
    counts = None if rows is None else dev(np.array(rows, np.int32))
    n = [C if rows is None else min(max(int(q), 0), C) for q in (rows if rows is not None else [0] * N)]
    for e in range(N):             # what lies beyond the valid rows must not matter
        if n[e] < C:
            x8[e, n[e]:] = 0x7f
            xs[e, :, n[e]:C] = 0xff
    b = stored(0.5 * r.standard_normal((N, Nout)), dtype) if bias else None
    out = torch.full((N, C, Nout), 77.0, dtype=TYPES[dtype], device="cuda:0") if y else None
    o8 = p8 = (None, None)
    if y8:
        o8 = B.alloc_fp8_rows(N, C, Nout)
        o8[0].fill_(0xAA), o8[1].fill_(0xAA)
    if pre8:
        p8 = B.alloc_fp8_rows(N, C, Nout)
        p8[0].fill_(0xAA), p8[1].fill_(0xAA)
    g8, g = (None, None), None
    if grad:
        g8, g = packed(2.0 * r.standard_normal((N, C, Nout)))
    args = B.make_fp8_gemm_args(x8, xs, w8, wsc, K, Nout, rows=counts, act=act, bias=None if b is None else dev(b, dtype), y=out,
                                y8=o8[0], y_scale=o8[1], pre8=p8[0], pre_scale=p8[1], grad8=g8[0], grad_scale=g8[1], dtype=dtype)
    B.smile_fp8_gemm(args)
    torch.cuda.synchronize()
    for e in range(N):
        k = n[e]
        p = x[e, :k] @ w[e].T + (0.0 if b is None else b[e])
        err = K * 2.0 ** -23 * (np.abs(x[e, :k]) @ np.abs(w[e]).T + (0.0 if b is None else np.abs(b[e])))
        if grad:
            slope = R.act_grad(g[e, :k], act)
            v = p * slope
            verr = err * np.abs(slope) + np.abs(p) * 4e-7 * (1 + np.abs(g[e, :k]))
        else:
            v = R.act(p, act)
            verr = err * 1.13 + (4e-7 * (1 + np.abs(p)) if act == "gelu" else 0.0)
        if y:
            got = host(out[e])
            near(got[:k], v, half(v, dtype) * (1 + 2.0 ** -10) + verr, ("y", e))
            assert np.all(got[k:] == 77.0)
        for given, (codes, scales), value, slack in ((y8, o8, v, verr), (pre8, p8, p, err)):
            if not given:
                continue
            c, s = host(codes[e]), host(scales[e])
            if k:
                got = R.unpack_rows(c[None, :k], s[None, :, :R.up(k, 16)], Nout)[0]
                near(got, value, R.row_step(value[None], s[None])[0] * (1 + 2.0 ** -10) + slack, ("8 bits", e))
                assert np.all(c[:k, Nout:] == 0)
                sv = 2.0 ** (s[:, :k].T.astype(np.float64) - 127)
                blocks = lambda a: np.pad(a, ((0, 0), (0, -Nout % 128))).reshape(k, -1, 128).max(2)    # noqa: E731
                assert np.all(blocks(np.abs(value) - slack) <= 448 * sv)
                assert np.all((blocks(np.abs(value) + slack) >= 224 * sv) | (s[:, :k].T == 1))
            assert np.all(c[k:] == 0xAA) and np.all(s[:, k:C] == 0xAA)


SHAPES = [  # N, C, K, Nout, rows
    (1, 1, 8, 8, None), (1, 1, 1024, 512, None), (2, 3, 136, 200, (3, 0)), (3, 16, 960, 320, (16, 5, 40)), (1, 33, 384, 128, None),
    (4, 40, 64, 264, (1, 40, 0, 33)), (2, 130, 768, 384, (130, 129)), (1, 300, 640, 520, None), (3, 257, 512, 256, (257, 128, 1)),
    (2, 520, 1600, 136, (513, 200)), (1, 129, 128, 1032, None), (5, 260, 256, 640, (260, 0, 127, 256, 64)), (1, 384, 2056, 768, None),
]


@pytest.mark.parametrize("N,C,K,Nout,rows", SHAPES)
def test_gemm_shapes(N, C, K, Nout, rows):
    gemm_case(N, C, K, Nout, rows=rows)
    gemm_case(N, C, K, Nout, rows=rows, act="gelu", bias=True, y=False, y8=True, pre8=True)
    gemm_case(N, C, K, Nout, rows=rows, act="gelu", y8=True, grad=True)


@pytest.mark.parametrize("dtype", ("bf16", "f16", "f32"))
@pytest.mark.parametrize("C,act,bias", [(5, "relu", True), (5, "gelu", False), (200, "none", True), (200, "gelu", True), (290, "relu", False)])
def test_gemm_types_and_epilogues(dtype, C, act, bias):
    rows = (C, C - 3)
    gemm_case(2, C, 520, 328, dtype, act, bias, rows)
    gemm_case(2, C, 520, 328, dtype, act, bias, rows, y=False, y8=True)
    gemm_case(2, C, 520, 328, dtype, act, bias, rows, y=True, y8=True, pre8=True)
    gemm_case(2, C, 520, 328, dtype, act, bias, rows, y=True, pre8=True)
    if act != "none":
        gemm_case(2, C, 520, 328, dtype, act, False, rows, y=True, grad=True)
        gemm_case(2, C, 520, 328, dtype, act, False, rows, y=False, y8=True, grad=True)


@pytest.mark.parametrize("N,C,K,Nout", [(40, 9, 520, 1032), (150, 1, 136, 72), (37, 32, 1024, 640)])
def test_gemm_many_groups_of_few_rows(N, C, K, Nout):
    rows = tuple((5 * k) % (C + 2) for k in range(N))
    gemm_case(N, C, K, Nout, rows=rows, act="gelu", bias=True, y=False, y8=True, pre8=True)
    gemm_case(N, C, K, Nout, "f16", rows=rows, act="relu", bias=True, y8=True)
    gemm_case(N, C, K, Nout, rows=rows, act="gelu", y8=True, grad=True)


@pytest.mark.parametrize("C", (7, 200))
def test_gemm_keeps_nan_to_its_row_and_column(C):
    r = np.random.default_rng(C)
    K, Nout = 512, 256
    (x8, xs), x = packed(r.standard_normal((1, C, K)))
    (w8, wsc), w = packed(r.standard_normal((1, Nout, K)), True)
    x8[0, 3, 100] = 0x7f
    w8[0, 140, 7] = 0xff
    out = torch.zeros((1, C, Nout), dtype=torch.float32, device="cuda:0")
    o8, os8 = B.alloc_fp8_rows(1, C, Nout)
    B.smile_fp8_gemm(B.make_fp8_gemm_args(x8, xs, w8, wsc, K, Nout, y=out))
    B.smile_fp8_gemm(B.make_fp8_gemm_args(x8, xs, w8, wsc, K, Nout, y8=o8, y_scale=os8))
    want = np.zeros((C, Nout), bool)
    want[3], want[:, 140] = True, True
    assert np.array_equal(np.isnan(host(out)[0]), want)
    assert np.array_equal((host(o8)[0] & 0x7f) == 0x7f, want)
    fine = x[0] @ w[0].T
    near(np.where(want, 0, host(out)[0]), np.where(want, 0, fine), K * 2.0 ** -23 * (np.abs(x[0]) @ np.abs(w[0]).T) + half(fine, "f32"), "the rest")


@pytest.mark.parametrize("C", (2, 150))
def test_gemm_at_the_ends_of_the_scales(C):
    """Operands whose scales multiply to 2^-100 and to 2^100: nothing is lost on the way."""
    r = np.random.default_rng(5)
    K, Nout = 256, 128
    for k in (-60, 50):
        (x8, xs), x = packed(r.standard_normal((1, C, K)) * 2.0 ** k)
        (w8, wsc), w = packed(r.standard_normal((1, Nout, K)) * 2.0 ** (k if k > 0 else k + 20), True)
        out = torch.zeros((1, C, Nout), dtype=torch.float32, device="cuda:0")
        B.smile_fp8_gemm(B.make_fp8_gemm_args(x8, xs, w8, wsc, K, Nout, y=out))
        want = x[0] @ w[0].T
        near(host(out)[0], want, K * 2.0 ** -23 * (np.abs(x[0]) @ np.abs(w[0]).T) + half(want, "f32"), k)


@pytest.mark.parametrize("C", (9, 140))
@pytest.mark.parametrize("K", (64, 512, 2048))
def test_gemm_of_codes_spread_over_all_exponents(C, K):
    r = np.random.default_rng(K + C)
    MFMA, Nout = 2.0 ** -12, 128

    def spread(rows):
        codes = r.integers(0, 0x7f, (1, rows, K)).astype(np.uint8) | (r.integers(0, 2, (1, rows, K)).astype(np.uint8) << 7)
        return codes

    x8, w8 = spread(C), spread(Nout)
    (X, XS), (W, WS) = B.alloc_fp8_rows(1, C, K), B.alloc_fp8_weights(1, Nout, K)
    X[:, :, :K], W[:, :, :K] = dev(x8), dev(w8)
    XS.fill_(127), WS.fill_(120)
    x, w = R.CODES[x8[0]], R.CODES[w8[0]] * 2.0 ** -7
    out = torch.zeros((1, C, Nout), dtype=torch.float32, device="cuda:0")
    B.smile_fp8_gemm(B.make_fp8_gemm_args(X, XS, W, WS, K, Nout, y=out))
    want, size = x @ w.T, np.abs(x) @ np.abs(w).T
    near(host(out)[0], want, MFMA * size, "spread")
    assert np.linalg.norm(host(out)[0] - want) <= 2.0 ** -12 * np.linalg.norm(want)


@pytest.mark.parametrize("N,C,K,Nout,rows,bias", [(16, 20, 1024, 4096, None, False), (3, 400, 768, 3000, (400, 0, 257), False), (2, 350, 1032, 2056, (340, 350), True)])
def test_checkpoint_of_relu_keeps_the_side_of_zero(N, C, K, Nout, rows, bias):
    """ReLU's derivative is one or zero by the kept pre-activation: none may be rounded over the border by the product's own error."""
    r = np.random.default_rng(N * C)
    (x8, xs), x = packed(r.standard_normal((N, C, K)) * np.exp(r.uniform(-2, 2, (N, C, 1))))
    (w8, wsc), w = packed(0.05 * r.standard_normal((N, Nout, K)), True)
    b = stored(0.01 * r.standard_normal((N, Nout)), "bf16") if bias else None
    counts = None if rows is None else dev(np.array(rows, np.int32))
    out = torch.zeros((N, C, Nout), dtype=torch.bfloat16, device="cuda:0")
    p8, ps = B.alloc_fp8_rows(N, C, Nout)
    p8.fill_(0xAA), ps.fill_(0xAA)
    B.smile_fp8_gemm(B.make_fp8_gemm_args(x8, xs, w8, wsc, K, Nout, rows=counts, act="relu", bias=None if b is None else dev(b, "bf16"), y=out,
                                          pre8=p8, pre_scale=ps, dtype="bf16"))
    for e in range(N):
        n = C if rows is None else rows[e]
        c, s = host(p8[e]), host(ps[e])
        assert np.all(c[n:] == 0xAA) and np.all(s[:, n:C] == 0xAA) and np.all(c[:n, Nout:] == 0)
        exact = x[e, :n] @ w[e].T + (0.0 if b is None else b[e])      # codes and scales: without a rounding that matters here
        step = np.repeat(2.0 ** (s[:, :n].T.astype(np.float64) - 127), 128, axis=1)[:, :Nout]
        got = c[:n, :Nout]
        wrong = ((got > 0) & (got < 0x80)) != (exact > 2.0 ** -10 * step)
        assert not wrong.any(), (e, int(wrong.sum()), np.argwhere(wrong)[:4], exact[wrong][:4])


# ------------------------------------------------------------------ weight gradient

@pytest.mark.parametrize("dtype", ("bf16", "f16", "f32"))
@pytest.mark.parametrize("N,C,Nout,K,rows", [(1, 1, 64, 64, None), (3, 17, 128, 192, (17, 0, 5)), (2, 300, 320, 960, (300, 129)), (1, 700, 64, 1600, None),
                                             # many tiles: bfloat16 without a widened copy
                                             (130, 70, 192, 320, tuple(k % 73 for k in range(130))), (256, 33, 64, 128, None), (33, 100, 320, 704, tuple(3 * k for k in range(33)))])
def test_weight_grad(dtype, N, C, Nout, K, rows):
    r = np.random.default_rng(C + K)
    (x8, xs), x = packed(r.standard_normal((N, C, K)) * np.exp(r.uniform(-1, 1, (N, C, 1))))
    dy = stored(r.standard_normal((N, C, Nout)), dtype)
    counts = None if rows is None else dev(np.array(rows, np.int32))
    DY = dev(dy, dtype)
    for e in range(N):
        if rows is not None:       # beyond the valid rows: anything
            x8[e, rows[e]:] = 0x7f
            DY[e, rows[e]:] = float("nan")
    dw = torch.full((N, Nout, K), 77.0, dtype=TYPES[dtype], device="cuda:0")
    ws = torch.empty(B.smile_fp8_weight_grad_workspace_bytes(N, C, K, dtype), dtype=torch.uint8, device="cuda:0").fill_(0xFF)
    B.smile_fp8_weight_grad(DY, x8, xs, dw, ws, rows=counts)
    got = host(dw)
    for e in range(N):
        n = C if rows is None else rows[e]
        xv = x[e, :n]
        want = dy[e, :n].T @ xv
        size = np.abs(dy[e, :n]).T @ np.abs(xv)
        operand = size * R.HALF["f16"] if dtype == "f16" else 0.0       # widening to half precision may round its subnormals
        near(got[e], want, half(want, dtype) + (n + 1) * 2.0 ** -23 * size + operand, ("dw", e))


@pytest.mark.parametrize("N,C,Nout,K", [(256, 40, 64, 192), (300, 65, 128, 256)])
def test_weight_grad_passes_over_scales_beyond_the_rows(N, C, Nout, K):
    """Scales of rows that are not there may be anything, NaN's byte too; those of neighbouring rows differ by many powers of two."""
    r = np.random.default_rng(N)
    rows = r.integers(0, C + 1, N)
    (x8, xs), x = packed(r.standard_normal((N, C, K)) * np.exp2(r.integers(-40, 41, (N, C, 1))))
    dy = stored(r.standard_normal((N, C, Nout)), "bf16")
    for e in range(N):
        x8[e, rows[e]:] = 0x7f
        xs[e, :, rows[e]:] = 0xff
    dw = torch.full((N, Nout, K), 77.0, dtype=torch.bfloat16, device="cuda:0")
    ws = torch.empty(B.smile_fp8_weight_grad_workspace_bytes(N, C, K, "bf16"), dtype=torch.uint8, device="cuda:0")
    B.smile_fp8_weight_grad(dev(dy, "bf16"), x8, xs, dw, ws, rows=dev(rows.astype(np.int32)))
    got = host(dw)
    for e in range(N):
        n = rows[e]
        want, size = dy[e, :n].T @ x[e, :n], np.abs(dy[e, :n]).T @ np.abs(x[e, :n])
        near(got[e], want, half(want, "bf16") + (n + 1) * 2.0 ** -23 * size, ("dw", e))


@pytest.mark.parametrize("N", (1, 260))
def test_weight_grad_in_half_precision_at_the_ends_of_its_range(N):
    """Operands beyond 65504 count as that, products beyond it are infinite, NaN stays NaN, subnormals are kept."""
    C, Nout, K = 5, 64, 128
    x = np.zeros((N, C, K))
    x[:, 0, :8], x[:, 1, :8], x[:, 2, 8:16], x[:, 3, 16:24] = 65536.0, -65536.0, 2.0 ** -20, 3.0
    (x8, xs), _ = packed(x)
    x8[:, 4, 30] = 0x7f
    dy = np.zeros((N, C, Nout))
    dy[:, 0, 0], dy[:, 1, 1], dy[:, 0, 2], dy[:, 2, 3], dy[:, 3, 4], dy[:, 4, 5] = 0.5, 1.0, 4.0, 2.0, 1.0, 1.0
    dw = torch.zeros((N, Nout, K), dtype=torch.float16, device="cuda:0")
    ws = torch.empty(B.smile_fp8_weight_grad_workspace_bytes(N, C, K, "f16"), dtype=torch.uint8, device="cuda:0")
    B.smile_fp8_weight_grad(dev(dy, "f16"), x8, xs, dw, ws)
    want = np.zeros((N, Nout, K))
    want[:, 0, :8], want[:, 1, :8], want[:, 2, :8], want[:, 3, 8:16], want[:, 4, 16:24] = 32752.0, -65504.0, np.inf, 2.0 ** -19, 3.0
    want[:, :, 30] = np.nan
    assert np.array_equal(host(dw), want, equal_nan=True)


# ------------------------------------------------------------------ streams and graphs

def test_other_stream_and_graph_replays():
    """norm -> product with 8-bit rows -> product, and the norm's gradient, on a stream of their own and captured: every replay gives what the
    eager calls give on the same inputs, with eager work in between."""
    T, d, F = 300, 320, 640
    g = torch.Generator(device="cuda:0").manual_seed(3)
    x, res = (torch.randn(T, d, device="cuda:0", generator=g).bfloat16() for _ in range(2))
    weight = torch.ones(d, device="cuda:0", dtype=torch.bfloat16)
    w1, w1s = B.alloc_fp8_weights(1, F, d)
    w2, w2s = B.alloc_fp8_weights(1, d, F)
    B.smile_fp8_pack_weights(0.05 * torch.randn(F, d, device="cuda:0", generator=g), w1, w1s)
    B.smile_fp8_pack_weights(0.05 * torch.randn(d, F, device="cuda:0", generator=g), w2, w2s)
    y8, h8 = B.alloc_fp8_rows(1, T, d), B.alloc_fp8_rows(1, T, F)
    total, out, ds = torch.zeros_like(x), torch.zeros_like(x), torch.zeros_like(x)
    rstd, dw = torch.zeros(T, device="cuda:0"), torch.zeros(d, device="cuda:0")
    dw2, wg = torch.zeros(d, F, device="cuda:0", dtype=torch.bfloat16), torch.empty(B.smile_fp8_weight_grad_workspace_bytes(1, T, F, "bf16"), dtype=torch.uint8, device="cuda:0")
    ws = torch.empty(B.smile_rms_norm_backward_workspace_bytes(T, d), dtype=torch.uint8, device="cuda:0")
    up = B.make_fp8_gemm_args(*y8, w1, w1s, d, F, act="gelu", y8=h8[0], y_scale=h8[1])
    down = B.make_fp8_gemm_args(*h8, w2, w2s, F, d, y=out)

    def step():
        B.smile_rms_norm(x, res, weight, EPS, sum=total, y8=y8[0], y8_scale=y8[1], rstd=rstd)
        B.smile_fp8_gemm(up)
        B.smile_fp8_gemm(down)
        B.smile_rms_norm_backward(out, total, weight, rstd, ds, dw, ws)
        B.smile_fp8_weight_grad(out, *h8, dw2, wg)

    def result():
        torch.cuda.synchronize()
        return [t.clone() for t in (total, y8[0], h8[0], h8[1], out, ds, dw, dw2)]

    side = torch.cuda.Stream()
    step()
    first = result()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    assert all(torch.equal(a, b) for a, b in zip(result(), first))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        x.copy_(torch.randn(T, d, device="cuda:0", generator=g).bfloat16() * (k + 1))
        step()
        eager = result()
        for t in (total, out, ds, dw, dw2, y8[0], h8[0]):
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(result(), eager)), k


def test_graph_replays_of_a_relu_checkpoint_and_the_gradient_of_many_tiles():
    r = np.random.default_rng(3)
    N, C, K, Nout = 24, 70, 256, 512
    (x8, xs), _ = packed(r.standard_normal((N, C, K)))
    (w8, wsc), _ = packed(0.05 * r.standard_normal((N, Nout, K)), True)
    dy = dev(stored(r.standard_normal((N, C, Nout)), "bf16"), "bf16")
    rows = dev(r.integers(0, C + 1, N).astype(np.int32))
    h8, p8 = B.alloc_fp8_rows(N, C, Nout), B.alloc_fp8_rows(N, C, Nout)
    dw = torch.empty((N, Nout, K), dtype=torch.bfloat16, device="cuda:0")
    ws = torch.empty(B.smile_fp8_weight_grad_workspace_bytes(N, C, K, "bf16"), dtype=torch.uint8, device="cuda:0")
    args = B.make_fp8_gemm_args(x8, xs, w8, wsc, K, Nout, rows=rows, act="relu", y8=h8[0], y_scale=h8[1], pre8=p8[0], pre_scale=p8[1], dtype="bf16")
    results = (*h8, *p8, dw)

    def step():
        B.smile_fp8_gemm(args)
        B.smile_fp8_weight_grad(dy, x8, xs, dw, ws, rows=rows)

    def clear():
        for t in results:
            t.fill_(1)

    clear()
    step()
    want = [t.clone() for t in results]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        clear()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(t, w) for t, w in zip(results, want))
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(t, w) for t, w in zip(results, want))
