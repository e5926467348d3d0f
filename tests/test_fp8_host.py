"""Host side of the 8-bit operators: size helpers, argument checks (which run before anything touches a GPU), the binding's
checks of shapes and types, and the reference itself against differences.  No kernel is launched here."""
import ctypes as C
import types

import numpy as np
import pytest
import torch

import fp8_reference as R
from paper_2212_05191_amd import binding as B

P = 4096          # a pointer that is aligned and never followed
ODD = P + 4       # one that is not


def test_size_helpers():
    for K in (1, 8, 127, 128, 129, 960, 1600, 32768):
        assert B.smile_fp8_pitch(K) == R.up(K, 128)
        assert B.smile_fp8_scale_pitch(K) == R.up(K, 16)
    for bad in (0, -1, 2 ** 31 - 1):
        assert B.smile_fp8_pitch(bad) == -1 and B.smile_fp8_scale_pitch(bad) == -1
    assert B.smile_rms_norm_backward_workspace_bytes(3, 64) == 3 * 64 * 4
    assert B.smile_rms_norm_backward_workspace_bytes(1 << 20, 1024) <= 1024 * 1024 * 4
    assert B.smile_fp8_weight_grad_workspace_bytes(3, 5, 64, "bf16") == R.up(3 * 5 * 64 * 2, 256)
    for args in ((0, 64), (3, 12), (3, 16392), ((1 << 30) + 1, 8)):
        with pytest.raises(B.SmileError) as e:
            B.smile_rms_norm_backward_workspace_bytes(*args)
        assert e.value.status == B.BAD_SHAPE


def test_norm_refusals():
    lib = B.load()

    def norm(T=4, d=64, dtype=1, x=P, residual=P, weight=P, eps=1e-5, total=P, y=P, y8=P, y8_scale=P, rstd=P):
        return lib.smile_rms_norm(T, d, dtype, x, residual, weight, eps, total, y, y8, y8_scale, rstd, None)

    for name in ("x", "weight"):
        assert norm(**{name: None}) == B.INVALID_ARG
    for name in ("x", "residual", "weight", "total", "y", "y8", "y8_scale", "rstd"):
        assert norm(**{name: ODD}) == B.INVALID_ARG, name
    assert norm(y=None, y8=None, y8_scale=None) == B.INVALID_ARG      # nothing to compute
    assert norm(y8=None) == B.INVALID_ARG and norm(y8_scale=None) == B.INVALID_ARG
    assert norm(residual=None) == B.INVALID_ARG                       # the sum would be x
    for bad in (dict(T=0), dict(T=-1), dict(T=(1 << 30) + 1), dict(d=0), dict(d=12), dict(d=16392), dict(eps=0.0),
                dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf"))):
        assert norm(**bad) == B.BAD_SHAPE, bad
    assert norm(dtype=3) == B.UNSUPPORTED and norm(dtype=-1) == B.UNSUPPORTED

    def back(T=4, d=64, dtype=1, dy=P, dsum=P, s=P, weight=P, rstd=P, ds=P, dweight=P, workspace=P, nbytes=1 << 20):
        return lib.smile_rms_norm_backward(T, d, dtype, dy, dsum, s, weight, rstd, ds, dweight, workspace, nbytes, None)

    for name in ("dy", "s", "weight", "rstd", "ds", "dweight", "workspace"):
        assert back(**{name: None}) == B.INVALID_ARG, name
    for name in ("dy", "dsum", "s", "weight", "rstd", "ds", "dweight"):
        assert back(**{name: ODD}) == B.INVALID_ARG, name
    assert back(workspace=P + 16) == B.WORKSPACE and back(nbytes=4 * 64 * 4 - 1) == B.WORKSPACE
    assert back(T=0) == B.BAD_SHAPE and back(d=20) == B.BAD_SHAPE and back(dtype=7) == B.UNSUPPORTED


def test_pack_refusals():
    lib = B.load()
    for f in (lib.smile_fp8_pack_rows, lib.smile_fp8_unpack_rows):
        def call(N=2, cap=4, K=64, dtype=1, a=P, b=P, c=P, d=P):
            return f(N, cap, K, dtype, a, b, c, d, None)
        required = ("a", "c", "d") if f is lib.smile_fp8_pack_rows else ("a", "b", "d")
        for name in required:
            assert call(**{name: None}) == B.INVALID_ARG, name
        for name in "abcd":
            assert call(**{name: ODD}) == B.INVALID_ARG, name
        for bad in (dict(N=0), dict(N=4097), dict(cap=0), dict(K=0), dict(K=4), dict(K=32776), dict(N=4096, cap=1 << 19),
                    dict(N=1024, cap=1 << 20, K=1024)):
            assert call(**bad) == B.BAD_SHAPE, bad
        assert call(dtype=9) == B.UNSUPPORTED

    def weights(N=2, O=64, K=64, dtype=1, w=P, c=P, s=P, ct=P, st=P):
        return lib.smile_fp8_pack_weights(N, O, K, dtype, w, c, s, ct, st, None)
    for name in ("w", "c", "s", "ct", "st"):
        assert weights(**{name: None}) == B.INVALID_ARG, name
        assert weights(**{name: ODD}) == B.INVALID_ARG, name
    for bad in (dict(O=12), dict(K=12), dict(O=32776), dict(N=0)):
        assert weights(**bad) == B.BAD_SHAPE, bad
    assert weights(dtype=5) == B.UNSUPPORTED
    assert lib.smile_fp8_dispatch(None, P, P, P, P, P, P, P, None) == B.INVALID_ARG


def _gemm(**kw):
    a = B.Fp8GemmArgs(2, 4, 64, 64, 1, 2)
    base = dict(x8=P, x_scale=P, w8=P, w_scale=P, bias=None, rows=None, y=P, y8=None, y_scale=None, pre8=None, pre_scale=None,
                grad8=None, grad_scale=None)
    base.update(kw)
    for k, v in base.items():
        setattr(a, k, v)
    return B.load().smile_fp8_gemm(C.byref(a), None)


def test_gemm_refusals():
    assert B.load().smile_fp8_gemm(None, None) == B.INVALID_ARG
    for name in ("x8", "x_scale", "w8", "w_scale"):
        assert _gemm(**{name: None}) == B.INVALID_ARG, name
    for name in ("x8", "x_scale", "w8", "w_scale", "bias", "rows", "y", "y8", "y_scale", "pre8", "pre_scale", "grad8", "grad_scale"):
        assert _gemm(**{name: ODD}) == B.INVALID_ARG, name
    assert _gemm(y=None) == B.INVALID_ARG
    assert _gemm(y8=P) == B.INVALID_ARG and _gemm(y_scale=P) == B.INVALID_ARG
    assert _gemm(pre8=P) == B.INVALID_ARG and _gemm(grad_scale=P) == B.INVALID_ARG
    assert _gemm(y=None, pre8=P, pre_scale=P) == B.INVALID_ARG                              # only a checkpoint
    assert _gemm(act=0, grad8=P, grad_scale=P, bias=P) == B.INVALID_ARG
    assert _gemm(act=0, grad8=P, grad_scale=P, pre8=P, pre_scale=P) == B.INVALID_ARG
    assert _gemm(act=2, grad8=P, grad_scale=P) == B.UNSUPPORTED                             # the derivative of what?
    assert _gemm(act=3) == B.UNSUPPORTED and _gemm(act=-1) == B.UNSUPPORTED and _gemm(dtype=4) == B.UNSUPPORTED
    for bad in (dict(N=0), dict(N=4097), dict(C=0), dict(K=0), dict(K=100), dict(Nout=4), dict(Nout=32776),
                dict(N=4096, C=1 << 19)):
        assert _gemm(**bad) == B.BAD_SHAPE, bad


def test_weight_grad_refusals():
    lib = B.load()

    def call(N=2, cap=4, O=64, K=128, dtype=1, dy=P, x8=P, xs=P, rows=None, dw=P, ws=P, nbytes=1 << 20):
        return lib.smile_fp8_weight_grad(N, cap, O, K, dtype, dy, x8, xs, rows, dw, ws, nbytes, None)
    for name in ("dy", "x8", "xs", "dw", "ws"):
        assert call(**{name: None}) == B.INVALID_ARG, name
    for name in ("dy", "x8", "xs", "rows", "dw"):
        assert call(**{name: ODD}) == B.INVALID_ARG, name
    assert call(ws=P + 64) == B.WORKSPACE and call(nbytes=2 * 4 * 128 * 2 - 1) == B.WORKSPACE
    for bad in (dict(O=32), dict(K=96), dict(O=0), dict(cap=0)):
        assert call(**bad) == B.BAD_SHAPE, bad
    assert call(dtype=8) == B.UNSUPPORTED


def test_binding_checks_shapes_and_types():
    bf = torch.bfloat16
    x, w = torch.zeros(4, 64, dtype=bf), torch.zeros(64, dtype=bf)
    codes, scales = B.alloc_fp8_rows(1, 4, 64, "cpu")
    wc, wsc = B.alloc_fp8_weights(1, 96, 64, "cpu")
    with pytest.raises(ValueError):
        B.smile_rms_norm(x, None, torch.zeros(32, dtype=bf), 1e-5, y=x)
    with pytest.raises(TypeError):
        B.smile_rms_norm(x, None, w.float(), 1e-5, y=x)
    with pytest.raises(TypeError):
        B.smile_rms_norm(x, None, w, 1e-5, y=x, rstd=torch.zeros(4, dtype=bf))
    with pytest.raises(TypeError):
        B.smile_rms_norm(x.double(), None, w.double(), 1e-5, y=x)
    with pytest.raises(ValueError):
        B.smile_fp8_pack_rows(torch.zeros(5, 64, dtype=bf), codes, scales)
    with pytest.raises(TypeError):
        B.smile_fp8_pack_rows(x, codes, scales, rows=torch.zeros(1, dtype=torch.int64))
    with pytest.raises(ValueError):
        B.make_fp8_gemm_args(codes, scales, wc, wsc, 64, 128, y=torch.zeros(4, 128, dtype=bf))
    with pytest.raises(ValueError):
        B.make_fp8_gemm_args(codes, scales, wc, wsc, 64, 96, y=torch.zeros(4, 64, dtype=bf))
    with pytest.raises(TypeError):
        B.make_fp8_gemm_args(codes, scales, wc, wsc, 64, 96, y=torch.zeros(4, 96, dtype=bf), bias=torch.zeros(96))
    with pytest.raises(AssertionError):
        B.make_fp8_gemm_args(codes, scales, wc, wsc, 64, 96, y=torch.zeros(96, 4, dtype=bf).T)
    args = B.make_fp8_gemm_args(codes, scales, wc, wsc, 64, 96, y=torch.zeros(4, 96, dtype=bf))
    assert (args.N, args.C, args.K, args.Nout, args.dtype, args.act) == (1, 4, 64, 96, 1, 2)


@pytest.mark.parametrize("which", (0, 1, 2))
def test_dispatch_checks_its_indices(which):
    """Indices of another type or fewer of them than tokens: the kernel would read beyond them, and write where they point."""
    T = 6
    ctx = types.SimpleNamespace(desc=B.make_desc(T, 64, 128, 2, 2, 3), handle=None)
    for bad, error in ((torch.zeros(T, dtype=torch.int64), TypeError), (torch.zeros(T - 1, dtype=torch.int32), ValueError),
                       (torch.zeros(T, 1, dtype=torch.int32), ValueError)):
        index = [torch.zeros(T, dtype=torch.int32) for _ in range(3)]
        index[which] = bad
        with pytest.raises(error):
            B.smile_fp8_dispatch(ctx, *B.alloc_fp8_rows(1, T, 64, "cpu"), *index, *B.alloc_fp8_rows(4, 3, 64, "cpu"))


def test_codes_without_scales_are_refused():
    x, w = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(64, dtype=torch.bfloat16)
    (codes, scales), (wc, wsc) = B.alloc_fp8_rows(1, 4, 64, "cpu"), B.alloc_fp8_weights(1, 64, 64, "cpu")
    y = torch.zeros(4, 64, dtype=torch.bfloat16)
    for call in (lambda: B.smile_rms_norm(x, None, w, 1e-5, y8=codes), lambda: B.smile_fp8_pack_rows(x, codes, None),
                 lambda: B.smile_fp8_pack_rows(x, None, scales), lambda: B.smile_fp8_unpack_rows(codes, None, y),
                 lambda: B.smile_fp8_pack_weights(torch.zeros(64, 64), wc, wsc, wc),
                 lambda: B.make_fp8_gemm_args(codes, None, wc, wsc, 64, 64, y=y), lambda: B.make_fp8_gemm_args(codes, scales, wc, None, 64, 64, y=y),
                 lambda: B.make_fp8_gemm_args(codes, scales, wc, wsc, 64, 64, y8=codes), lambda: B.make_fp8_gemm_args(codes, scales, wc, wsc, 64, 64, y=y, pre8=codes),
                 lambda: B.make_fp8_gemm_args(codes, scales, wc, wsc, 64, 64, act="relu", y=y, grad8=codes)):
        with pytest.raises(ValueError):
            call()


# ------------------------------------------------------------------ the reference

def test_reference_codes_agree_with_torch():
    u = np.concatenate([np.linspace(-448, 448, 20001), R.CODES[np.isfinite(R.CODES)], np.float64(2) ** -np.arange(1, 14),
                        (R.CODES[:0x7e] + R.CODES[1:0x7f]) / 2]).astype(np.float32)      # ties too
    t = torch.from_numpy(u).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(R.encode(u), t)


def test_reference_scales():
    for k in (-140, -126, -20, 0, 3, 100):
        assert R.scale_bytes(448.0 * 2.0 ** k) == max(1, k + 127)
        assert R.scale_bytes(np.nextafter(448.0 * 2.0 ** k, np.inf)) == max(1, k + 128)
    assert R.scale_bytes(0.0) == 1


@pytest.mark.parametrize("dsum", (False, True))
def test_reference_norm_gradient_is_the_difference_quotient(dsum):
    r = np.random.default_rng(3)
    T, d, eps, h = 5, 24, 1e-3, 1e-6
    s, w, dy = r.standard_normal((T, d)), r.standard_normal(d), r.standard_normal((T, d))
    extra = r.standard_normal((T, d)) if dsum else None

    def loss(s, w):
        return np.sum(R.rms_norm(s, w, eps)[1] * dy) + (np.sum(extra * s) if dsum else 0.0)

    ds, dw = R.rms_norm_backward(dy, s, w, eps, extra)
    for _ in range(20):
        t, k = r.integers(T), r.integers(d)
        e = np.zeros_like(s)
        e[t, k] = h
        assert abs((loss(s + e, w) - loss(s - e, w)) / (2 * h) - ds[t, k]) < 1e-7
        e = np.zeros_like(w)
        e[k] = h
        assert abs((loss(s, w + e) - loss(s, w - e)) / (2 * h) - dw[k]) < 1e-7


@pytest.mark.parametrize("name", ("relu", "gelu"))
def test_reference_activation_gradient_is_the_difference_quotient(name):
    v = np.linspace(-9, 9, 1001) + 1e-3
    q = (R.act(v + 1e-5, name) - R.act(v - 1e-5, name)) / 2e-5
    assert np.max(np.abs(q - R.act_grad(v, name))) < 1e-8
