"""What is not finite in the products of 8-bit operands: NaN stays in its row and column through the activations and their derivatives, and a product
that overflows keeps to its element.  Both kernels, by the library's own rule.  Tolerances as in test_gpu_fp8.py."""
import numpy as np
import pytest
import torch

import fp8_reference as R
from paper_2212_05191_amd import binding as B
from test_gpu_fp8 import half, host, near, packed

pytestmark = pytest.mark.gpu

FEW, RING = (7, 512, 256), (300, 640, 2048)      # rows, contraction, columns
KINDS = pytest.mark.parametrize("C,K,Nout", (FEW, RING))


def expected_kernel(C, K, Nout, rows8, act):
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    assert R.kernel_of(cus, 1, C, K, Nout, rows8, act) == ((1 if rows8 else 0) if C == FEW[0] else 2)


def product(x8, xs, w8, wsc, K, Nout, act, y=None, y8=False, pre8=False, grad8=(None, None)):
    """y (of the storage type `y`), (y8, its scales), (pre8, its scales) of one group"""
    C = x8.shape[1]
    expected_kernel(C, K, Nout, bool(y8 or pre8 or grad8[0] is not None), act)
    out = torch.zeros((1, C, Nout), dtype=y, device="cuda:0") if y else None
    o8, p8 = (B.alloc_fp8_rows(1, C, Nout) if want else (None, None) for want in (y8, pre8))
    B.smile_fp8_gemm(B.make_fp8_gemm_args(x8, xs, w8, wsc, K, Nout, act=act, y=out, y8=o8[0], y_scale=o8[1], pre8=p8[0], pre_scale=p8[1],
                                          grad8=grad8[0], grad_scale=grad8[1], dtype="bf16"))
    return out, o8, p8


def check_values(got, want, tol, lost, what):
    """`lost`: where the values are NaN; the others as given"""
    assert np.array_equal(np.isnan(got), lost), (what, int(np.isnan(got).sum()), int(lost.sum()))
    near(np.where(lost, 0.0, got), np.where(lost, 0.0, want), tol, what)


def check_rows8(rows8, want, slack, lost, what):
    codes, scales = host(rows8[0]), host(rows8[1])
    assert np.array_equal((codes[0] & 0x7f) == 0x7f, lost), (what, int(((codes[0] & 0x7f) == 0x7f).sum()), int(lost.sum()))
    got = R.unpack_rows(codes, scales, want.shape[1])[0]
    fine = np.where(lost, 0.0, want)
    near(np.where(lost, 0.0, got), fine, R.row_step(fine[None], scales)[0] * (1 + 2.0 ** -10) + slack, what)


def operands(C, K, Nout, seed):
    r = np.random.default_rng(seed + C)
    return r, r.standard_normal((1, C, K)), 0.05 * r.standard_normal((1, Nout, K))


def nan_operands(C, K, Nout):
    r, x, w = operands(C, K, Nout, 1)
    (x8, xs), x = packed(x)
    (w8, wsc), w = packed(w, True)
    x8[0, 3, 100] = 0x7f
    w8[0, 140, 7] = 0xff
    lost = np.zeros((C, Nout), bool)
    lost[3], lost[:, 140] = True, True
    return r, (x8, xs, w8, wsc), x[0] @ w[0].T, max(K, 256) * 2.0 ** -23 * (np.abs(x[0]) @ np.abs(w[0]).T), lost


@KINDS
@pytest.mark.parametrize("act", ("relu", "gelu"))
def test_nan_passes_through_the_activation(C, K, Nout, act):
    _, ops, p, err, lost = nan_operands(C, K, Nout)
    v, verr = R.act(p, act), err * 1.13 + 4e-7 * (1 + np.abs(p))
    for y in (torch.float32, torch.bfloat16):
        out = product(*ops, K, Nout, act, y=y)[0]
        check_values(host(out)[0], v, verr + half(v, "f32" if y is torch.float32 else "bf16") * (1 + 2.0 ** -10), lost, y)
    out, y8, p8 = product(*ops, K, Nout, act, y=torch.float32, y8=True, pre8=True)
    check_values(host(out)[0], v, verr + half(v, "f32"), lost, "y beside 8 bits")
    check_rows8(y8, v, verr, lost, "y8")
    check_rows8(p8, p, err, lost, "pre8")


@KINDS
@pytest.mark.parametrize("act", ("relu", "gelu"))
def test_nan_of_a_kept_value_passes_through_the_derivative(C, K, Nout, act):
    r, x, w = operands(C, K, Nout, 2)
    (x8, xs), x = packed(x)
    (w8, wsc), w = packed(w, True)
    g8, g = packed(2.0 * r.standard_normal((1, C, Nout)))
    g8[0][0, 2, 50], g8[0][0, C - 1, Nout - 1] = 0x7f, 0xff
    lost = np.zeros((C, Nout), bool)
    lost[2, 50] = lost[C - 1, Nout - 1] = True
    p, err, slope = x[0] @ w[0].T, max(K, 256) * 2.0 ** -23 * (np.abs(x[0]) @ np.abs(w[0]).T), R.act_grad(g[0], act)
    v, verr = p * slope, err * np.abs(slope) + np.abs(p) * 4e-7 * (1 + np.abs(g[0]))
    out, y8, _ = product(x8, xs, w8, wsc, K, Nout, act, y=torch.float32, y8=True, grad8=g8)
    check_values(host(out)[0], v, verr + half(v, "f32"), lost, "y")
    check_rows8(y8, v, verr, lost, "y8")


@KINDS
@pytest.mark.parametrize("act", ("none", "relu", "gelu"))
def test_a_product_that_overflows_keeps_to_its_element(C, K, Nout, act):
    """Row 3: 2^127 times 4 in column 5, times -4 in column 200; everything else is ordinary."""
    _, x, w = operands(C, K, Nout, 3)
    x[0, 3, :128], x[0, :, 7], w[0, :, 7] = 0.0, 0.0, 0.0
    x[0, 3, 7], w[0, 5, 7], w[0, 200, 7] = 2.0 ** 127, 4.0, -4.0
    (x8, xs), x = packed(x)
    (w8, wsc), w = packed(w, True)
    x[0, :, 7] = 0.0
    p, err = x[0] @ w[0].T, max(K, 256) * 2.0 ** -23 * (np.abs(x[0]) @ np.abs(w[0]).T)
    v, verr = R.act(p, act), err * 1.13 + 4e-7 * (1 + np.abs(p))
    v[3, 5], v[3, 200] = np.inf, -np.inf if act == "none" else 0.0
    verr[3, 5] = verr[3, 200] = 0.0
    none = np.zeros((C, Nout), bool)
    for y in (torch.float32, torch.bfloat16):
        out = host(product(x8, xs, w8, wsc, K, Nout, act, y=y)[0])[0]
        near(out, v, verr + np.where(np.isinf(v), 0.0, half(np.where(np.isinf(v), 0.0, v), "f32" if y is torch.float32 else "bf16")) * (1 + 2.0 ** -10), y)
    out, y8, p8 = product(x8, xs, w8, wsc, K, Nout, act, y=torch.float32, y8=True, pre8=True)
    near(host(out)[0], v, verr + half(np.where(np.isinf(v), 0.0, v), "f32"), "y beside 8 bits")
    lost, kept = none.copy(), none.copy()
    lost[3, 5], lost[3, 200] = True, act == "none"
    kept[3, 5] = kept[3, 200] = True
    check_rows8(y8, v, verr, lost, "y8")
    check_rows8(p8, p, err, kept, "pre8")
