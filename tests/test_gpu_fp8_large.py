"""The 8-bit operators on tensors of more than 2^32 elements and bytes: rows on both sides of 2^31 and 2^32 and the last ones, against the definition in
64 bits.  Tolerances as in test_gpu_fp8_tiles.py."""
import numpy as np
import pytest
import torch

import fp8_reference as R
from paper_2212_05191_amd import binding as B
from test_gpu_fp8_tiles import CHAIN, EPS, act, check_rows8, generator, half, near, row_scales, row_values, slope, weight_values

pytestmark = pytest.mark.gpu

C, K = (1 << 21) + 200, 2112        # 2176 bytes of codes a row
BF16 = torch.bfloat16


@pytest.fixture(autouse=True)
def memory():
    yield
    torch.cuda.empty_cache()


def sample():
    at = [r for size in (2176, 4224) for border in (2 ** 31, 2 ** 32) for r in range(border // size - 20, border // size + 20)]
    return torch.tensor(sorted({r for r in [*range(40), *at, *range(C - 150, C)] if r < C}), device="cuda:0")


def normal(g, *shape, std=1.0):
    out = torch.empty(shape, dtype=BF16, device="cuda:0")
    for part in out.view(-1).split(1 << 28):
        part.normal_(0.0, std, generator=g)
    return out


def rows_of(pair, e, at):
    """8-bit rows `at` of a group, as a group of their own: codes, scales"""
    codes, scales = pair
    s = torch.zeros((scales.shape[1], R.up(len(at), 16)), dtype=torch.uint8, device="cuda:0")
    s[:, :len(at)] = scales[e][:, at]
    return codes[e][at], s


def test_pack_products_and_unpack():
    g, at = generator(1), sample()
    src = normal(g, C, K)
    x = B.alloc_fp8_rows(1, C, K)
    B.smile_fp8_pack_rows(src, *x)
    codes, scales = rows_of(x, 0, at)
    want_c, want_s = R.pack_rows(src[at].double().cpu().numpy()[None])
    assert np.array_equal(codes.cpu().numpy(), want_c[0]) and np.array_equal(scales.cpu().numpy()[:, :len(at)], want_s[0][:, :len(at)])
    w = B.alloc_fp8_weights(1, K, K)
    B.smile_fp8_pack_weights(normal(g, K, K, std=0.05), *w)
    xv, wv = row_values(codes, scales, K), weight_values(w[0][0], w[1][0], K)
    p, err = xv @ wv.T, K * 2.0 ** -23 * (xv.abs() @ wv.abs().T)
    y = src            # of the same size, and packed already
    h, pre = B.alloc_fp8_rows(1, C, K), B.alloc_fp8_rows(1, C, K)
    for name in ("relu", "gelu"):
        B.smile_fp8_gemm(B.make_fp8_gemm_args(*x, *w, K, K, act=name, y=y, y8=h[0], y_scale=h[1], pre8=pre[0], pre_scale=pre[1]))
        v, verr = act(p, name), err * 1.13 + 4e-7 * (1 + p.abs())
        near(y[at].double(), v, half(v, "bf16") * (1 + 2.0 ** -10) + verr, name)
        check_rows8(*rows_of(h, 0, at), v, verr, (name, "y8"))
        check_rows8(*rows_of(pre, 0, at), p, err, (name, "pre8"))
        if name == "relu":
            got, s = rows_of(pre, 0, at)
            wrong = ((got[:, :K] > 0) & (got[:, :K] < 0x80)) != (p > 2.0 ** -10 * row_scales(s, len(at), K))
            assert not bool(wrong.any())
    kept = row_values(*rows_of(pre, 0, at), K)
    B.smile_fp8_gemm(B.make_fp8_gemm_args(*x, *w, K, K, act="gelu", y=y, y8=h[0], y_scale=h[1], grad8=pre[0], grad_scale=pre[1]))
    v = p * slope(kept, "gelu")
    verr = err * slope(kept, "gelu").abs() + p.abs() * 4e-7 * (1 + kept.abs())
    near(y[at].double(), v, half(v, "bf16") * (1 + 2.0 ** -10) + verr, "slope")
    check_rows8(*rows_of(h, 0, at), v, verr, ("slope", "y8"))
    B.smile_fp8_unpack_rows(*x, y)
    assert torch.equal(y[at].double(), xv)


def test_norm_and_its_gradient():
    g, at = generator(2), sample()
    x, res, dy = normal(g, C, K), normal(g, C, K, std=3.0), normal(g, C, K)
    w = 1.0 + normal(g, K, std=0.1)
    total, y = torch.empty_like(x), torch.empty_like(x)
    rstd, dw = torch.zeros(C, device="cuda:0"), torch.zeros(K, device="cuda:0")
    y8 = B.alloc_fp8_rows(1, C, K)
    B.smile_rms_norm(x, res, w, EPS, sum=total, y=y, y8=y8[0], y8_scale=y8[1], rstd=rstd)
    both, s = x[at].double() + res[at].double(), total[at].double()
    near(s, both, half(both, "bf16") + both.abs() * 2.0 ** -24, "sum")
    want_rstd = torch.rsqrt(s.square().mean(1) + EPS)
    near(rstd[at].double(), want_rstd, want_rstd * CHAIN, "rstd")
    u, weight = s * want_rstd[:, None], w.double()
    near(y[at].double(), u * weight, half(u * weight, "bf16") + (u * weight).abs() * CHAIN, "y")
    check_rows8(*rows_of(y8, 0, at), u * weight, (u * weight).abs() * CHAIN, "y8")
    ws = torch.empty(B.smile_rms_norm_backward_workspace_bytes(C, K), dtype=torch.uint8, device="cuda:0")
    B.smile_rms_norm_backward(dy, total, w, rstd, y, dw, ws, dsum=x)
    gw = dy[at].double() * weight
    want = x[at].double() + want_rstd[:, None] * (gw - u * (gw * u).mean(1, keepdim=True))
    slack = want_rstd[:, None] * (gw.abs() + u.abs() * (gw * u).abs().mean(1, keepdim=True)) * 2 * CHAIN
    near(y[at].double(), want, half(want, "bf16") + slack + x[at].double().abs() * 2.0 ** -23, "ds")
    want, size = (torch.zeros(K, dtype=torch.float64, device="cuda:0") for _ in range(2))
    for k in range(0, C, 1 << 16):
        s = total[k:k + (1 << 16)].double()
        terms = dy[k:k + (1 << 16)].double() * s * torch.rsqrt(s.square().mean(1, keepdim=True) + EPS)
        want += terms.sum(0)
        size += terms.abs().sum(0)
    chain = (C // 768 + 1 + 16) * 2.0 ** -24         # additions in fp32
    near(dw.double(), want, (chain + 2 * CHAIN) * size, "dweight")


@pytest.mark.parametrize("dtype", ("bf16", "f16"))      # the direct kernel, the widened copy
def test_weight_gradient_of_the_last_groups(dtype):
    N, cap, Nout = 64, 40000, 64
    g = generator(3)
    st = B.torch_dtype(dtype)
    rows = [0] * N
    rows[0], rows[40], rows[49], rows[N - 1] = 33, 77, 5, 300
    src = torch.randn((N, 300, K), device="cuda:0", generator=g)
    x = B.alloc_fp8_rows(N, cap, K)
    dy = torch.zeros((N, cap, Nout), dtype=st, device="cuda:0")
    for e in range(N):
        if rows[e]:
            part = B.alloc_fp8_rows(1, 300, K)
            B.smile_fp8_pack_rows(src[e], *part)
            x[0][e, :300], x[1][e, :, :300] = part[0][0], part[1][0, :, :300]
            dy[e, :300] = torch.randn((300, Nout), device="cuda:0", generator=g).to(st)
    dw = torch.full((N, Nout, K), 77.0, dtype=st, device="cuda:0")
    ws = torch.empty(B.smile_fp8_weight_grad_workspace_bytes(N, cap, K, dtype), dtype=torch.uint8, device="cuda:0")
    B.smile_fp8_weight_grad(dy, *x, dw, ws, rows=torch.tensor(rows, dtype=torch.int32, device="cuda:0"))
    for e in range(N):
        xv, d = row_values(x[0][e, :rows[e]], x[1][e], K), dy[e, :rows[e]].double()
        want, size = d.T @ xv, d.abs().T @ xv.abs()
        near(dw[e].double(), want, half(want, dtype) + ((rows[e] + 1) * 2.0 ** -23 + (R.HALF["f16"] if dtype == "f16" else 0.0)) * size, e)


def test_dispatch_to_the_last_rows():
    N, cap, T = 64, 40000, 640
    r = np.random.default_rng(4)
    desc = B.make_desc(T, K, 128, 8, 8, cap)
    ctx = B.Ctx(desc)
    x8, xs = B.alloc_fp8_rows(1, T, K)
    x8.copy_(torch.from_numpy(r.integers(0, 256, tuple(x8.shape)).astype(np.uint8)))
    xs.copy_(torch.from_numpy(r.integers(0, 256, tuple(xs.shape)).astype(np.uint8)))
    xe8, xes = B.alloc_fp8_rows(N, cap, K)
    t = torch.arange(T, device="cuda:0", dtype=torch.int32)
    e, slot = t % N, cap - 1 - t // N * 3999
    B.smile_fp8_dispatch(ctx, x8, xs, (e // 8).int(), (e % 8).int(), slot.int(), xe8, xes)
    assert torch.equal(xe8[e.long(), slot.long()], x8[0]) and torch.equal(xes[e.long(), :, slot.long()], xs[0, :, :T].T)
    filled = torch.zeros((N, cap), dtype=torch.bool, device="cuda:0")
    filled[e.long(), slot.long()] = True
    for k in range(N):
        assert not bool(xe8[k][~filled[k]].any()) and not bool(xes[k][:, :cap][:, ~filled[k]].any())
    ctx.close()
