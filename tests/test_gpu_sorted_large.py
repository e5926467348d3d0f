"""The operators of a layer without dropped tokens on tensors of more than 2^32 elements: rows on both sides of 2^31 and 2^32 elements and the last ones, against their
definitions in 64 bits.  Tolerances as in test_gpu_sorted.py."""
import math

import pytest
import torch

import sorted_reference as R
from paper_2212_05191_amd import binding as B
from test_gpu_sorted import DEV, gen, ints, near, normal, scratch

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


@pytest.fixture(autouse=True)
def memory():
    B.load()
    yield
    torch.cuda.empty_cache()


def big(g, *shape, std=1.0, dtype=BF16):
    out = torch.empty(shape, dtype=dtype, device=DEV)
    for part in out.view(-1).split(1 << 28):
        part.normal_(0.0, std, generator=g)
    return out


def sample(rows, width):
    at = [r for border in (2 ** 31, 2 ** 32) for r in range(border // width - 4, border // width + 4)]
    return torch.tensor(sorted({r for r in [*range(4), *at, *range(rows - 70, rows)] if 0 <= r < rows}), device=DEV)


def test_products_of_long_tensors():
    g = gen(1)
    rows, K, F = (1 << 20) + 300, 4104, 72
    x, w = big(g, rows, K), normal(g, 1, F, K, std=K ** -0.5, dtype="bf16")
    at = sample(rows, K)
    y = torch.zeros(rows, F, dtype=BF16, device=DEV)
    B.smile_linear(B.make_linear_args(x, w, y))
    want, _, size = R.linear(x[at], w, None, "none", None, None)
    tol = size * (K + 2) * R.E32
    near(y[at], want, tol * (1 + R.HALF[BF16]) + R.half_step(want, BF16) * (1 + 1e-3), "y")
    # gradients of a loss on the sampled rows alone; the others' rows of dx are zeros
    dy = torch.zeros(rows, F, dtype=BF16, device=DEV)
    dy[at] = normal(g, len(at), F, dtype="bf16")
    dx, dw, db = torch.full_like(x, 3.0), torch.zeros_like(w), torch.zeros(1, F, dtype=BF16, device=DEV)
    args = B.make_linear_backward_args(dy, x, w, dx=dx, dw=dw, dbias=db)
    B.smile_linear_backward(args, scratch(B.smile_linear_backward_workspace_bytes(args)))
    want = R.linear_backward(dy[at], x[at], w, None, "none", None)
    for key, got, n in (("dx", dx[at], F), ("dw", dw, len(at)), ("dbias", db, len(at))):     # (adding zeros rounds nothing)
        value, size = want[key][:2]
        tol = size * (n + 2) * R.E32
        near(got, value, tol * (1 + R.HALF[BF16]) + R.half_step(value, BF16) * (1 + 1e-3), key)
    dx[at] = 0
    assert not any(bool(part.any()) for part in dx.split(1 << 17))


def test_wide_results_of_long_tensors():
    """y, residual and pre beyond 2^32 elements, in groups"""
    g = gen(2)
    rows, K, F = (1 << 20) + 300, 72, 4104
    first = [0, 1000, 1000, rows - 500, rows - 20]
    start = torch.tensor(first, dtype=torch.int32, device=DEV)
    x, w, b = big(g, rows, K), normal(g, 4, F, K, std=K ** -0.5, dtype="bf16"), normal(g, 4, F, dtype="bf16")
    y, pre = (torch.full((rows, F), 5.0, dtype=BF16, device=DEV) for _ in range(2))
    res = big(g, rows, F)
    B.smile_linear(B.make_linear_args(x, w, y, bias=b, act="gelu", residual=res, start=start, pre=pre))
    at = sample(rows, F)
    counts = torch.tensor([int((at < f).sum()) for f in first], dtype=torch.int32, device=DEV)
    want, p, size = R.linear(x[at], w, b, "gelu", res[at], counts)
    live = torch.arange(len(at), device=DEV) < counts[-1]
    chain = size * (K + 2) * R.E32
    tol = 1.13 * chain + 4e-7 * (1 + p.abs()) + 2 * R.E32 * want.abs()
    near(y[at][live], want[live], (tol * (1 + R.HALF[BF16]) + R.half_step(want, BF16) * (1 + 1e-3))[live], "y")
    near(pre[at][live], p[live], (chain * (1 + R.HALF[BF16]) + R.half_step(p, BF16) * (1 + 1e-3))[live], "pre")
    assert bool((y[at][~live] == 5).all()) and bool((pre[at][~live] == 5).all())


def test_rows_of_long_tensors():
    g = gen(3)
    T, k, d, N = (1 << 16) + 40, 8, 8200, 64
    idx = torch.randint(0, N, (T, k), generator=g, device=DEV, dtype=torch.int32)
    count, start, pos, source = ints(N), ints(N + 1), ints(T, k), ints(T * k)
    B.smile_sort_experts(idx, count, start, pos, source, scratch(B.smile_sort_experts_workspace_bytes(T, k, N)))
    assert torch.equal(source.long(), torch.argsort(idx.flatten(), stable=True))
    x, xs = big(g, T, d), torch.zeros(T * k, d, dtype=BF16, device=DEV)
    B.smile_sorted_dispatch(x, pos, xs)
    at = sample(T * k, d)
    assert torch.equal(xs[at], x[torch.div(source[at].long(), k, rounding_mode="floor")])
    weight, y, dys, dweight = torch.rand(T, k, generator=g, device=DEV), torch.zeros_like(x), torch.zeros_like(xs), torch.zeros(T, k, device=DEV)
    B.smile_sorted_combine(xs, pos, y, weight=weight)
    tokens = torch.unique(torch.div(source[at].long(), k, rounding_mode="floor"))
    rows = xs[pos[tokens].long()].double()
    scaled = rows * weight[tokens].double()[..., None]
    near(y[tokens], scaled.sum(1), scaled.abs().sum(1) * (k + 1) * R.E32 + R.half_step(scaled.sum(1), BF16) * (1 + 1e-3), "y")
    B.smile_sorted_combine_backward(x, xs, pos, weight, dys, dweight)
    dy = x[tokens].double()[:, None]
    near(dweight[tokens], (dy * rows).sum(2), (dy * rows).abs().sum(2) * d * R.E32, "dweight")
    want = dy * weight[tokens].double()[..., None]
    near(dys[pos[tokens].long()], want, R.half_step(want, BF16) * (1 + 1e-3) + want.abs() * R.E32, "dys")


def test_choice_among_long_logits():
    g = gen(4)
    T, N, k = (1 << 20) + 9, 4096, 3
    logits = big(g, T, N, std=3.0, dtype=torch.float32)
    idx, weight, p_sum = ints(T, k), torch.zeros(T, k, device=DEV), torch.zeros(N, device=DEV)
    B.smile_topk(logits, idx, weight, p_sum=p_sum, workspace=scratch(B.smile_topk_workspace_bytes(T, N)))
    at = sample(T, N)
    want_idx, want_w, p, v = R.topk(logits[at], None, k, False)
    span = (v.abs().amax(1, keepdim=True).double() * 2 + N + 16) * R.E32 * 2
    assert torch.equal(idx[at], want_idx)
    near(weight[at], want_w, want_w * span + 1e-37, "weight")
    total = torch.zeros(N, dtype=torch.float64, device=DEV)
    for part in logits.split(1 << 15):
        total += torch.softmax(part.double(), 1).sum(0)
    near(p_sum, total, total * (40 + N + 16) * 4 * R.E32 + total * T / 1024 * R.E32, "p_sum")   # a lane sums the tokens of one of 1024 workgroups at most
    dweight = normal(g, T, k)
    dlogits = torch.full_like(logits, math.nan)
    B.smile_topk_backward(logits, idx, dweight, dlogits)
    want, terms = R.topk_backward(p, want_idx, want_w, dweight[at], False, None, 0.0)
    size = torch.zeros_like(p).scatter_add(1, want_idx.long(), dweight[at].double().abs())
    near(dlogits[at], want, p * (size + (p * size).sum(1, keepdim=True)) * (3 * span + (N + 8) * R.E32) + terms * (N + 8) * 2.0 ** -53 + 1e-36, "dlogits")


def test_adamw_of_a_long_tensor():
    g = gen(5)
    n = 2 ** 32 - 24
    t = dict(param=big(g, n, std=0.1), grad=big(g, n, std=1e-2), m=torch.zeros(n, device=DEV), v=torch.zeros(n, device=DEV), weight_decay=0.1)
    small = dict(param=torch.ones(5, dtype=BF16, device=DEV), grad=torch.ones(5, dtype=BF16, device=DEV), m=torch.zeros(5, device=DEV), v=torch.zeros(5, device=DEV))
    parts = [slice(0, 5000), slice(2 ** 31 - 3000, 2 ** 31 + 3000), slice(n - 5000, n)]
    before = [t["param"][part].double() for part in parts]
    lr, step = torch.full((1,), 1e-2, device=DEV), ints(1)
    B.smile_adamw(B.AdamW([t, small], beta1=0.9, beta2=0.99), lr, step)
    for part, p0 in zip(parts, before):
        gr = t["grad"][part].double()
        want, m1, v1, update = R.adamw(p0, gr, torch.zeros_like(gr), torch.zeros_like(gr), 1, float(lr), 0.1, 0.9, 0.99, 1e-8)
        near(t["m"][part], m1, 0.1 * gr.abs() * 4 * R.E32 + 1e-44, "m")
        near(t["v"][part], v1, v1 * 6 * R.E32 + 1e-44, "v")
        # a new state: 16 roundings of the update, and four of m that carry to it
        tol = float(lr) * (update.abs() * 20 * R.E32 + 0.1 * p0.abs() * 4 * R.E32) + 4 * R.E32 * (p0.abs() + float(lr) * update.abs())
        near(t["param"][part], want, tol * (1 + R.HALF[BF16]) + R.half_step(want, BF16) * (1 + 1e-3), "param")
    assert bool((small["m"] > 0).all()) and int(step) == 1


def test_gradient_of_the_most_tokens():
    """As many tokens as a call takes, one workgroup for four of them: 2^32 threads"""
    g = gen(6)
    T, N = 2 ** 26 - 1, 513
    logits = torch.zeros(T, N, device=DEV)
    at = sample(T, N)
    logits[at] = normal(g, len(at), N, std=3.0)
    want_idx, want_w, p, v = R.topk(logits[at], None, 1, False)
    idx, dweight = ints(T, 1), torch.zeros(T, 1, device=DEV)
    idx[at], dweight[at] = want_idx, normal(g, len(at), 1)
    B.smile_topk_backward(logits, idx, dweight, logits)
    span = (v.abs().amax(1, keepdim=True).double() * 2 + N + 16) * R.E32 * 2
    want, terms = R.topk_backward(p, want_idx, want_w, dweight[at], False, None, 0.0)
    size = torch.zeros_like(p).scatter_add(1, want_idx.long(), dweight[at].double().abs())
    near(logits[at], want, p * (size + (p * size).sum(1, keepdim=True)) * (3 * span + (N + 8) * R.E32) + terms * (N + 8) * 2.0 ** -53 + 1e-36, "dlogits")
    logits[at] = 0
    assert not any(bool(part.any()) for part in logits.split(1 << 20))        # (tokens whose weights have no gradient)
