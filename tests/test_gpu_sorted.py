"""GPU parity of the operators of a layer without dropped tokens and of its optimizer with their definitions in 64 bits (sorted_reference.py).

Tolerances.  A rounding to a storage type is off by half a step (R.HALF relative, R.TINY among the subnormals).  fp32 sums of n terms, in any order: at most
n 2^-24 of the sum of magnitudes.  Softmax: the argument v - max is rounded once (2^-24 |v - max|, which the exponential makes relative), the
exponential and the division cost a few units of the last place and the sum of N terms N 2^-24: (|v - max| + N + 16) 2^-24 relative.  GELU and its derivative:
4e-7 (1 + |v|) in the 16-bit types, from the erfc approximation's 1.5e-7; in 32 bits 2^-21 (1 + |v|), eight roundings."""
import math

import pytest
import torch

import sorted_reference as R
from paper_2212_05191_amd import binding as B

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "these tests need the MI355X"
    B.load()


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def normal(g, *shape, std=1.0, dtype="f32"):
    return (torch.randn(*shape, generator=g, device=DEV) * std).to(TYPES[dtype])


def ints(*shape, value=0):
    return torch.full(shape, value, dtype=torch.int32, device=DEV)


def scratch(nbytes):
    return torch.empty(nbytes, dtype=torch.uint8, device=DEV) if nbytes else None


def near(got, want, tol, what):
    got, want = got.double(), want.double()
    tol = torch.as_tensor(tol, dtype=torch.float64, device=got.device).expand_as(got)
    same = (got == want) | (got.isnan() & want.isnan())
    off = torch.where(same, 0.0, (got - want).abs() - tol)
    off = torch.where(off.isnan(), math.inf, off)
    if off.numel() and float(off.max()) > 0:
        i = int(off.argmax())
        raise AssertionError((what, i, float(got.flatten()[i]), float(want.flatten()[i]), float(tol.flatten()[i])))


# ------------------------------------------------------------------ the choice of experts

def run_topk(logits, k, bias=None, normalize=False, p_sum=True):
    T, N = logits.shape
    idx, weight = ints(T, k, value=-7), torch.full((T, k), math.nan, device=DEV)
    total = torch.full((N,), math.nan, device=DEV) if p_sum else None
    B.smile_topk(logits, idx, weight, bias=bias, normalize=normalize, p_sum=total, workspace=scratch(B.smile_topk_workspace_bytes(T, N)) if p_sum else None)
    return idx, weight, total


SHAPES = [(1, 1, 1), (1, 64, 2), (3, 5, 5), (7, 16, 16), (33, 17, 3), (65, 33, 8), (130, 64, 8), (257, 100, 6), (1000, 128, 8), (300, 129, 64), (77, 256, 1),
          (50, 300, 2), (20, 513, 33), (9, 1025, 64), (5, 2049, 7), (3, 4096, 64), (4097, 8, 2),
          (35001, 31, 3), (17003, 63, 9), (9001, 128, 8), (8999, 127, 17), (4500, 256, 33), (2101, 511, 40)]


@pytest.mark.parametrize("normalize", (False, True))
@pytest.mark.parametrize("T,N,k", SHAPES)
def test_topk_and_its_gradient(T, N, k, normalize):
    g = gen(T * N + k)
    logits = normal(g, T, N, std=3.0)
    bias = None
    if N > 2 and T % 2:
        bias = normal(g, N)
        bias[torch.randperm(N, generator=g, device=DEV)[:N // 3]] = -math.inf          # with N = k some choices find nothing
    idx, weight, p_sum = run_topk(logits, k, bias, normalize)
    want_idx, want_w, p, v = R.topk(logits, bias, k, normalize)
    assert torch.equal(idx, want_idx)
    span = (v.masked_fill(v == -math.inf, 0.0).abs().amax(1, keepdim=True).double() * 2 + N + 16) * R.E32 * 2
    near(weight, want_w, want_w * span + 1e-37, "weight")
    near(p_sum, p.sum(0), (p * (span + (T + 2) * R.E32)).sum(0) + 1e-37, "p_sum")
    dweight, count = normal(g, T, k), torch.randint(0, 50, (N,), generator=g, device=DEV, dtype=torch.int32)
    for c, coef in ((None, 0.0), (count, 0.013)):
        dlogits = torch.full((T, N), math.nan, device=DEV)
        B.smile_topk_backward(logits, idx, dweight, dlogits, bias=bias, normalize=normalize, count=c, coef=coef)
        want, terms = R.topk_backward(p, want_idx, want_w, dweight, normalize, c, coef)
        at, none = want_idx.long().clamp_min(0), want_idx < 0
        size = torch.zeros_like(p).scatter_add(1, at, dweight.double().abs().masked_fill(none, 0.0))
        through = (coef * c.double()).expand_as(p) if c is not None else torch.zeros_like(p)
        if normalize:   # the chosen part is scaled by the weights
            chosen = torch.zeros_like(p).scatter_add(1, at, want_w)
            bound = p * (through + (p * through).sum(1, keepdim=True)) + chosen * (size + (chosen * size).sum(1, keepdim=True))
        else:
            bound = p * (size + through + (p * (size + through)).sum(1, keepdim=True))
        near(dlogits, want, bound * (3 * span + (N + 8) * R.E32) + terms * (N + 8) * 2.0 ** -53 + 1e-36, "dlogits")


def test_topk_ties_take_the_lowest_index():
    logits = torch.tensor([[1.0, 3.0, 3.0, 1.0, 3.0], [0.0, 0.0, 0.0, 0.0, 0.0], [-0.0, 0.0, -5.0, -5.0, 0.0]], device=DEV)
    idx, _, _ = run_topk(logits, 4)
    assert idx.tolist() == [[1, 2, 4, 0], [0, 1, 2, 3], [0, 1, 4, 2]]
    wide = torch.zeros(2, 4096, device=DEV)
    assert run_topk(wide, 64)[0].tolist() == [list(range(64))] * 2


def test_topk_of_masked_and_unusual_values():
    inf, nan = math.inf, math.nan
    logits = torch.tensor([[1.0, nan, inf, 2.0], [5.0, 1.0, 1.0, -inf], [-inf, 0.0, 0.0, -inf]], device=DEV)
    bias = torch.tensor([0.0, -inf, -inf, 0.0], device=DEV)       # what lies under a shut-off expert does not count
    idx, weight, p_sum = run_topk(logits, 3, bias, True)
    assert idx.tolist() == [[3, 0, -1], [0, -1, -1], [-1, -1, -1]]
    e = math.exp(-1.0)
    near(weight, torch.tensor([[1 / (1 + e), e / (1 + e), 0], [1, 0, 0], [0, 0, 0]], device=DEV), 1e-6, "weight")
    near(p_sum, torch.tensor([1 + e / (1 + e), 0, 0, 1 / (1 + e)], device=DEV), 1e-6, "p_sum")
    d = torch.full((3, 4), nan, device=DEV)
    B.smile_topk_backward(logits, idx, torch.ones(3, 3, device=DEV), d, bias=bias, normalize=False, count=ints(4, value=3), coef=1.0)
    assert bool(d.isfinite().all()) and bool((d[:, 1:3] == 0).all()) and bool((d[2] == 0).all())
    for value in (nan, inf):                                      # not masked: the token's weights and the sums are NaN, the indices in range
        logits = torch.tensor([[1.0, value, 0.5, 2.0], [1.0, 2.0, 3.0, 4.0]], device=DEV)
        for normalize in (False, True):
            idx, weight, p_sum = run_topk(logits, 2, None, normalize)
            assert bool(((idx >= 0) & (idx < 4)).all()) and bool(weight[0].isnan().all()) and bool(weight[1].isfinite().all()) and bool(p_sum.isnan().all())
    assert run_topk(torch.full((2, 4), nan, device=DEV), 2)[0].tolist() == [[-1, -1], [-1, -1]]


def test_topk_backward_against_differences():
    g = gen(5)
    logits, dweight, count = normal(g, 6, 9), normal(g, 6, 3), torch.randint(0, 9, (9,), generator=g, device=DEV, dtype=torch.int32)
    direction = normal(g, 6, 9)
    for normalize in (False, True):
        idx, _, _ = run_topk(logits, 3, None, normalize)
        d = torch.zeros(6, 9, device=DEV)
        B.smile_topk_backward(logits, idx, dweight, d, normalize=normalize, count=count, coef=0.1)

        def loss(x):
            p = torch.softmax(x, 1)
            w = p.gather(1, idx.long())
            if normalize:
                w = w / w.sum(1, keepdim=True)
            return float((dweight.double() * w).sum() + 0.1 * (count.double() * p.sum(0)).sum())
        h = 1e-5
        slope = (loss(logits.double() + h * direction.double()) - loss(logits.double() - h * direction.double())) / (2 * h)
        size = float((d.double().abs() * direction.double().abs()).sum())
        assert abs(slope - float((d.double() * direction.double()).sum())) <= 1e-5 * size + 1e-6   # h^2 and the roundings of the difference


@pytest.mark.parametrize("N", (5, 16, 300, 2051))
def test_topk_backward_in_place(N):
    g = gen(N)
    logits, dweight = normal(g, 70, N), normal(g, 70, 2)
    idx, _, _ = run_topk(logits, 2, None, True, p_sum=False)
    want = torch.zeros_like(logits)
    B.smile_topk_backward(logits, idx, dweight, want, normalize=True)
    B.smile_topk_backward(logits, idx, dweight, logits, normalize=True)
    assert torch.equal(logits, want)


@pytest.mark.parametrize("N,k", [(2, 1), (7, 1), (128, 1), (300, 1), (6, 6)])
def test_normalised_weights_without_freedom_send_nothing_back(N, k):
    """One choice has the weight 1 whatever the logits: exactly no gradient, and beside a small balance term that term's alone"""
    g = gen(N)
    logits, count = normal(g, 500, N, std=3.0), torch.randint(0, 50, (N,), generator=g, device=DEV, dtype=torch.int32)
    idx, weight, _ = run_topk(logits, k, None, True)
    if k == 1:
        assert bool((weight == 1).all())
    dweight = normal(g, 500, k) if k == 1 else torch.ones(500, k, device=DEV)
    d = torch.full((500, N), math.nan, device=DEV)
    B.smile_topk_backward(logits, idx, dweight, d, normalize=True)
    assert bool((d == 0).all()) if k == 1 else float(d.abs().max()) <= 4 * N * R.E32
    B.smile_topk_backward(logits, idx, dweight, d, normalize=True, count=count, coef=1e-6)
    if k == 1:
        p = torch.softmax(logits.double(), 1)
        u = 1e-6 * count.double()
        want, size = p * (u - (p * u).sum(1, keepdim=True)), p * (u + (p * u).sum(1, keepdim=True))
        near(d, want, size * (N + 60) * R.E32, "balance term alone")


def test_balance_term_of_nearly_even_counts():
    """Counts that differ in their last places: what counts is their differences, which fp32 keeps only if they are taken before the sums"""
    g = gen(8)
    logits = normal(g, 300, 5, std=2.0)
    count = torch.tensor([10000000, 10000003, 9999998, 10000001, 10000000], dtype=torch.int32, device=DEV)
    idx, _, _ = run_topk(logits, 2, None, False)
    d = torch.full((300, 5), math.nan, device=DEV)
    B.smile_topk_backward(logits, idx, torch.zeros(300, 2, device=DEV), d, count=count, coef=1e-3)
    p, u = torch.softmax(logits.double(), 1), 1e-3 * (count.double() - 1e7)
    near(d, p * (u - (p * u).sum(1, keepdim=True)), p * (u.abs() + (p * u.abs()).sum(1, keepdim=True)) * 64 * R.E32, "dlogits")


# ------------------------------------------------------------------ sort

@pytest.mark.parametrize("T,k,N", [(1, 1, 1), (3, 2, 5), (16, 2, 64), (1000, 3, 7), (2048, 2, 4), (2049, 2, 255), (700, 8, 257), (5003, 2, 15), (900, 5, 1024),
                                   (1500, 4, 1025), (300, 16, 4096), (40000, 4, 64), (1025, 1, 9), (6001, 4, 300), (6001, 4, 1030), (11003, 2, 4095), (12001, 4, 4096)])
def test_sort_experts(T, k, N):
    g = gen(T + N)
    idx = torch.randint(0, N, (T, k), generator=g, device=DEV, dtype=torch.int32)
    idx[torch.rand(T, k, generator=g, device=DEV) < 0.2] = -1
    if N > 3:
        idx[idx == 1] = 0                       # an expert without pairs, one with many
        idx[:2] = N + 3                         # no expert
    out = [ints(N, value=9), ints(N + 1, value=9), ints(T, k, value=9), ints(T * k, value=9)]
    B.smile_sort_experts(idx, *out, scratch(B.smile_sort_experts_workspace_bytes(T, k, N)))
    for got, want, name in zip(out, R.sort_experts(idx.cpu(), N), ("count", "start", "pos", "source")):
        assert torch.equal(got.cpu(), want), name


def test_sort_of_one_expert_and_of_none():
    for value, n in ((2, 3000 * 3), (-1, 0), (2 ** 31 - 1, 0), (-2 ** 31, 0)):
        idx = ints(3000, 3, value=value)
        out = [ints(5), ints(6), ints(3000, 3), ints(9000)]
        B.smile_sort_experts(idx, *out, scratch(B.smile_sort_experts_workspace_bytes(3000, 3, 5)))
        assert out[0].tolist() == [0, 0, n, 0, 0] and out[1].tolist() == [0, 0, 0, n, n, n]
        order = torch.arange(9000, dtype=torch.int32, device=DEV)
        assert torch.equal(out[2].view(-1), order if n else order * 0 - 1) and torch.equal(out[3], order if n else order * 0 - 1)


# ------------------------------------------------------------------ rows

def pairs(g, T, k, N, drop=0.2):
    """pos of a sort with dropped pairs"""
    idx = torch.argsort(torch.rand(T, N, generator=g, device=DEV), 1)[:, :k].to(torch.int32).contiguous()
    idx[torch.rand(T, k, generator=g, device=DEV) < drop] = -1
    out = [ints(N), ints(N + 1), ints(T, k), ints(T * k)]
    B.smile_sort_experts(idx, *out, scratch(B.smile_sort_experts_workspace_bytes(T, k, N)))
    return out


ROWS = [(1, 1, 8, 1), (5, 2, 8, 3), (16, 2, 1024, 64), (33, 3, 136, 5), (130, 8, 64, 16), (257, 4, 960, 15), (64, 5, 2048, 9), (7, 1, 16384, 2), (300, 33, 72, 40)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,k,d,N", ROWS)
def test_rows_there_and_back(T, k, d, N, dtype):
    g = gen(T + d)
    count, start, pos, source = pairs(g, T, k, N)
    st, R_ = TYPES[dtype], T * k + 5
    x, marker = normal(g, T, d, dtype=dtype), 7.0
    xs = torch.full((R_, d), marker, dtype=st, device=DEV)
    B.smile_sorted_dispatch(x, pos, xs)
    live = int(start[-1])
    src = source[:live].long()
    assert torch.equal(xs[:live], x[torch.div(src, k, rounding_mode="floor")]) and bool((xs[live:] == marker).all())

    ys, residual = normal(g, R_, d, dtype=dtype), normal(g, T, d, std=3.0, dtype=dtype)
    ys[live:] = math.nan                                                  # rows of no pair do not count
    weight = torch.rand(T, k, generator=g, device=DEV)
    some, at = pos >= 0, pos.long().clamp_min(0)
    rows = ys.double()[at.view(-1)].view(T, k, d).masked_fill(~some[..., None], 0.0)
    for w, res in ((weight, residual), (weight, None), (None, None), (None, residual)):
        y = torch.full((T, d), math.nan, dtype=st, device=DEV)
        B.smile_sorted_combine(ys, pos, y, weight=w, residual=res)
        scaled = rows if w is None else rows * w.double()[..., None]
        want, size = scaled.sum(1), scaled.abs().sum(1)
        if res is not None:
            want, size = want + res.double(), size + res.double().abs()
        near(y, want, size * (k + 1) * R.E32 + R.half_step(want, st) * (1 + 1e-3), "y")
    y = residual.clone()
    B.smile_sorted_combine(ys, pos, y, weight=weight, residual=y)         # in place
    want, size = (rows * weight.double()[..., None]).sum(1) + residual.double(), (rows * weight.double()[..., None]).abs().sum(1) + residual.double().abs()
    near(y, want, size * (k + 1) * R.E32 + R.half_step(want, st) * (1 + 1e-3), "y in place")

    dy = normal(g, T, d, dtype=dtype)
    dys, dweight = torch.full((R_, d), marker, dtype=st, device=DEV), torch.full((T, k), math.nan, device=DEV)
    B.smile_sorted_combine_backward(dy, ys, pos, weight, dys, dweight)
    want = (dy.double()[:, None] * rows).sum(2)
    near(dweight, want, (dy.double().abs()[:, None] * rows.abs()).sum(2) * d * R.E32, "dweight")
    want = dy.double()[torch.div(src, k, rounding_mode="floor")] * weight.double().view(-1)[src][:, None]
    near(dys[:live], want, R.half_step(want, st) * (1 + 1e-3) + want.abs() * R.E32, "dys")
    assert bool((dys[live:] == marker).all())
    again = torch.full((R_, d), marker, dtype=st, device=DEV)
    B.smile_sorted_combine_backward(dy, None, pos, weight, again, None)
    assert torch.equal(again, dys)


def test_row_numbers_outside_their_tensor_count_as_none():
    pos = torch.tensor([[0, 3], [4, -9], [2 ** 31 - 1, 1]], dtype=torch.int32, device=DEV)
    x = torch.arange(24, dtype=torch.float32, device=DEV).view(3, 8) + 1
    xs = torch.zeros(4, 8, device=DEV)
    B.smile_sorted_dispatch(x, pos, xs)
    assert torch.equal(xs, torch.stack([x[0], x[2], x[0] * 0, x[0]]))
    y = torch.zeros(3, 8, device=DEV)
    B.smile_sorted_combine(xs, pos, y, weight=torch.ones(3, 2, device=DEV))
    assert torch.equal(y, torch.stack([2 * x[0], 0 * x[0], x[2]]))
    dys, dweight = torch.zeros(4, 8, device=DEV), torch.ones(3, 2, device=DEV)
    B.smile_sorted_combine_backward(x, xs, pos, torch.ones(3, 2, device=DEV), dys, dweight)
    assert torch.equal(dys, xs) and bool((dweight[1] == 0).all()) and float(dweight[2, 0]) == 0


# ------------------------------------------------------------------ products

def gelu_tolerance(v, dtype, name):
    if name != "gelu":
        return torch.zeros_like(v)
    return (4e-7 if dtype != "f32" else 2.0 ** -21) * (1 + v.abs())


def run_linear(g, N, rows, K, F, dtype, name, bias, residual, start, pre=False, poison=False):
    st = TYPES[dtype]
    x, w = normal(g, rows, K, dtype=dtype), normal(g, N, F, K, std=K ** -0.5, dtype=dtype)
    b = normal(g, N, F, std=0.3, dtype=dtype) if bias else None
    res = normal(g, rows, F, std=2.0, dtype=dtype) if residual else None
    live = torch.zeros(rows, dtype=torch.bool, device=DEV)
    for lo, hi in R.groups(start, rows):
        live[lo:hi] = True
    if poison:
        x[~live] = math.nan
        if res is not None:
            res[~live] = math.nan
    marker = 5.0
    y = torch.full((rows, F), marker, dtype=st, device=DEV)
    kept = torch.full((rows, F), marker, dtype=st, device=DEV) if pre else None
    B.smile_linear(B.make_linear_args(x, w, y, bias=b, act=name, residual=res, start=start, pre=kept))
    want, p, size = R.linear(x, w, b, name, res, start)
    chain = size * (K + 2) * R.E32
    slope = 1.13 if name == "gelu" else 1.0                                # the largest of GELU's slopes
    tol = slope * chain + gelu_tolerance(p, dtype, name) + 2 * R.E32 * want.abs()
    near(y[live], want[live], (tol + R.half_step(want, st) * (1 + 1e-3) + R.HALF[st] * tol)[live], "y")
    assert bool((y[~live] == marker).all())
    if pre:
        near(kept[live], p[live], (chain + R.half_step(p, st) * (1 + 1e-3) + R.HALF[st] * chain)[live], "pre")
        assert bool((kept[~live] == marker).all())
    return x, w, b, res, y, kept, live


def run_linear_backward(g, x, w, kept, name, start, live, dtype, bias=True):
    st = TYPES[dtype]
    (N, F, K), rows = w.shape, x.shape[0]
    dy = normal(g, rows, F, dtype=dtype)
    dy[~live] = math.nan                                                   # rows of no group do not count
    marker = 5.0
    dx, dw, db = (torch.full(s, marker, dtype=st, device=DEV) for s in ((rows, K), (N, F, K), (N, F)))
    args = B.make_linear_backward_args(dy, x, w, dx=dx, dw=dw, dbias=db if bias else None, pre=kept, act=name, start=start)
    B.smile_linear_backward(args, scratch(B.smile_linear_backward_workspace_bytes(args)))
    want = R.linear_backward(dy, x, w, kept, name, start)
    slope = 0.0 if name != "gelu" else 4e-7 if dtype != "f32" else 2.0 ** -21            # of the derivative's error, over 1 + |pre|
    g_half = R.HALF[st] if name != "none" else 0.0                          # the gradient at the activation's argument, rounded
    for key, got, n in (("dx", dx, F), ("dw", dw, rows), ("dbias", db, rows)):
        if key == "dbias" and not bias:
            continue
        value, size, wide, ones = want[key]
        tol = size * ((n + 2) * R.E32 + (g_half if key != "dbias" else 0.0) + 4 * R.E32)
        tol = tol + wide * slope + (ones * R.TINY[st] if g_half and key != "dbias" else 0.0)
        tol = tol * (1 + R.HALF[st]) + R.half_step(value, st) * (1 + 1e-3)
        if key == "dx":
            near(got[live], value[live], tol[live], key)
            assert bool((got[~live] == marker).all())
        else:
            near(got, value, tol, key)
    return dy, dx, dw, db


def starts(g, N, rows, behind=0, empty=False, skew=False):
    if N == 1 and not behind:
        return None
    if skew:
        e = (torch.rand(rows - behind, generator=g, device=DEV) ** 4 * N).long()
    else:
        e = torch.randint(0, N, (rows - behind,), generator=g, device=DEV)
    if empty and N > 2:
        e[(e == 1) | (e == N - 1)] = 0
    count = torch.bincount(e, minlength=N)
    return torch.cat([torch.zeros(1, device=DEV), torch.cumsum(count, 0)]).to(torch.int32)


# N, rows, K, F, act, bias, residual, rows of no group, groups without rows
LINEAR = [(1, 1, 8, 8, "none", False, False, 0, False), (1, 1, 1024, 520, "gelu", True, False, 0, False), (1, 2, 72, 64, "relu", True, True, 0, False),
          (1, 16, 256, 136, "gelu", True, True, 0, False), (1, 17, 64, 264, "none", False, True, 0, False), (1, 33, 520, 72, "relu", True, False, 0, False),
          (1, 65, 128, 128, "gelu", False, False, 0, False), (1, 129, 200, 192, "none", True, True, 1, False), (1, 300, 960, 640, "gelu", True, True, 0, False),
          (1, 511, 64, 1032, "relu", True, True, 0, False), (1, 1030, 328, 264, "none", True, False, 7, False), (1, 2100, 512, 2048, "gelu", True, True, 0, False),
          (3, 5, 64, 64, "gelu", True, True, 1, True), (64, 16, 256, 128, "gelu", True, False, 0, False), (4, 200, 72, 200, "relu", True, True, 3, True),
          (5, 1000, 136, 520, "gelu", True, True, 37, True), (8, 3000, 192, 256, "none", False, True, 0, False), (70, 2000, 64, 72, "relu", True, False, 9, True),
          (300, 4000, 128, 64, "none", True, True, 5, True), (4096, 3000, 8, 16, "gelu", True, True, 11, False), (2, 900, 1288, 776, "gelu", True, False, 0, False),
          (6, 5000, 256, 768, "gelu", True, True, 100, True), (1, 70, 8192, 64, "none", True, False, 0, False), (1, 5000, 64, 64, "gelu", True, True, 0, False)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("case", LINEAR, ids=lambda c: "-".join(str(v) for v in c))
def test_linear_and_its_gradients(case, dtype):
    N, rows, K, F, name, bias, residual, behind, empty = case
    g = gen(sum(case[:4]))
    start = starts(g, N, rows, behind, empty)
    x, w, b, res, y, kept, live = run_linear(g, N, rows, K, F, dtype, name, bias, residual, start, pre=True, poison=True)
    run_linear_backward(g, x, w, kept if name != "none" else None, name, start, live, dtype, bias)


@pytest.mark.parametrize("dtype", TYPES)
def test_linear_of_a_skewed_router(dtype):
    g = gen(3)
    start = starts(g, 32, 3000, skew=True)
    x, w, b, res, y, kept, live = run_linear(g, 32, 3000, 128, 192, dtype, "gelu", True, True, start, pre=True)
    run_linear_backward(g, x, w, kept, "gelu", start, live, dtype)


@pytest.mark.parametrize("dtype", ("bf16", "f16"))
@pytest.mark.parametrize("name,N,rows,K,F,behind,skew", [("gelu", 1, 7900, 712, 2040, 0, False), ("relu", 1, 8190, 776, 2040, 5, False), ("gelu", 5, 7000, 2040, 1288, 100, False),
                                                         ("none", 9, 15500, 2056, 1544, 33, True)])
def test_linear_of_many_rows(name, N, rows, K, F, behind, skew, dtype):
    """Enough tiles of 256 x 256 for the chip: terms, rows and columns that end inside them, rows of no group, groups of a few rows and of most"""
    g = gen(rows)
    start = starts(g, N, rows, behind, skew=skew)
    x, w, b, res, y, kept, live = run_linear(g, N, rows, K, F, dtype, name, True, True, start, pre=True, poison=True)
    run_linear_backward(g, x, w, kept if name != "none" else None, name, start, live, dtype)


@pytest.mark.parametrize("first", ([0, 0, 0, 6000, 6000, 6001, 15000, 15000, 15500, 15500], [0, 15500, 15500, 15500, 15500, 15500, 15500, 15500, 15500, 15500],
                                   [40, 40, 40, 40, 40, 40, 40, 40, 40, 15500], [7, 7, 7, 7, 7, 7, 7, 7, 7, 7]))
def test_linear_of_many_rows_in_few_groups(first):
    """Tiles without a term among others, at the beginning and at the end of a workgroup's"""
    g = gen(first[3] + first[-1])
    start = torch.tensor(first, dtype=torch.int32, device=DEV)
    x, w, b, res, y, kept, live = run_linear(g, 9, 15500, 2056, 1544, "bf16", "gelu", True, False, start, pre=True, poison=True)
    run_linear_backward(g, x, w, kept, "gelu", start, live, "bf16")


@pytest.mark.parametrize("dtype", ("bf16", "f16"))
def test_weights_gradient_of_many_rows_in_parts(dtype):
    """16000 rows in two parts of 256 x 256 tiles, their sums joined"""
    g = gen(17)
    rows, K, F = 16000, 2800, 2800
    start = torch.tensor([0, rows - 77], dtype=torch.int32, device=DEV)
    dy, x, dw = normal(g, rows, F, dtype=dtype), normal(g, rows, K, dtype=dtype), torch.full((1, F, K), math.nan, dtype=TYPES[dtype], device=DEV)
    dy[rows - 77:], x[rows - 77:] = math.nan, math.nan
    args = B.make_linear_backward_args(dy, x, dw, dw=dw, start=start)
    nbytes = B.smile_linear_backward_workspace_bytes(args)
    assert nbytes >= 2 * F * K * 4
    B.smile_linear_backward(args, scratch(nbytes).fill_(0xFF))
    a, b = dy[:rows - 77].double(), x[:rows - 77].double()
    want = a.T.contiguous() @ b
    tol = a.abs().T.contiguous() @ b.abs() * (rows + 2) * R.E32
    near(dw[0], want, tol * (1 + R.HALF[TYPES[dtype]]) + R.half_step(want, TYPES[dtype]) * (1 + 1e-3), "dw")


@pytest.mark.parametrize("dtype", TYPES)
def test_linear_without_any_row(dtype):
    """First rows that are all the same: nothing is written but zeros of the weights' gradients; and one group that holds everything."""
    g = gen(4)
    for first in ([0, 0, 0, 0], [7, 7, 7, 7], [200, 200, 200, 200], [0, 0, 200, 200]):
        start = torch.tensor(first, dtype=torch.int32, device=DEV)
        x, w, b, res, y, kept, live = run_linear(g, 3, 200, 64, 72, dtype, "gelu", True, True, start, pre=True, poison=True)
        run_linear_backward(g, x, w, kept, "gelu", start, live, dtype)


def test_linear_with_first_rows_out_of_order_stays_in_its_tensors():
    for first in ([-5, 300, 40, 2 ** 31 - 1], [2 ** 31 - 1, -2 ** 31, 5, 5], [100, 50, 25, 0]):
        start = torch.tensor(first, dtype=torch.int32, device=DEV)
        for dtype in TYPES.values():
            guard = torch.full((3, 128, 64), 3.0, dtype=dtype, device=DEV)
            x, w, y, dw = torch.ones(128, 64, dtype=dtype, device=DEV), torch.ones(3, 64, 64, dtype=dtype, device=DEV), guard[1], torch.zeros(3, 64, 64, dtype=dtype, device=DEV)
            B.smile_linear(B.make_linear_args(x, w, y, start=start))
            args = B.make_linear_backward_args(y, x, w, dx=x.clone(), dw=dw, dbias=torch.zeros(3, 64, dtype=dtype, device=DEV), start=start)
            B.smile_linear_backward(args, scratch(B.smile_linear_backward_workspace_bytes(args)))
            assert bool((guard[0] == 3).all()) and bool((guard[2] == 3).all()) and bool(((y == 3) | (y == 64)).all()) and bool(dw.isfinite().all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,K,F", [(16, 256, 136), (300, 200, 264), (700, 512, 520), (7900, 712, 2040)])
def test_linear_keeps_nan_and_infinity_in_their_row_and_column(rows, K, F, dtype):
    g = gen(9)
    x, w = normal(g, rows, K, dtype=dtype), normal(g, 1, F, K, std=0.1, dtype=dtype)
    x[rows // 2, K - 1], x[0, 0], w[0, F - 1, 3] = math.nan, math.inf, math.nan
    bad = torch.zeros(rows, F, dtype=torch.bool, device=DEV)
    bad[rows // 2], bad[:, F - 1] = True, True
    for name in ("none", "relu", "gelu"):
        y, pre = torch.zeros(rows, F, dtype=TYPES[dtype], device=DEV), torch.zeros(rows, F, dtype=TYPES[dtype], device=DEV)
        B.smile_linear(B.make_linear_args(x, w, y, act=name, pre=pre))
        assert bool(y[bad].isnan().all()) and bool(pre[bad].isnan().all())
        fine = ~bad
        fine[0] = False
        assert bool(y[fine].isfinite().all()) and bool(pre[0, :F - 1].isinf().all())
        if name != "none":
            up, down = pre[0, :F - 1] > 0, pre[0, :F - 1] < 0
            assert bool((y[0, :F - 1][up] == math.inf).all()) and bool((y[0, :F - 1][down] == 0).all())
        dy = torch.ones(rows, F, dtype=TYPES[dtype], device=DEV)
        dx, dw, db = torch.zeros_like(x), torch.zeros_like(w), torch.zeros(1, F, dtype=TYPES[dtype], device=DEV)
        args = B.make_linear_backward_args(dy, x, w, dx=dx, dw=dw, dbias=db, pre=pre if name != "none" else None, act=name)
        B.smile_linear_backward(args, scratch(B.smile_linear_backward_workspace_bytes(args)))
        if name != "none":
            assert bool(db.isnan().all()) and bool(dx.isnan().any(1).all())        # column F - 1 of pre is NaN in every row
        assert bool(dw[0, :, K - 1].isnan().all()) and bool(dw[0, :F - 1, 5].isfinite().all()) == (name == "none")


@pytest.mark.parametrize("dtype", TYPES)
def test_linear_gradient_is_the_slope_of_its_values(dtype):
    """Along a direction of x and of w, by differences of the definition in 64 bits"""
    g = gen(11)
    start = torch.tensor([0, 20, 20, 50], dtype=torch.int32, device=DEV)
    x, w, b, res, y, kept, live = run_linear(g, 3, 53, 72, 40, dtype, "gelu", True, False, start, pre=True)
    dy, dx, dw, db = run_linear_backward(g, x, w, kept, "gelu", start, live, dtype)
    vx, vw, vb = normal(g, 53, 72), normal(g, 3, 40, 72, std=0.1), normal(g, 3, 40, std=0.1)

    def loss(h):
        out, _, _ = R.linear(x.double() + h * vx.double(), w.double() + h * vw.double(), b.double() + h * vb.double(), "gelu", None, start)
        return float((out * dy.double())[live].sum())
    slope = (loss(1e-5) - loss(-1e-5)) / 2e-5
    parts = [(dx.double() * vx.double())[live], dw.double() * vw.double(), db.double() * vb.double()]
    total, size = sum(float(p.sum()) for p in parts), sum(float(p.abs().sum()) for p in parts)
    # the kept argument and g are rounded once each, the results once: three half steps of the sum of magnitudes, which cancel beyond a few of it
    assert abs(slope - total) <= 4 * R.HALF[TYPES[dtype]] * size + 1e-5 * size


def test_linear_in_place_and_repeated():
    g = gen(12)
    for dtype in TYPES:
        x, w, res = normal(g, 700, 264, dtype=dtype), normal(g, 1, 520, 264, std=0.06, dtype=dtype), normal(g, 700, 520, dtype=dtype)
        y = torch.zeros_like(res)
        B.smile_linear(B.make_linear_args(x, w, y, act="gelu", residual=res))
        inplace = res.clone()
        B.smile_linear(B.make_linear_args(x, w[0], inplace, act="gelu", residual=inplace))
        assert torch.equal(y, inplace)
        args = None
        seen = []
        for _ in range(2):
            dw, db = torch.zeros_like(w), torch.zeros(520, dtype=TYPES[dtype], device=DEV)
            args = B.make_linear_backward_args(res, x, w, dw=dw, dbias=db)
            B.smile_linear_backward(args, scratch(B.smile_linear_backward_workspace_bytes(args)).fill_(0xFF))
            seen.append((dw, db))
        assert torch.equal(seen[0][0], seen[1][0]) and torch.equal(seen[0][1], seen[1][1])


# ------------------------------------------------------------------ AdamW

BETAS = dict(beta1=0.9, beta2=0.99, eps=1e-8)


def adam_tensors(g, sizes, dtype, grad, bits, master, new):
    out = []
    for i, n in enumerate(sizes):
        blocks = -(-n // 128)
        p = normal(g, n, std=0.1)
        t = dict(param=p.to(TYPES[dtype]), grad=normal(g, n, std=1e-2).to(TYPES[grad]), master=p if master else None, weight_decay=0.1 * (i % 2))
        if bits == 32:
            t.update(m=normal(g, n, std=0 if new else 1e-2), v=normal(g, n, std=0 if new else 1e-2) ** 2)
        else:
            t.update({k: torch.zeros(blocks * s, dtype=torch.uint8, device=DEV) for k, s in (("m", 128), ("v", 128), ("m_scale", 1), ("v_scale", 1))})
            if not new:
                code = torch.randint(0, 256, (n,), generator=g, device=DEV)
                t["m"][:n] = torch.where(code & 0x7F == 0x7F, 0, code).to(torch.uint8)
                t["v"][:n] = torch.randint(0, 249, (n,), generator=g, device=DEV).to(torch.uint8)
                t["m_scale"][:] = torch.randint(100, 112, (blocks,), generator=g, device=DEV).to(torch.uint8)
                t["v_scale"][:] = torch.randint(95, 115, (blocks,), generator=g, device=DEV).to(torch.uint8)
        out.append(t)
    return out


@pytest.mark.parametrize("dtype,grad,bits,master", [("f32", "f32", 32, False), ("f32", "f32", 8, False), ("bf16", "bf16", 32, True), ("bf16", "f32", 8, True),
                                                    ("bf16", "bf16", 8, False), ("f16", "f16", 8, True), ("f16", "f32", 32, False)])
@pytest.mark.parametrize("new", (True, False))
def test_adamw(dtype, grad, bits, master, new):
    g = gen(bits + new)
    tensors = adam_tensors(g, [1, 7, 128, 130, 2048, 2049, 5000, 40961], dtype, grad, bits, master, new)
    opt = B.AdamW(tensors, seed=77, **BETAS)
    lr, step = torch.full((1,), 1e-2, device=DEV), ints(1, value=0 if new else 41)
    st = TYPES[dtype]
    for _ in range(2):
        before = [{k: v.clone() if torch.is_tensor(v) else v for k, v in t.items()} for t in tensors]
        t_now = int(step) + 1
        B.smile_adamw(opt, lr, step)
        assert int(step) == t_now
        for i, (old, t) in enumerate(zip(before, tensors)):
            n = t["param"].numel()
            if bits == 32:
                m, v = old["m"].double(), old["v"].double()
            else:
                m, v = R.m_value(old["m"], old["m_scale"])[:n], R.v_value(old["v"], old["v_scale"])[:n]
            p0, gr = (old["master"] if master else old["param"]).double(), old["grad"].double()
            want, m1, v1, update = R.adamw(p0, gr, m, v, t_now, float(lr), old["weight_decay"], 0.9, 0.99, 1e-8)
            # two products and their sum of each moment, the scaled quotient: a dozen roundings of the update, two of the parameter
            m_tol, v_tol = (0.9 * m.abs() + 0.1 * gr.abs()) * 4 * R.E32, v1 * 6 * R.E32
            u_tol = update.abs() * 16 * R.E32 + m_tol / (1 - 0.9 ** t_now) / (torch.sqrt(v1 / (1 - 0.99 ** t_now)) + 1e-8)
            tol = float(lr) * (u_tol + old["weight_decay"] * p0.abs() * 4 * R.E32) + 4 * R.E32 * (p0.abs() + float(lr) * update.abs())
            if master:
                near(t["master"], want, tol, "master")
                assert torch.equal(t["param"], t["master"].to(st))
            else:
                near(t["param"], want, tol * (1 + R.HALF[st]) + R.half_step(want, st) * (1 + 1e-3), "param")
            if bits == 32:
                near(t["m"], m1, m_tol + 1e-44, "m")
                near(t["v"], v1, v_tol + 1e-44, "v")
                continue
            # rounding goes up with the value: the stored one lies between those of the value's ends
            r = R.random_bits(77, t_now, i, n, DEV)
            pad = lambda x: torch.nn.functional.pad(x, (0, -n % 128)).view(-1, 128)       # noqa: E731
            for key, value, err, byte, rnd, bits16 in (("m", m1, m_tol, R.m_byte, R.m_round, r & 0xFFFF), ("v", v1, v_tol, R.v_byte, R.v_round, r >> 16)):
                got_b = t[key + "_scale"].long()
                top = pad(value.abs()).amax(1)
                slack = pad(err).amax(1)
                low, high = byte((top - slack).clamp_min(0)), byte(top + slack)
                assert bool(((got_b.cpu() >= low) & (got_b.cpu() <= high)).all()), key
                b = got_b[:, None]
                got = (R.m_value if key == "m" else R.v_value)(t[key], t[key + "_scale"])
                ends = [rnd(pad(value + s * err) if key == "m" else pad((value + s * err).clamp_min(0)), pad(bits16), b).view(-1) for s in (-1, 1)]
                assert bool(((got >= torch.minimum(*ends)) & (got <= torch.maximum(*ends)))[:n].all()), key
                assert bool((t[key][n:] == 0).all())


def test_adamw_random_rounding_is_even_handed():
    """Values between two codes go up as often as their place says: of 2^17 the mean is off by at most 5 / sqrt(4 * 2^17) of a step."""
    n = 1 << 17
    for value in (1.0 + 1 / 32, 1.0 + 3 / 32, 1.99):
        t = dict(param=torch.zeros(n, device=DEV), grad=torch.full((n,), value, device=DEV), m=torch.zeros(n, dtype=torch.uint8, device=DEV),
                 v=torch.zeros(n, dtype=torch.uint8, device=DEV), m_scale=torch.zeros(n // 128, dtype=torch.uint8, device=DEV),
                 v_scale=torch.zeros(n // 128, dtype=torch.uint8, device=DEV))
        t["grad"][::128] = 448.0                                          # the block's largest: its power of two is 1
        opt = B.AdamW([t], beta1=0.0, beta2=0.0, seed=5)
        B.smile_adamw(opt, torch.zeros(1, device=DEV), ints(1))
        got = R.m_value(t["m"], t["m_scale"])
        rest = torch.arange(n, device=DEV) % 128 != 0
        assert abs(float(got[rest].mean()) - value) <= 0.125 * 5 / math.sqrt(4 * n) * 2
        assert set(got[rest].tolist()) <= {math.floor(value * 8) / 8, math.floor(value * 8) / 8 + 0.125}


def test_adamw_of_gradients_that_are_not_finite():
    n = 300
    for bits in (8, 32):
        t = adam_tensors(gen(1), [n], "bf16", "f32", bits, True, False)[0]
        t["grad"][5], t["grad"][140], t["grad"][141] = math.nan, math.inf, -math.inf
        keep = t["master"].clone()
        B.smile_adamw(B.AdamW([t], **BETAS), torch.full((1,), 1e-3, device=DEV), ints(1, value=3))
        hit = torch.zeros(n, dtype=torch.bool, device=DEV)
        hit[[5, 140, 141]] = True
        assert bool(t["master"][hit].isnan().all()) and bool(t["param"][hit].isnan().all()) and bool(t["master"][~hit].isfinite().all())
        assert bool((t["master"][~hit] != keep[~hit]).any())
        if bits == 8:
            m, v = R.m_value(t["m"], t["m_scale"])[:n], R.v_value(t["v"], t["v_scale"])[:n]
            assert bool(m[hit].isnan().all()) and bool(m[~hit].isfinite().all()) and bool(v.isfinite().all())


@pytest.mark.parametrize("dtype", ("f32", "bf16"))
def test_unpacked_states(dtype):
    n = 2048 * 3 + 128
    g = gen(2)
    t = adam_tensors(g, [n], "f32", "f32", 8, False, False)[0]
    m, v = (torch.zeros(n, dtype=TYPES[dtype], device=DEV) for _ in range(2))
    B.smile_adamw_unpack_states(t["m"], t["m_scale"], t["v"], t["v_scale"], m, v)
    for got, want in ((m, R.m_value(t["m"], t["m_scale"])), (v, R.v_value(t["v"], t["v_scale"]))):
        assert torch.equal(got, want.to(TYPES[dtype]))


# ------------------------------------------------------------------ streams and graphs

def test_operators_run_on_the_stream_that_is_current():
    """Work behind a long run of another stream is neither waited for nor disturbed; the stream's own order holds"""
    g = gen(31)
    x, w = normal(g, 2000, 512, dtype="bf16"), normal(g, 1, 1024, 512, std=0.05, dtype="bf16")
    logits = normal(g, 2000, 16)
    want, want_idx = torch.zeros(2000, 1024, dtype=torch.bfloat16, device=DEV), R.topk(logits, None, 2, True)[0]
    B.smile_linear(B.make_linear_args(x, w, want, act="relu"))
    late, late_logits, y = torch.zeros_like(x), torch.zeros_like(logits), torch.zeros_like(want)
    big = normal(g, 4096, 4096)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        for _ in range(20):
            big = (big @ big).clamp(-1, 1)
        late.copy_(x)
        late_logits.copy_(logits)
        B.smile_linear(B.make_linear_args(late, w, y, act="relu"))
        idx, weight, _ = run_topk(late_logits, 2, None, True, p_sum=False)
    stream.synchronize()
    assert torch.equal(y, want) and torch.equal(idx, want_idx)
    y.zero_()
    torch.cuda.synchronize()
    B.smile_linear(B.make_linear_args(x, w, y, act="relu"), stream=stream)
    stream.synchronize()
    assert torch.equal(y, want)


def test_tensors_of_the_host_are_refused():
    z = torch.zeros
    with pytest.raises(ValueError):
        B.smile_topk(z(4, 8), ints(4, 2), z(4, 2, device=DEV))
    with pytest.raises(ValueError):
        B.smile_sorted_dispatch(z(4, 64, device=DEV), ints(4, 2), z(8, 64))
    x, w, y = z(4, 64, device=DEV), z(1, 72, 64), z(4, 72, device=DEV)
    with pytest.raises(ValueError):
        B.smile_linear(B.make_linear_args(x, w, y))
    args = B.make_linear_backward_args(y, x, w.to(DEV), dbias=z(72, device=DEV))
    with pytest.raises(ValueError):
        B.smile_linear_backward(args, torch.zeros(B.smile_linear_backward_workspace_bytes(args), dtype=torch.uint8))
    opt = B.AdamW([dict(param=z(8, device=DEV), grad=z(8, device=DEV), m=z(8, device=DEV), v=z(8, device=DEV))])
    with pytest.raises(ValueError):
        B.smile_adamw(opt, z(1), ints(1))


def test_captured_step_follows_its_inputs():
    """A training step of the operators, captured once and replayed with other inputs, a new learning rate and the step's own count, beside eager work"""
    g = gen(21)
    T, N, k, d, F = 300, 8, 2, 128, 256
    logits, x = normal(g, T, N), normal(g, T, d, dtype="bf16")
    w, b = normal(g, N, F, d, std=0.1, dtype="bf16"), normal(g, N, F, std=0.1, dtype="bf16")
    dy = normal(g, T, F, dtype="bf16")

    def buffers():
        s = dict(idx=ints(T, k), weight=torch.zeros(T, k, device=DEV), p_sum=torch.zeros(N, device=DEV), count=ints(N), start=ints(N + 1), pos=ints(T, k), source=ints(T * k),
                 xs=torch.zeros(T * k, d, dtype=torch.bfloat16, device=DEV), ys=torch.zeros(T * k, F, dtype=torch.bfloat16, device=DEV), pre=torch.zeros(T * k, F, dtype=torch.bfloat16, device=DEV),
                 y=torch.zeros(T, F, dtype=torch.bfloat16, device=DEV), dys=torch.zeros(T * k, F, dtype=torch.bfloat16, device=DEV), dweight=torch.zeros(T, k, device=DEV),
                 dxs=torch.zeros(T * k, d, dtype=torch.bfloat16, device=DEV), dw=torch.zeros_like(w), db=torch.zeros_like(b), dx=torch.zeros_like(x), dlogits=torch.zeros(T, N, device=DEV),
                 w=w.clone(), m=torch.zeros(w.numel(), device=DEV), v=torch.zeros(w.numel(), device=DEV), lr=torch.full((1,), 1e-2, device=DEV), step=ints(1))
        s["up"] = B.make_linear_args(s["xs"], s["w"], s["ys"], bias=b, act="gelu", start=s["start"], pre=s["pre"])
        s["back"] = B.make_linear_backward_args(s["dys"], s["xs"], s["w"], dx=s["dxs"], dw=s["dw"], dbias=s["db"], pre=s["pre"], act="gelu", start=s["start"])
        s["ws"] = [scratch(B.smile_topk_workspace_bytes(T, N)), scratch(B.smile_sort_experts_workspace_bytes(T, k, N)), scratch(B.smile_linear_backward_workspace_bytes(s["back"]))]
        s["opt"] = B.AdamW([dict(param=s["w"].view(-1), grad=s["dw"].view(-1), m=s["m"], v=s["v"], weight_decay=0.1)])
        return s

    def run(s):
        B.smile_topk(logits, s["idx"], s["weight"], normalize=True, p_sum=s["p_sum"], workspace=s["ws"][0])
        B.smile_sort_experts(s["idx"], s["count"], s["start"], s["pos"], s["source"], s["ws"][1])
        B.smile_sorted_dispatch(x, s["pos"], s["xs"])
        B.smile_linear(s["up"])
        B.smile_sorted_combine(s["ys"], s["pos"], s["y"], weight=s["weight"])
        B.smile_sorted_combine_backward(dy, s["ys"], s["pos"], s["weight"], s["dys"], s["dweight"])
        B.smile_linear_backward(s["back"], s["ws"][2])
        B.smile_sorted_combine(s["dxs"], s["pos"], s["dx"])
        B.smile_topk_backward(logits, s["idx"], s["dweight"], s["dlogits"], normalize=True, count=s["count"], coef=0.01)
        B.smile_adamw(s["opt"], s["lr"], s["step"])

    eager, captured = buffers(), buffers()
    warm = buffers()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        run(warm)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            run(captured)
    for i in range(4):
        logits.copy_(normal(g, T, N))
        x.copy_(normal(g, T, d, dtype="bf16"))
        for s in (eager, captured):
            s["lr"].fill_(1e-2 / (i + 1))
        run(eager)
        graph.replay()
        torch.cuda.synchronize()
        for name in ("idx", "weight", "p_sum", "count", "start", "pos", "source", "xs", "y", "dweight", "dw", "db", "dx", "dlogits", "w", "m", "v", "step"):
            rows = int(eager["start"][-1]) if name == "xs" else None
            assert torch.equal(eager[name][:rows], captured[name][:rows]), (i, name)
    assert int(eager["step"]) == 4


# ------------------------------------------------------------------ at the ends of the ranges

@pytest.mark.parametrize("bits", (8, 32))
@pytest.mark.parametrize("dtype,value", [("f32", 1e21), ("f32", -1e30), ("bf16", 3e38)])
def test_adamw_of_a_gradient_whose_square_is_infinite(dtype, value, bits):
    """v is infinite, in the state too, and m is not: the element's update is 0 in this step and in those that follow, whatever the others' moments are"""
    n, hit = 300, 140
    t = adam_tensors(gen(1), [n], dtype, dtype, bits, False, False)[0]
    rest = torch.arange(n, device=DEV) != hit
    opt, step = B.AdamW([t], **BETAS), ints(1, value=1000)
    keep = t["param"].clone()
    for g in (value, 0.0, 1e-3, 0.0):
        t["grad"][hit] = g
        B.smile_adamw(opt, torch.full((1,), 1e-2, device=DEV), step)
        m, v = t["m"], t["v"]
        if bits == 8:
            m, v = torch.full((384,), math.nan, device=DEV), torch.full((384,), math.nan, device=DEV)
            B.smile_adamw_unpack_states(t["m"], t["m_scale"], t["v"], t["v_scale"], m, v)
        assert float(t["param"][hit]) == float(keep[hit]), g
        assert float(v[hit]) == math.inf and bool(m.isfinite().all()), g
        # the others' power of two goes by the finite ones alone: at most 448 2^(111 - 127) at the start, and squares of gradients below 1
        assert bool((v[:n][rest] <= 2.0 ** 4).all()) and bool(t["param"].isfinite().all()), g


@pytest.mark.parametrize("size", (1e-18, 1e-19, 3e-20))
def test_adamw_of_second_moments_below_the_normal_range(size):
    """v of 1e-38 to 1e-41, whose root is far above a small eps"""
    g = gen(3)
    n = 5000
    t = dict(param=normal(g, n), grad=normal(g, n).abs() * size + size, m=torch.zeros(n, device=DEV), v=torch.zeros(n, device=DEV))
    p0, eps = t["param"].double(), 2.0 ** -100
    lr = torch.full((1,), 1e-2, device=DEV)
    B.smile_adamw(B.AdamW([t], beta1=0.9, beta2=0.99, eps=eps), lr, ints(1, value=99))
    m, v = t["m"].double(), t["v"].double()
    near(m, 0.1 * t["grad"].double(), t["grad"].double() * R.E32, "m")
    near(v, 0.01 * t["grad"].double() ** 2, t["grad"].double() ** 2 * 0.01 * 6 * R.E32 + 4 * 2.0 ** -149, "v")
    # from the moments as they are stored: the quotient's dozen roundings, and half a step of 2^-149 of v / (1 - beta2^t), of which the root takes half
    c2 = 1 - 0.99 ** 100
    update = m / (1 - 0.9 ** 100) / (torch.sqrt(v / c2) + eps)
    tol = float(lr) * update * (16 * R.E32 + 2.0 ** -150 / (v / c2) / 2) + 4 * R.E32 * p0.abs()
    near(t["param"], p0 - float(lr) * update, tol, "param")


@pytest.mark.parametrize("eps", (2.0 ** -126, 1e-30))
def test_adamw_of_the_least_eps(eps):
    """An element whose gradient and moments are 0 stays where it is"""
    for bits in (8, 32):
        t = adam_tensors(gen(1), [300], "f32", "f32", bits, False, True)[0]
        t["grad"].zero_()
        keep = t["param"].clone()
        B.smile_adamw(B.AdamW([t], beta1=0.9, beta2=0.99, eps=eps), torch.full((1,), 1e-2, device=DEV), ints(1))
        assert torch.equal(t["param"], keep)


def test_a_workspace_that_is_not_needed_may_be_anything():
    logits = normal(gen(1), 3, 8)
    want = run_topk(logits, 2)
    assert B.smile_topk_workspace_bytes(3, 8) == 0
    out = [torch.zeros_like(t) for t in want]
    B.smile_topk(logits, out[0], out[1], p_sum=out[2], workspace=logits.view(-1)[4:])
    assert all(torch.equal(a, b) for a, b in zip(want, out))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("N,rows,K,F,parts", [(4, 4096, 256, 256, "dw"), (4, 2000, 256, 1024, "dx"), (3, 1500, 520, 1032, "dx"), (2, 3000, 136, 2056, "dw dx"),
                                              (7, 9000, 264, 128, "dw"), (4, 8000, 136, 4104, "dw dx")])
def test_gradients_of_several_groups_in_parts(N, rows, K, F, parts, dtype):
    """Sums of several groups cut into parts (the last case: tiles of 256 x 256): groups without rows, groups that end inside of a part, rows of no group in front and behind;
    and the same bits whatever the workspace held"""
    g = gen(rows + K)
    cuts = [int(rows * f) for f in torch.rand(N - 1, generator=torch.Generator().manual_seed(N)).tolist()]
    for first in ([0, *cuts, rows], [5, *cuts, rows - 37], [rows // 2] * N + [rows], [0] + [rows // 3 + 1] * (N - 1) + [rows - 1]):
        start = torch.tensor(sorted(first), dtype=torch.int32, device=DEV)
        x, w, b, res, y, kept, live = run_linear(g, N, rows, K, F, dtype, "gelu", True, False, start, pre=True, poison=True)
        dy, dx, dw, db = run_linear_backward(g, x, w, kept, "gelu", start, live, dtype)
        if dtype != "f32":
            alone = [B.make_linear_backward_args(dy, x, w, start=start, **one) for one in (dict(dw=dw), dict(dx=dx))]
            assert [B.smile_linear_backward_workspace_bytes(a) > 0 for a in alone] == ["dw" in parts, "dx" in parts]
        again = [t.clone() for t in (dx, dw, db)]
        args = B.make_linear_backward_args(dy, x, w, dx=again[0], dw=again[1], dbias=again[2], pre=kept, act="gelu", start=start)
        B.smile_linear_backward(args, scratch(B.smile_linear_backward_workspace_bytes(args)).fill_(0xFF))
        assert all(torch.equal(p, q) for p, q in zip((dx, dw, db), again))


@pytest.mark.parametrize("N", (2, 6, 40))
def test_balance_term_beside_weights_of_all_experts(N):
    """Every expert chosen and every weight's gradient the same: the weights, which add up to one, send nothing back, and the balance term is left"""
    g = gen(N)
    logits, count = normal(g, 500, N, std=3.0), torch.randint(0, 50, (N,), generator=g, device=DEV, dtype=torch.int32)
    idx, weight, _ = run_topk(logits, N, None, True)
    d = torch.full((500, N), math.nan, device=DEV)
    B.smile_topk_backward(logits, idx, torch.ones(500, N, device=DEV), d, normalize=True, count=count, coef=0.01)
    p, u = torch.softmax(logits.double(), 1), 0.01 * count.double()
    want, size = p * (u - (p * u).sum(1, keepdim=True)), p * (u + (p * u).sum(1, keepdim=True))
    # of the weights: w (1 - sum w), where the sum of N weights is off by its N roundings, N of the sum that they were divided by and 2 of each weight
    near(d, want, size * (2 * N + 120) * R.E32 + p * (2 * N + 6) * R.E32, "balance term")


@pytest.mark.parametrize("bits", (8, 32))
def test_adamw_without_a_memory_of_squares(bits):
    """beta2 0: v is the gradient's square alone, whatever it was before, infinity included"""
    t = adam_tensors(gen(1), [300], "f32", "f32", bits, False, True)[0]
    opt, step = B.AdamW([t], beta1=0.0, beta2=0.0, eps=1e-30), ints(1)
    for i, g in enumerate((1e25, 1e-3, -1e25, -2.0)):
        before = t["param"].double().clone()
        t["grad"][7] = g
        B.smile_adamw(opt, torch.full((1,), 1e-2, device=DEV), step)
        # the update is the gradient's sign (a dozen roundings), or 0 where the square is infinite
        want = before - 1e-2 * torch.sign(t["grad"].double()) * (t["grad"].double().abs() < 1e18)
        near(t["param"], want, 1e-2 * 16 * R.E32 + 4 * R.E32 * before.abs(), i)
