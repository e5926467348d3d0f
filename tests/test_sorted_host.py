"""Host side of the operators of a layer without dropped tokens and of its optimizer: argument checks (which run before anything touches a GPU), sizes, the
binding's checks, the plan of an optimizer step, and the reference itself against differences.  No kernel is launched here."""
import ctypes as C

import pytest
import torch

import sorted_reference as R
from paper_2212_05191_amd import binding as B

P = 4096          # a pointer that is aligned and never followed
ODD = P + 4       # one that is not
BIG = 1 << 40


def test_topk_refusals():
    lib = B.load()

    def call(T=4, N=8, k=2, logits=P, bias=P, idx=P, weight=P, p_sum=P, workspace=P, nbytes=BIG):
        return lib.smile_topk(T, N, k, 1, logits, bias, idx, weight, p_sum, workspace, nbytes, None)

    for name in ("logits", "idx", "weight"):
        assert call(**{name: None}) == B.INVALID_ARG, name
    for name in ("logits", "bias", "idx", "weight", "p_sum"):
        assert call(**{name: ODD}) == B.INVALID_ARG, name
    for bad in (dict(T=0), dict(N=0), dict(N=4097), dict(k=0), dict(k=9), dict(k=65, N=100), dict(T=1 << 25), dict(T=-1)):
        assert call(**bad) == B.BAD_SHAPE, bad
    assert call(T=100000, workspace=None) == B.INVALID_ARG and call(T=100000, workspace=P + 16) == B.WORKSPACE
    assert call(T=100000, nbytes=B.smile_topk_workspace_bytes(100000, 8) - 1) == B.WORKSPACE

    def back(T=4, N=8, k=2, logits=P, bias=P, idx=P, dweight=P, count=P, dlogits=P):
        return lib.smile_topk_backward(T, N, k, 0, logits, bias, idx, dweight, count, 1.0, dlogits, None)

    for name in ("logits", "idx", "dweight", "dlogits"):
        assert back(**{name: None}) == B.INVALID_ARG, name
    for name in ("logits", "bias", "idx", "dweight", "count", "dlogits"):
        assert back(**{name: ODD}) == B.INVALID_ARG, name
    assert back(T=0) == B.BAD_SHAPE and back(k=9) == B.BAD_SHAPE


def test_sort_refusals():
    lib = B.load()

    def call(T=4, k=2, N=8, idx=P, count=P, start=P, pos=P, source=P, workspace=P, nbytes=BIG):
        return lib.smile_sort_experts(T, k, N, idx, count, start, pos, source, workspace, nbytes, None)

    for name in ("idx", "count", "start", "pos", "source"):
        assert call(**{name: None}) == B.INVALID_ARG and call(**{name: ODD}) == B.INVALID_ARG, name
    for bad in (dict(T=0), dict(k=0), dict(k=65), dict(N=0), dict(N=4097), dict(T=1 << 25, k=2)):
        assert call(**bad) == B.BAD_SHAPE, bad
    assert call(T=100000, workspace=None) == B.INVALID_ARG and call(T=100000, workspace=P + 128) == B.WORKSPACE
    assert call(T=100000, nbytes=B.smile_sort_experts_workspace_bytes(100000, 2, 8) - 1) == B.WORKSPACE


def test_row_refusals():
    lib = B.load()

    def dispatch(T=4, k=2, d=64, R_=8, dtype=1, x=P, pos=P, xs=P):
        return lib.smile_sorted_dispatch(T, k, d, R_, dtype, x, pos, xs, None)

    def combine(T=4, k=2, d=64, R_=8, dtype=1, ys=P, pos=P, weight=P, residual=P, y=P):
        return lib.smile_sorted_combine(T, k, d, R_, dtype, ys, pos, weight, residual, y, None)

    def back(T=4, k=2, d=64, R_=8, dtype=1, dy=P, ys=P, pos=P, weight=P, dys=2 * P, dweight=P):
        return lib.smile_sorted_combine_backward(T, k, d, R_, dtype, dy, ys, pos, weight, dys, dweight, None)

    for f, needed, all_ in ((dispatch, ("x", "pos", "xs"), ("x", "pos", "xs")), (combine, ("ys", "pos", "y"), ("ys", "pos", "weight", "residual", "y")),
                            (back, ("dy", "pos", "weight", "dys"), ("dy", "ys", "pos", "weight", "dys", "dweight"))):
        for name in needed:
            assert f(**{name: None}) == B.INVALID_ARG, (f, name)
        for name in all_:
            assert f(**{name: ODD}) == B.INVALID_ARG, (f, name)
        for bad in (dict(T=0), dict(k=0), dict(k=65), dict(R_=0), dict(R_=(1 << 27) + 1), dict(d=0), dict(d=12), dict(d=16392), dict(T=1 << 26, k=1)):
            assert f(**bad) == B.BAD_SHAPE, (f, bad)
        assert f(dtype=3) == B.UNSUPPORTED and f(dtype=-1) == B.UNSUPPORTED
    assert back(ys=None) == B.INVALID_ARG and back(dweight=None) == B.INVALID_ARG and back(dys=P) == B.INVALID_ARG


def test_linear_refusals():
    lib = B.load()

    def args(cls, **kw):
        a = cls(*(kw.pop(n, v) for n, v in (("N", 2), ("rows", 16), ("K", 64), ("F", 64), ("dtype", 1), ("act", 1))))
        for i, (name, _) in enumerate(cls._fields_[6:]):
            setattr(a, name, kw.pop(name, P * (i + 1)))
        assert not kw
        return a

    call = lambda **kw: lib.smile_linear(C.byref(args(B.LinearArgs, **kw)), None)                                                # noqa: E731
    size = C.c_size_t(0)
    need = lambda **kw: lib.smile_linear_backward_workspace_bytes(C.byref(args(B.LinearBackwardArgs, **kw)), C.byref(size))      # noqa: E731
    back = lambda ws=P, n=BIG, **kw: lib.smile_linear_backward(C.byref(args(B.LinearBackwardArgs, **kw)), ws, n, None)           # noqa: E731
    assert lib.smile_linear(None, None) == B.INVALID_ARG and lib.smile_linear_backward(None, P, BIG, None) == B.INVALID_ARG
    for name in ("x", "w", "y", "start"):                  # start: N is 2
        assert call(**{name: None}) == B.INVALID_ARG, name
    for name in ("x", "w", "bias", "residual", "start", "y", "pre"):
        assert call(**{name: ODD}) == B.INVALID_ARG, name
    assert call(y=P) == B.INVALID_ARG and call(pre=6 * P) == B.INVALID_ARG and call(pre=4 * P) == B.INVALID_ARG     # y is x; pre is y, the residual
    for name in ("dy", "start"):
        assert back(**{name: None}) == B.INVALID_ARG and need(**{name: None}) == B.INVALID_ARG, name
    for name in ("dy", "x", "w", "pre", "start", "dx", "dw", "dbias"):
        assert back(**{name: ODD}) == B.INVALID_ARG and need(**{name: ODD}) == B.INVALID_ARG, name
    assert back(dx=None, dw=None, dbias=None) == B.INVALID_ARG                             # nothing to compute
    assert back(w=None) == B.INVALID_ARG and back(x=None) == B.INVALID_ARG and back(pre=None) == B.INVALID_ARG
    assert need(w=None, dx=None) == B.OK and need(x=None, dw=None) == B.OK and need(pre=None, act=2) == B.OK
    for f in (call, back, need):
        for bad in (dict(N=0), dict(N=4097), dict(rows=0), dict(rows=(1 << 27) + 1), dict(K=0), dict(K=12), dict(K=32776), dict(F=0), dict(F=20), dict(F=32776),
                    dict(rows=1 << 27, K=16384), dict(N=4096, K=32768, F=32768), dict(rows=1 << 24, N=4096), dict(rows=1 << 27, N=512)):
            assert f(**bad) == B.BAD_SHAPE, bad
        assert f(dtype=3) == B.UNSUPPORTED and f(dtype=-1) == B.UNSUPPORTED and f(act=3) == B.UNSUPPORTED and f(act=-1) == B.UNSUPPORTED
    assert need() == B.OK and size.value > 0
    assert back(ws=None) == B.INVALID_ARG and back(ws=P + 16) == B.WORKSPACE and back(n=size.value - 1) == B.WORKSPACE


def adam(n=300, bits=8, master=True, dtype=torch.bfloat16, grad=torch.float32):
    blocks = -(-n // 128)
    t = dict(param=torch.zeros(n, dtype=dtype), grad=torch.zeros(n, dtype=grad), master=torch.zeros(n) if master else None)
    if bits == 8:
        return {**t, "m": torch.zeros(blocks * 128, dtype=torch.uint8), "v": torch.zeros(blocks * 128, dtype=torch.uint8), "m_scale": torch.zeros(blocks, dtype=torch.uint8),
                "v_scale": torch.zeros(blocks, dtype=torch.uint8)}
    return {**t, "m": torch.zeros(n), "v": torch.zeros(n)}


def test_adamw_plan_lists_every_chunk():
    opt = B.AdamW([adam(n) for n in (1, 2048, 2049, 9000)])
    assert opt.args.chunks == 1 + 1 + 2 + 5 and opt.args.state_bits == 8 and opt.args.has_master == 1
    words = opt.plan[opt.plan.numel() - 8 * 9:].view(torch.int32).view(-1, 2).tolist()
    assert words == [[0, 0], [1, 0], [2, 0], [2, 1]] + [[3, c] for c in range(5)]
    assert bool((opt.plan[:256] == 0).all())


def test_adamw_refusals():
    lib = B.load()
    for wrong, error in ((dict(grad=torch.zeros(299)), ValueError), (dict(m=torch.zeros(300, dtype=torch.uint8)), ValueError), (dict(v=torch.zeros(384)), TypeError),
                         (dict(master=torch.zeros(300, dtype=torch.float64)), TypeError), (dict(v_scale=torch.zeros(2, dtype=torch.uint8)), ValueError),
                         (dict(grad=torch.zeros(300, dtype=torch.float16)), B.SmileError), (dict(param=torch.zeros(300, dtype=torch.int32)), TypeError),
                         (dict(v_scale=None), B.SmileError), (dict(weight_decay=float("inf")), B.SmileError)):
        with pytest.raises(error):
            B.AdamW([{**adam(), **wrong}])
    with pytest.raises(ValueError):
        B.AdamW([adam(), adam(master=False)])
    with pytest.raises(TypeError):
        B.AdamW([adam(), adam(dtype=torch.float16)])
    for wrong in (dict(beta1=1.0), dict(beta2=-0.1), dict(eps=0.0), dict(eps=2.0), dict(beta1=float("nan"))):
        with pytest.raises(B.SmileError) as e:
            B.AdamW([adam()], **wrong)
        assert e.value.status == B.BAD_SHAPE
    with pytest.raises(B.SmileError) as e:                                  # a master of 32-bit parameters
        B.AdamW([adam(dtype=torch.float32)])
    assert e.value.status == B.UNSUPPORTED
    opt = B.AdamW([adam()])
    call = lambda plan=P, nbytes=opt.plan.numel(), lr=P, step=P: lib.smile_adamw(C.byref(opt.args), plan, nbytes, lr, step, None)    # noqa: E731
    assert call(plan=None) == B.INVALID_ARG and call(lr=None) == B.INVALID_ARG and call(step=None) == B.INVALID_ARG
    assert call(lr=P + 2) == B.INVALID_ARG and call(step=P + 1) == B.INVALID_ARG
    assert call(plan=P + 16) == B.WORKSPACE and call(nbytes=opt.plan.numel() - 1) == B.WORKSPACE
    unpack = lambda n=256, dtype=0, m=P, ms=P, v=P, vs=P, mv=P, vv=P: lib.smile_adamw_unpack_states(n, dtype, m, ms, v, vs, mv, vv, None)    # noqa: E731
    for bad in (dict(m=None), dict(ms=None), dict(v=ODD), dict(vs=None), dict(mv=None), dict(vv=ODD)):
        assert unpack(**bad) == B.INVALID_ARG, bad
    assert unpack(n=100) == B.BAD_SHAPE and unpack(n=0) == B.BAD_SHAPE and unpack(dtype=2) == B.UNSUPPORTED


def test_overlapping_memory_is_refused():
    """What is written lies apart from what is read and from what else is written, but where a tensor may be another.  (No call here gets as far as a launch: the first
    rows that may coincide are covered on the GPU.)"""
    lib = B.load()
    M = 1 << 20                                             # pointers this far apart do not overlap
    T, k, N, d, rows, F = 16, 2, 8, 64, 32, 128
    topk = lambda **kw: lib.smile_topk(T, N, k, 1, *({**dict(logits=M, bias=2 * M, idx=3 * M, weight=4 * M, p_sum=5 * M), **kw}).values(), 6 * M, BIG, None)       # noqa: E731
    for wrong in (dict(idx=M), dict(weight=M + 16), dict(p_sum=2 * M), dict(weight=3 * M + 64), dict(idx=M + T * N * 4 - 16)):
        assert topk(**wrong) == B.INVALID_ARG, wrong
    tback = lambda **kw: lib.smile_topk_backward(T, N, k, 1, *({**dict(logits=M, bias=2 * M, idx=3 * M, dweight=4 * M, count=5 * M), **kw}).values(), 1.0, 6 * M, None)     # noqa: E731
    for wrong in (dict(logits=6 * M + 16), dict(bias=6 * M), dict(idx=6 * M + 64), dict(dweight=6 * M), dict(count=6 * M)):
        assert tback(**wrong) == B.INVALID_ARG, wrong
    sort = lambda **kw: lib.smile_sort_experts(T, k, N, *({**dict(idx=M, count=2 * M, start=3 * M, pos=4 * M, source=5 * M), **kw}).values(), 6 * M, BIG, None)      # noqa: E731
    for wrong in (dict(pos=M), dict(source=4 * M), dict(count=3 * M + 32), dict(start=M + 64)):
        assert sort(**wrong) == B.INVALID_ARG, wrong
    assert lib.smile_sorted_dispatch(T, k, d, rows, 1, M, 2 * M, M + 16, None) == B.INVALID_ARG
    assert lib.smile_sorted_dispatch(T, k, d, rows, 1, M, 2 * M, 2 * M + 16, None) == B.INVALID_ARG
    combine = lambda **kw: lib.smile_sorted_combine(T, k, d, rows, 1, *({**dict(ys=M, pos=2 * M, weight=3 * M, residual=4 * M, y=5 * M), **kw}).values(), None)      # noqa: E731
    for wrong in (dict(ys=5 * M), dict(pos=5 * M), dict(weight=5 * M + 16), dict(residual=5 * M + 16)):
        assert combine(**wrong) == B.INVALID_ARG, wrong
    back = lambda **kw: lib.smile_sorted_combine_backward(T, k, d, rows, 1, *({**dict(dy=M, ys=2 * M, pos=3 * M, weight=4 * M, dys=5 * M, dweight=6 * M), **kw}).values(), None)      # noqa: E731
    for wrong in (dict(dys=M), dict(dys=2 * M + 128), dict(dweight=4 * M), dict(dweight=5 * M), dict(pos=6 * M)):
        assert back(**wrong) == B.INVALID_ARG, wrong

    def linear(cls, function, tail, **kw):
        a = cls(N, rows, d, F, 1, kw.pop("act", 1))
        for i, (name, _) in enumerate(cls._fields_[6:]):
            setattr(a, name, kw.pop(name, M * (i + 1)))
        assert not kw
        return function(C.byref(a), *tail, None)

    forward = lambda **kw: linear(B.LinearArgs, lib.smile_linear, (), **kw)                                       # noqa: E731
    x, w, bias, residual, start, y, pre = (M * (i + 1) for i in range(7))
    for wrong in (dict(y=x), dict(y=w + 16), dict(y=bias), dict(y=start), dict(y=residual + 16), dict(pre=y), dict(pre=x + 128), dict(pre=residual), dict(y=residual, pre=residual)):
        assert forward(**wrong) == B.INVALID_ARG, wrong
    backward = lambda **kw: linear(B.LinearBackwardArgs, lib.smile_linear_backward, (64 * M, BIG), **kw)          # noqa: E731
    dy, x, w, pre, start, dx, dw, db = (M * (i + 1) for i in range(8))
    for wrong in (dict(dx=dy), dict(dx=x + 16), dict(dx=w), dict(dx=pre), dict(dw=x), dict(dw=w), dict(dw=dx), dict(dbias=start), dict(dbias=dw + 1024), dict(dw=dy + 32)):
        assert backward(**wrong) == B.INVALID_ARG, wrong
        assert backward(act=0, **wrong) == B.INVALID_ARG, wrong
    shared = adam()
    for wrong in ([shared, shared], [shared, {**adam(), "param": shared["param"]}], [{**adam(), "m": shared["v"], "v": shared["v"]}],
                  [shared, {**adam(), "m_scale": shared["v_scale"]}]):
        with pytest.raises(B.SmileError) as e:
            B.AdamW(wrong)
        assert e.value.status == B.INVALID_ARG
    B.AdamW([shared, {**adam(), "grad": shared["grad"]}])   # a gradient is only read


def test_binding_refuses_shapes_and_types():
    f32, i32 = torch.float32, torch.int32
    z = torch.zeros
    with pytest.raises(TypeError):
        B.smile_topk(z(4, 8, dtype=torch.bfloat16), z(4, 2, dtype=i32), z(4, 2))
    with pytest.raises(ValueError):
        B.smile_topk(z(4, 8), z(4, 2, dtype=i32), z(4, 3))
    with pytest.raises(ValueError):
        B.smile_topk_backward(z(4, 8), z(4, 2, dtype=i32), z(4, 2), z(4, 7))
    with pytest.raises(ValueError):
        B.smile_sort_experts(z(4, 2, dtype=i32), z(8, dtype=i32), z(8, dtype=i32), z(4, 2, dtype=i32), z(8, dtype=i32))
    with pytest.raises(TypeError):
        B.smile_sorted_dispatch(z(4, 64), z(4, 2, dtype=torch.int64), z(8, 64))
    with pytest.raises(ValueError):
        B.smile_sorted_combine(z(8, 64), z(4, 2, dtype=i32), z(4, 72))
    with pytest.raises(ValueError):
        B.smile_sorted_combine_backward(z(4, 64), z(7, 64), z(4, 2, dtype=i32), z(4, 2), z(8, 64), z(4, 2))
    x, w, y = z(4, 64), z(2, 72, 64), z(4, 72)
    for wrong in (dict(w=z(2, 72, 56)), dict(y=z(4, 64)), dict(bias=z(72)), dict(residual=z(3, 72)), dict(start=z(2, dtype=i32)), dict(pre=z(4, 71))):
        with pytest.raises(ValueError):
            B.make_linear_args(**{**dict(x=x, w=w, y=y, start=z(3, dtype=i32)), **wrong})
    for wrong in (dict(w=w.half()), dict(bias=z(2, 72, dtype=torch.float16)), dict(start=z(3, dtype=torch.int64))):
        with pytest.raises(TypeError):
            B.make_linear_args(**{**dict(x=x, w=w, y=y, start=z(3, dtype=i32)), **wrong})
    with pytest.raises(AssertionError):                     # rows of another stride
        B.make_linear_args(x=z(4, 128)[:, ::2], w=w, y=y, start=z(3, dtype=i32))
    with pytest.raises(ValueError):
        B.make_linear_backward_args(y, x, w, dx=z(4, 72), start=z(3, dtype=i32))


def test_reference_gradients_against_differences():
    g = torch.Generator().manual_seed(1)
    n = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)        # noqa: E731
    start = torch.tensor([0, 3, 3, 9])
    x, w, b, dy, vx, vw, vb = n(9, 5), n(3, 4, 5), n(3, 4), n(9, 4), n(9, 5), n(3, 4, 5), n(3, 4)
    for name in ("none", "gelu"):
        def loss(h):
            return float((R.linear(x + h * vx, w + h * vw, b + h * vb, name, None, start)[0] * dy).sum())
        out = R.linear_backward(dy, x, w, R.linear(x, w, b, name, None, start)[1], name, start)
        total = sum(float((out[k][0] * v).sum()) for k, v in (("dx", vx), ("dw", vw), ("dbias", vb)))
        assert abs((loss(1e-6) - loss(-1e-6)) / 2e-6 - total) < 1e-6 * (1 + abs(total))
    logits, dweight, count, v = n(6, 7).float(), n(6, 3).float(), torch.arange(7, dtype=torch.int32), n(6, 7)
    for normalize in (False, True):
        idx, weight, p, _ = R.topk(logits, None, 3, normalize)
        grad, _ = R.topk_backward(p, idx, weight, dweight, normalize, count, 0.1)

        def loss(h):
            p = torch.softmax(logits.double() + h * v, 1)
            ww = p.gather(1, idx.long())
            return float((dweight.double() * (ww / ww.sum(1, keepdim=True) if normalize else ww)).sum() + 0.1 * (count.double() * p.sum(0)).sum())
        assert abs((loss(1e-6) - loss(-1e-6)) / 2e-6 - float((grad * v).sum())) < 1e-6


def test_adamw_refuses_an_eps_below_the_normal_range():
    """fp32 has no reciprocal of it"""
    for eps in (1e-300, 2.0 ** -149, 2.9e-39, 2.0 ** -126 * (1 - 2.0 ** -20), -1e-8, float("nan")):
        with pytest.raises(B.SmileError) as e:
            B.AdamW([adam()], eps=eps)
        assert e.value.status == B.BAD_SHAPE, eps
    for eps in (2.0 ** -126, 1e-30, 1.0):
        B.AdamW([adam()], eps=eps)


def test_memory_that_may_be_another_tensors_is_no_other():
    """y may be the residual, dlogits the logits; no further tensor may lie there too, though it begins at the same place"""
    lib = B.load()
    M = 1 << 20
    a = B.LinearArgs(1, 32, 64, 64, 1, 1)
    for name, at in dict(x=M, w=2 * M, residual=M, y=M).items():
        setattr(a, name, at)
    assert lib.smile_linear(C.byref(a), None) == B.INVALID_ARG                    # x
    a.x, a.bias = 3 * M, M
    assert lib.smile_linear(C.byref(a), None) == B.INVALID_ARG                    # the bias
    a.bias, a.w = None, M
    assert lib.smile_linear(C.byref(a), None) == B.INVALID_ARG                    # w
    combine = lambda ys, pos, weight: lib.smile_sorted_combine(16, 2, 64, 32, 1, ys, pos, weight, 5 * M, 5 * M, None)       # noqa: E731
    assert combine(5 * M, 2 * M, 3 * M) == combine(M, 5 * M, 3 * M) == combine(M, 2 * M, 5 * M) == B.INVALID_ARG
    back = lambda bias, idx, dweight, count: lib.smile_topk_backward(16, 8, 2, 1, M, bias, idx, dweight, count, 1.0, M, None)      # noqa: E731
    for i in range(4):
        assert back(*(M if j == i else (j + 2) * M for j in range(4))) == B.INVALID_ARG, i


def test_gradients_lie_apart_from_what_a_step_writes():
    """A chunk's gradient is read while others are stored: it shares no memory with any tensor's parameter or state.  Gradients may share theirs."""
    flat = torch.zeros(1 << 14)
    cut = lambda lo, n=300: flat[lo:lo + n]                                                 # noqa: E731
    one = lambda at: dict(param=cut(at), grad=cut(at + 400), m=cut(at + 800), v=cut(at + 1200))    # noqa: E731
    B.AdamW([one(0), one(2000), one(4000)])
    B.AdamW([one(0), {**one(2000), "grad": cut(404)}, {**one(4000), "grad": cut(500)}])     # (between two tensors that are written)
    for at in (0, 2000, 2296, 1704, 800, 1200, 2800 + 296, 3200 - 296):
        for i in (0, 1):
            tensors = [one(0), one(2000)]
            tensors[i]["grad"] = cut(at)
            with pytest.raises(B.SmileError) as e:
                B.AdamW(tensors)
            assert e.value.status == B.INVALID_ARG, (at, i)
    for name in ("master", "m", "v", "m_scale", "v_scale"):                                 # states in 8 bits, a master
        t = adam(n=1024, grad=torch.float32)
        big = torch.zeros(1 << 13, dtype=torch.uint8)
        t["grad"] = big[:4096].view(torch.float32)
        t[name] = big[4096 - 16:4096 - 16 + t[name].numel() * t[name].element_size()].view(t[name].dtype)
        with pytest.raises(B.SmileError) as e:
            B.AdamW([t])
        assert e.value.status == B.INVALID_ARG, name


def test_workspaces_lie_apart_from_the_tensors():
    """Kernels of one call write the workspace and read it again between reading and writing the others"""
    lib = B.load()
    M = 1 << 24
    T, k, N = 20000, 2, 64
    topk = lambda ws, **kw: lib.smile_topk(T, N, k, 1, *({**dict(logits=M, bias=2 * M, idx=3 * M, weight=4 * M, p_sum=5 * M), **kw}).values(), ws, BIG, None)       # noqa: E731
    need = B.smile_topk_workspace_bytes(T, N)
    assert need > 0
    for i in range(1, 6):
        assert topk(i * M) == B.INVALID_ARG and topk(i * M - need + 256) == B.INVALID_ARG, i
    sort = lambda ws: lib.smile_sort_experts(T, k, N, M, 2 * M, 3 * M, 4 * M, 5 * M, ws, BIG, None)         # noqa: E731
    need = B.smile_sort_experts_workspace_bytes(T, k, N)
    assert need > 0
    for i in range(1, 6):
        assert sort(i * M) == B.INVALID_ARG and sort(i * M - need + 256) == B.INVALID_ARG, i
    for act in (1, 2):
        a = B.LinearBackwardArgs(2, 64, 64, 128, 1, act)
        names = [name for name, _ in B.LinearBackwardArgs._fields_[6:]]
        for i, name in enumerate(names):
            setattr(a, name, (i + 1) * M)
        size = C.c_size_t(0)
        assert lib.smile_linear_backward_workspace_bytes(C.byref(a), C.byref(size)) == B.OK and size.value > 0
        for i, name in enumerate(names):
            if not (name == "pre" and act == 2):        # (not read without an activation)
                assert lib.smile_linear_backward(C.byref(a), (i + 1) * M, BIG, None) == B.INVALID_ARG, name
                assert lib.smile_linear_backward(C.byref(a), (i + 1) * M - size.value + 256, BIG, None) == B.INVALID_ARG, name


def test_states_as_values_lie_apart_from_their_codes():
    lib = B.load()
    M, n = 1 << 20, 1 << 12
    unpack = lambda dtype=0, **kw: lib.smile_adamw_unpack_states(n, dtype, *({**dict(m=M, ms=2 * M, v=3 * M, vs=4 * M, mv=5 * M, vv=6 * M), **kw}).values(), None)    # noqa: E731
    for wrong in (dict(mv=M), dict(vv=3 * M), dict(mv=3 * M + n - 16), dict(vv=M), dict(ms=5 * M + 1), dict(vs=6 * M + 4 * n - 1), dict(mv=6 * M), dict(mv=6 * M - 4 * n + 16),
                  dict(m=6 * M + 4 * n - 16)):
        assert unpack(**wrong) == B.INVALID_ARG, wrong
    for wrong in (dict(mv=6 * M - 2 * n + 16), dict(v=5 * M + 2 * n - 16)):
        assert unpack(dtype=1, **wrong) == B.INVALID_ARG, wrong


def test_step_learning_rate_and_plan_lie_apart():
    lib = B.load()
    M, opt = 1 << 20, B.AdamW([adam()])
    n = opt.plan.numel()
    call = lambda plan=M, lr=2 * M, step=3 * M: lib.smile_adamw(C.byref(opt.args), plan, n, lr, step, None)      # noqa: E731
    for wrong in (dict(lr=3 * M), dict(lr=M), dict(lr=M + 4 * (n // 4) - 4), dict(step=M), dict(step=M + 256)):
        assert call(**wrong) == B.INVALID_ARG, wrong
