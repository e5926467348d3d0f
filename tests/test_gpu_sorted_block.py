"""The layer without dropped tokens (sorted_block.py) end to end: against automatic differentiation of its definition in 64 bits, with the experts that the GPU chose, and
its whole training step captured into a graph.

Tolerance, normwise: a chain of at most six roundings to the storage type (rows' gradients pass the return, the product, the activation's argument, its gradient, the
product, the sum), each at most half a step: 6 * 2^-8 for bfloat16, 6 * 2^-11 for half precision, and for fp32 sums of at most 512 terms beside a softmax, 2^-24 * 512."""
import math

import pytest
import torch

import sorted_reference as R
from paper_2212_05191_amd import binding as B
from paper_2212_05191_amd.sorted_block import SortedBlock

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
TOL = {"f32": 512 * 2.0 ** -24, "bf16": 6 * 2.0 ** -8, "f16": 6 * 2.0 ** -11}


def make(g, T, k, N, d, F, dtype, **kw):
    st = TYPES[dtype]
    normal = lambda *s, std=1.0: (std * torch.randn(*s, device="cuda:0", generator=g)).to(st)       # noqa: E731
    params = [normal(N, d, std=0.3), normal(N, F, d, std=d ** -0.5), normal(N, F, std=0.2), normal(N, d, F, std=F ** -0.5), normal(N, d, std=0.2)]
    return SortedBlock(T, k, *params, **kw), normal


def definition(x, residual, wr, w1, b1, w2, b2, idx, bias, act, normalize, balance):
    """y and the load-balancing term, experts' choice given"""
    T, k = idx.shape
    N = wr.shape[0]
    v = x @ wr.T
    if bias is not None:
        v = torch.where(bias == -math.inf, -math.inf, v + bias)
    p = torch.softmax(v, 1)
    w = p.gather(1, idx.clamp_min(0)) * (idx >= 0)
    if normalize:
        w = w / w.sum(1, keepdim=True)
    y = residual
    count = torch.zeros(N, dtype=torch.float64, device=x.device)
    for e in range(N):
        t, j = torch.nonzero(idx == e, as_tuple=True)
        count[e] = t.numel()
        h = R.act(x[t] @ w1[e].T + b1[e], act)
        y = y.index_add(0, t, w[t, j][:, None] * (h @ w2[e].T + b2[e]))
    return y, balance * N / (k * T * T) * (count * p.sum(0)).sum()


CASES = [("bf16", "gelu", 300, 2, 8, 128, 256, True, False), ("f16", "relu", 257, 3, 5, 64, 192, False, True), ("f32", "gelu", 130, 2, 6, 72, 136, True, True),
         ("bf16", "none", 1, 1, 2, 64, 64, False, False), ("bf16", "gelu", 64, 8, 16, 64, 128, True, True)]


@pytest.mark.parametrize("dtype,act,T,k,N,d,F,normalize,masked", CASES)
def test_block_forward_and_backward(dtype, act, T, k, N, d, F, normalize, masked):
    g = torch.Generator(device="cuda:0").manual_seed(T)
    bias = None
    if masked:
        bias = torch.randn(N, device="cuda:0", generator=g) * 0.3
        bias[1] = -math.inf
    block, normal = make(g, T, k, N, d, F, dtype, act=act, normalize=normalize, bias=bias, balance=2.0)
    x, residual, dy = normal(T, d), normal(T, d), normal(T, d)
    y = block.forward(x, residual)
    loss = block.loss()
    dx = block.backward(x, dy, dloss=0.7)
    torch.cuda.synchronize()
    leaves = [t.double().requires_grad_(True) for t in (x, residual, block.w_router, block.w1, block.b1, block.w2, block.b2)]
    want, want_loss = definition(*leaves, block.idx.long(), None if bias is None else bias.double(), act, normalize, 2.0)
    if act == "relu":   # the side of zero of a sum next to it goes by its roundings: such units count on neither side
        rows = x.double()[torch.div(block.source[:int(block.start[-1])].long(), k, rounding_mode="floor")]
        pre = torch.cat([rows[lo:hi] @ block.w1[e].double().T + block.b1[e].double() for e, (lo, hi) in enumerate(R.groups(block.start, T * k)) if hi > lo])
        kept = block.pre[:pre.shape[0]].double()
        assert bool((((kept > 0) == (pre > 0)) | (pre.abs() < 1e-3)).all())
    ((want * dy.double()).sum() + 0.7 * want_loss).backward()
    assert torch.equal(leaves[1].grad, dy.double())
    names = ("y", "dx", "dw_router", "dw1", "db1", "dw2", "db2")
    for name, got, ref in zip(names, (y, dx, block.dw_router, block.dw1, block.db1, block.dw2, block.db2),
                              (want, leaves[0].grad, *(leaf.grad for leaf in leaves[2:]))):
        ref = ref.detach()
        if float(ref.norm()) == 0.0:
            assert bool((got == 0).all()), name
            continue
        off = float((got.double() - ref).norm() / ref.norm())
        assert off <= TOL[dtype], (name, off)
    assert abs(float(loss) - float(want_loss.detach())) <= 1e-4 * float(want_loss.detach())
    count = torch.bincount(block.idx[block.idx >= 0].flatten().long(), minlength=N)
    assert torch.equal(block.count.long(), count) and int(block.start[-1]) == int(count.sum())
    block.close()


@pytest.mark.parametrize("bits", (8, 32))
def test_captured_training_step(bits):
    """forward, backward and AdamW as one graph, replayed with other tokens, beside eager steps of a twin: the same bits, steps counted"""
    T, k, N, d, F = 200, 2, 6, 64, 128
    a, normal = make(torch.Generator(device="cuda:0").manual_seed(3), T, k, N, d, F, "bf16", optimizer=bits)
    b, _ = make(torch.Generator(device="cuda:0").manual_seed(3), T, k, N, d, F, "bf16", optimizer=bits)
    x, residual, dy, lr = normal(T, d), normal(T, d), normal(T, d), torch.full((1,), 1e-2, device="cuda:0")

    def run(block):
        block.forward(x, residual)
        block.backward(x, dy)
        block.step(lr)

    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        run(a), run(b)
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            run(b)
    for i in range(4):
        x.copy_(normal(T, d))
        lr.fill_(1e-2 / (i + 1))
        run(a)
        graph.replay()
        torch.cuda.synchronize()
        assert float((a.w1 != 0).float().mean()) > 0.5
        for name in ("y", "dx", "w_router", "w1", "b1", "w2", "b2", "dw1", "dw_router"):
            assert torch.equal(getattr(a, name), getattr(b, name)), (i, name)
    for (_, ta, ca), (_, tb, cb) in zip(a.optimizers, b.optimizers):
        assert int(ca) == int(cb) == 5
        for u, v in zip(ta, tb):
            assert all(torch.equal(u[n], v[n]) for n in ("m", "v", "master"))
    a.close(), b.close()


def test_step_moves_the_parameters_as_the_definition_does():
    T, k, N, d, F = 150, 2, 4, 64, 64
    block, normal = make(torch.Generator(device="cuda:0").manual_seed(5), T, k, N, d, F, "bf16", optimizer=32, weight_decay=0.1)
    x, dy, lr = normal(T, d), normal(T, d), torch.full((1,), 1e-2, device="cuda:0")
    block.forward(x)
    block.backward(x, dy)
    before = {n: getattr(block, n).double() for n in ("w_router", "w1", "b1", "w2", "b2")}
    block.step(lr)
    for n, p in before.items():
        g = getattr(block, "d" + n).double()
        want, *_ = R.adamw(p, g, torch.zeros_like(p), torch.zeros_like(p), 1, float(lr), 0.1 if n.startswith("w") else 0.0, 0.9, 0.999, 1e-8)
        got = getattr(block, n).double()
        # the first update is lr times the sign of the gradient (a dozen roundings of it), the parameter is rounded once
        assert bool(((got - want).abs() <= want.abs() * 2.0 ** -8 * 1.001 + 1e-2 * 2.0 ** -19).all()), n
    block.close()


@pytest.mark.parametrize("dtype,bits", [("bf16", 8), ("bf16", 32), ("f32", 32)])
def test_parameters_that_are_loaded_stay(dtype, bits):
    """After a checkpoint's parameters were copied in, a step moves those; with new states the block is the one that was made with them"""
    T, k, N, d, F = 100, 2, 4, 64, 64
    gen = lambda seed: torch.Generator(device="cuda:0").manual_seed(seed)           # noqa: E731
    names = ("w_router", "w1", "b1", "w2", "b2")
    block, normal = make(gen(5), T, k, N, d, F, dtype, optimizer=bits)
    fresh, _ = make(gen(6), T, k, N, d, F, dtype, optimizer=bits)
    x, dy, lr = normal(T, d), normal(T, d), torch.full((1,), 1e-3, device="cuda:0")

    def run(b):
        b.forward(x)
        b.backward(x, dy)
        b.step(lr)
    run(block)
    loaded = {n: getattr(fresh, n).clone() for n in names}
    for n in names:
        getattr(block, n).copy_(loaded[n])
    block.take_parameters()
    run(block)
    # the second step of AdamW: with |m| <= 0.1 (0.9 |g1| + |g2|) / 0.19 and v >= 0.001 (0.999 g1^2 + g2^2) / 0.002 the quotient is below 1.01; beside it the decay, 0.1 |p|.  (Not so
    # with moments in 8 bits: one that is rounded up beside larger ones may exceed its own v's root by far.)
    for n in names if bits == 32 else ():
        p, q = getattr(block, n).double(), loaded[n].double()
        assert bool(((p - q).abs() <= 1e-3 * (1.01 + 0.1 * q.abs()) + q.abs() * R.HALF[TYPES[dtype]] * 1.01).all()) and bool((p != q).any()), n
    for n in names:
        getattr(block, n).copy_(loaded[n])
    block.take_parameters(new_states=True)
    run(block), run(fresh)
    for n in names:
        assert torch.equal(getattr(block, n), getattr(fresh, n)), n
    for (_, a, ca), (_, b, cb) in zip(block.optimizers, fresh.optimizers):
        assert int(ca) == int(cb) == 1 and all(torch.equal(u[m], v[m]) for u, v in zip(a, b) for m in ("m", "v"))
    block.close(), fresh.close()
