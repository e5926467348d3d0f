"""The 8-bit block (fp8_block.py) end to end against the definition in 64 bits, with the routing decisions of the GPU.

Tolerance: normwise 2e-2.  The outputs are bfloat16 chains of at most four roundings of 2^-8 at most each (rms a third of that), and an 8-bit code
that falls the other way at a tie moves a value by a sixteenth at most, which fewer than one value in a hundred does (its 32-bit sum is off by
a few 2^-17): sqrt(0.01) / 16 < 1e-2."""
import numpy as np
import pytest
import torch

import fp8_reference as R
from paper_2212_05191_amd import binding as B
from paper_2212_05191_amd.fp8_block import Fp8Block

pytestmark = pytest.mark.gpu
TOL = 2e-2


def host(t):
    return t.detach().cpu().double().numpy() if t.is_floating_point() else t.detach().cpu().numpy().astype(np.int64)


def q8(v):
    c, s = R.pack_rows(v)
    return R.unpack_rows(c, s, v.shape[2])


def near(name, got, want):
    got = host(got)
    off = np.linalg.norm(got - want) / np.linalg.norm(want)
    assert off <= TOL, (name, off)


@pytest.mark.parametrize("act,dtype,T,d,F,n,m,cap", [("gelu", "bf16", 500, 192, 320, 2, 3, 96), ("relu", "f16", 300, 128, 256, 2, 2, 60),
                                                     ("gelu", "bf16", 1, 64, 128, 2, 2, 1)])
def test_block_forward_and_backward(act, dtype, T, d, F, n, m, cap):
    st = B.torch_dtype(dtype)
    g = torch.Generator(device="cuda:0").manual_seed(T)

    def normal(*shape, std=1.0):
        return (std * torch.randn(*shape, device="cuda:0", generator=g)).to(st)

    N = n * m
    x, res, dy, dsum = normal(T, d), normal(T, d, std=2.0), normal(T, d), normal(T, d)
    nw, wi, wq, w1, w2 = normal(d, std=0.1) + 1, normal(n, d, std=0.1), normal(m, d, std=0.1), normal(N, F, d, std=0.05), normal(N, d, F, std=0.05)
    desc = B.make_desc(T, d, F, n, m, cap, dtype, act)
    block = Fp8Block(desc, nw, wi, wq, w1, w2)
    s, y = block.forward(x, res)
    ds = block.backward(dy, dsum=dsum)
    torch.cuda.synchronize()
    b, bw = block.buf, block.bwd
    gi, li, slot, kept = host(b.group_idx), host(b.local_idx), host(b.slot), host(b.kept_count)

    # forward
    sv, u_kept = host(s), host(block.u)
    near("s", s, host(x) + host(res))
    rstd, u = R.rms_norm(sv, host(nw), 1e-5)
    near("u", block.u, u)
    u8 = R.unpack_rows(*(host(t).astype(np.uint8) for t in block.u8), d)[0]       # the GPU's own codes: ties are tested elsewhere
    assert np.linalg.norm(u8 - u) <= 2.0 ** -4 * np.linalg.norm(u)
    lp, lq = u_kept @ host(wi).T, u_kept @ host(wq).T
    assert np.array_equal(gi, host(b.logits_inter).argmax(1)) and np.abs(host(b.logits_inter) - lp).max() < 1e-3
    p, q = (np.exp(a - a.max(1, keepdims=True)) for a in (lp, lq))
    p, q = p / p.sum(1, keepdims=True), q / q.sum(1, keepdims=True)
    at = np.arange(T)
    gate = p[at, gi] * q[at, li]
    e = gi * m + li
    live = slot >= 0
    xe = np.zeros((N, cap, d))
    xe[e[live], slot[live]] = u8[live]
    W1, W2 = (R.unpack_weights(*(a for a in R.pack_weights(host(w))), w.shape[2]) for w in (w1, w2))
    pre = xe @ W1.transpose(0, 2, 1)
    h = q8(R.act(pre, act))
    ye = h @ W2.transpose(0, 2, 1)
    yv = np.where(live[:, None], gate[:, None] * ye[e, np.maximum(slot, 0)], 0.0)
    near("y", y, yv)

    # backward
    mask = (np.arange(cap)[None, :] < kept[:, None])[:, :, None]
    dyv = host(dy)
    dye, dgate = np.zeros((N, cap, d)), np.zeros(T)
    # rounded to the storage type as the definition has it: the 8-bit rows are made of that, and a step of bfloat16 moves one code in twenty
    dye[e[live], slot[live]] = torch.from_numpy((gate[live, None] * dyv[live]).astype(np.float32)).to(st).double().numpy()
    dgate[live] = np.sum(dyv[live] * ye[e[live], slot[live]], axis=1)
    dpre = (q8(dye) @ W2) * R.act_grad(q8(pre), act) * mask
    dxe = q8(dpre) @ W1
    near("dw2", bw.dw2, dye.transpose(0, 2, 1) @ (h * mask))
    near("dw1", bw.dw1, dpre.transpose(0, 2, 1) @ (xe * mask))
    f, fq = np.bincount(gi, minlength=n) / T, np.bincount(li, minlength=m) / T
    up = 0.005 * n * f[None, :] / T + np.eye(n)[gi] * (dgate * q[at, li])[:, None]
    uq = 0.005 * m * fq[None, :] / T + np.eye(m)[li] * (dgate * p[at, gi])[:, None]
    dlp, dlq = p * (up - (up * p).sum(1, keepdims=True)), q * (uq - (uq * q).sum(1, keepdims=True))
    near("dw_inter", bw.dw_inter, dlp.T @ u_kept)
    near("dw_intra", bw.dw_intra, dlq.T @ u_kept)
    du = dlp @ host(wi) + dlq @ host(wq)
    du[live] += dxe[e[live], slot[live]]
    want_ds, want_dn = R.rms_norm_backward(du, sv, host(nw), 1e-5, host(dsum))
    near("ds", ds, want_ds)
    near("dnorm", block.dnorm, want_dn)
    block.close()


def test_serving_block_keeps_nothing_for_a_backward_pass_and_gives_the_same_y():
    T, d, F = 40, 128, 256
    g = torch.Generator(device="cuda:0").manual_seed(2)
    r = lambda *shape, std=1.0: (std * torch.randn(*shape, device="cuda:0", generator=g)).bfloat16()      # noqa: E731
    desc = B.make_desc(T, d, F, 2, 2, 30, "bf16", "gelu")
    args = (r(d) + 1, r(2, d), r(2, d), r(4, F, d, std=0.05), r(4, d, F, std=0.05))
    x, res = r(T, d), r(T, d)
    train, serve = Fp8Block(desc, *args), Fp8Block(desc, *args, training=False)
    assert not hasattr(serve, "pre8") and serve.w1t is None
    a, b = train.forward(x, res), serve.forward(x, res)
    torch.cuda.synchronize()
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    train.close()
    serve.close()


def test_weights_are_packed_on_the_stream_that_the_step_takes():
    """A step as a program takes it whose work goes to a stream of its own by handle: the new weights are packed there, in front of the forward pass
    that reads them."""
    desc = B.make_desc(64, 128, 256, 2, 2, 32, "bf16", "gelu")
    g = torch.Generator(device="cuda:0").manual_seed(9)
    normal = lambda *shape: (0.05 * torch.randn(*shape, device="cuda:0", generator=g)).bfloat16()      # noqa: E731
    x, res, nw, wi, wq = normal(64, 128) * 20, normal(64, 128) * 20, normal(128) + 1, normal(2, 128), normal(2, 128)
    w1, w2, new1, new2 = normal(4, 256, 128), normal(4, 128, 256), normal(4, 256, 128), normal(4, 128, 256)
    want = Fp8Block(desc, nw, wi, wq, new1, new2)
    expect = want.forward(x, res)[1].clone()
    block = Fp8Block(desc, nw, wi, wq, w1, w2)
    assert not torch.equal(block.forward(x, res)[1], expect)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    block.pack_weights(new1, new2, stream=side)
    _, y = block.forward(x, res, stream=side)
    side.synchronize()
    assert torch.equal(y, expect)
    for a, b in ((block.w1t, want.w1t), (block.w2t, want.w2t)):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    want.close()
    block.close()


def test_a_stack_of_blocks_shares_its_scratch_memory():
    """Two blocks, the second on what the first returns: gradients with one scratch memory for both are those with two, and a block
    with a shared one allocates none."""
    desc = B.make_desc(200, 128, 256, 2, 2, 60, "bf16", "gelu")
    g = torch.Generator(device="cuda:0").manual_seed(4)
    normal = lambda *shape: (0.05 * torch.randn(*shape, device="cuda:0", generator=g)).bfloat16()      # noqa: E731
    x, res, dy = normal(200, 128) * 20, normal(200, 128) * 20, normal(200, 128) * 20
    weights = [(normal(128) + 1, normal(2, 128), normal(2, 128), normal(4, 256, 128), normal(4, 128, 256)) for _ in range(2)]

    def gradients(share):
        first = Fp8Block(desc, *weights[0])
        second = Fp8Block(desc, *weights[1], scratch=first.scratch if share else None)
        assert (second.scratch is first.scratch) == share
        with pytest.raises(ValueError):
            Fp8Block(B.make_desc(201, 128, 256, 2, 2, 60, "bf16", "gelu"), *weights[1], scratch=first.scratch)
        s, y = first.forward(x, res)
        second.forward(y, s)
        ds = second.backward(dy)              # the gradient of y and of s alike
        first.backward(ds, dsum=ds)
        torch.cuda.synchronize()
        out = [t.clone() for b in (first, second) for t in (b.ds, b.dnorm, b.bwd.dw1, b.bwd.dw2, b.bwd.dw_inter, b.bwd.dw_intra)]
        first.close()
        second.close()
        return out

    assert all(torch.equal(a, b) and bool(a.abs().sum() > 0) for a, b in zip(gradients(True), gradients(False)))
