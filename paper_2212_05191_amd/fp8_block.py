"""A pre-norm expert block on the 8-bit operators: what stands around and inside the layer when its products run in 8 bits.

    s = x + residual,  u = rms_norm(s) in the storage type (for the routers) and in 8 bits (for the experts)
    routing of u as in the 16-bit layer, dispatch of the 8-bit rows, up-projection with activation to 8-bit hidden rows,
    down-projection, gate-weighted return y, load-balancing loss

and its backward pass, for which the forward pass keeps 8-bit rows alone: the dispatched tokens, the hidden rows and the
pre-activations, half of the bytes of the 16-bit layer.  Marshalling only: every step is a library call.

    python -m paper_2212_05191_amd.fp8_block     # one training step of the base layer, timed, beside the 16-bit layer's
"""
from __future__ import annotations

import torch

from . import binding as B


class Fp8Scratch:
    """What a block's backward pass needs while it runs: the experts' gradients on their way and one workspace for all of its calls.  Blocks of one
    desc whose backward passes follow each other on one stream can share it."""

    def __init__(self, desc: B.LayerDesc, device="cuda:0"):
        T, d, F, cap = desc.T, desc.d_model, desc.d_ff, desc.capacity
        N = desc.n_groups * desc.m_local
        st = B.torch_dtype(desc.dtype)
        self.made_for = self._key(desc)
        self.dye, self.dxe = (torch.empty((N, cap, d), dtype=st, device=device) for _ in range(2))
        self.dpre = torch.empty((N, cap, F), dtype=st, device=device)
        self.dye8, self.dpre8 = B.alloc_fp8_rows(N, cap, d, device), B.alloc_fp8_rows(N, cap, F, device)
        nbytes = max(B.smile_backward_workspace_bytes(desc), B.smile_rms_norm_backward_workspace_bytes(T, d),
                     B.smile_fp8_weight_grad_workspace_bytes(N, cap, max(d, F), desc.dtype))
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=device)

    @staticmethod
    def _key(desc):
        return desc.T, desc.d_model, desc.d_ff, desc.n_groups, desc.m_local, desc.capacity, desc.dtype

    def check(self, desc):
        if self.made_for != self._key(desc):
            raise ValueError(f"scratch memory of a block of {self.made_for}, not {self._key(desc)} (tokens, widths, experts, capacity, type)")

    def nbytes(self):
        return sum(t.numel() * t.element_size() for t in (self.dye, self.dxe, self.dpre, *self.dye8, *self.dpre8, self.workspace))


class Fp8Block:
    """Weights, buffers and argument blocks of one block for T tokens; w1[N, F, d], w2[N, d, F], the routers' weights and
    norm_weight[d] in a 16-bit storage type, without expert biases.  scratch: that of another block, to share it."""

    def __init__(self, desc: B.LayerDesc, norm_weight, w_inter, w_intra, w1, w2, eps=1e-5, training=True, scratch=None):
        T, d, F, cap = desc.T, desc.d_model, desc.d_ff, desc.capacity
        N = desc.n_groups * desc.m_local
        st, dev = B.torch_dtype(desc.dtype), w1.device
        act = {0: "relu", 1: "gelu"}[desc.act]
        self.desc, self.eps = desc, eps
        self.norm_weight, self.w_inter, self.w_intra = norm_weight, w_inter, w_intra
        self.ctx = B.Ctx(desc)
        self.buf = B.alloc_buffers(desc, dev)
        b = self.buf
        b.xe = None                      # the experts read 8-bit rows
        self.sum, self.u = (torch.empty((T, d), dtype=st, device=dev) for _ in range(2))
        self.rstd = torch.empty(T, dtype=torch.float32, device=dev)
        self.u8, self.xe8, self.h8 = B.alloc_fp8_rows(1, T, d, dev), B.alloc_fp8_rows(N, cap, d, dev), B.alloc_fp8_rows(N, cap, F, dev)
        self.w1, self.w2 = B.alloc_fp8_weights(N, F, d, dev), B.alloc_fp8_weights(N, d, F, dev)
        self.w1t = self.w2t = None
        keep = {}
        if training:
            self.w1t, self.w2t = B.alloc_fp8_weights(N, d, F, dev), B.alloc_fp8_weights(N, F, d, dev)
            self.pre8 = B.alloc_fp8_rows(N, cap, F, dev)
            keep = dict(pre8=self.pre8[0], pre_scale=self.pre8[1])
        self.pack_weights(w1, w2)
        rows = b.kept_count
        self.up = B.make_fp8_gemm_args(*self.xe8, *self.w1, d, F, rows=rows, act=act, y8=self.h8[0], y_scale=self.h8[1], **keep)
        self.down = B.make_fp8_gemm_args(*self.h8, *self.w2, F, d, rows=rows, y=b.ye)
        if not training:
            return
        self.bwd = B.alloc_backward_buffers(desc, dev)
        g = self.scratch = scratch or Fp8Scratch(desc, dev)
        g.check(desc)
        self.bwd.dye, self.bwd.dxe = g.dye, g.dxe
        self.ds, self.dnorm = torch.empty((T, d), dtype=st, device=dev), torch.empty(d, dtype=torch.float32, device=dev)
        self.dup = B.make_fp8_gemm_args(*g.dye8, *self.w2t, d, F, rows=rows, act=act, y=g.dpre, y8=g.dpre8[0], y_scale=g.dpre8[1],
                                        grad8=self.pre8[0], grad_scale=self.pre8[1])
        self.ddown = B.make_fp8_gemm_args(*g.dpre8, *self.w1t, F, d, rows=rows, y=g.dxe)

    def pack_weights(self, w1, w2, stream=None):
        """The experts' weights to 8 bits: once for serving, after every optimizer step in training."""
        for w, packed, transposed in ((w1, self.w1, self.w1t), (w2, self.w2, self.w2t)):
            B.smile_fp8_pack_weights(w, *packed, *(transposed or (None, None)), stream=stream)

    def forward(self, x, residual, stream=None):
        """x, residual [T, d] -> (s, y): the residual stream after the addition, and what the block adds to it next."""
        b, ctx = self.buf, self.ctx
        B.smile_rms_norm(x, residual, self.norm_weight, self.eps, sum=self.sum, y=self.u, y8=self.u8[0], y8_scale=self.u8[1],
                         rstd=self.rstd, stream=stream)
        B.smile_gate_logits(ctx, self.u, self.w_inter, self.w_intra, b.logits_inter, b.logits_intra, stream)
        B.smile_route_bilevel(ctx, b.logits_inter, b.logits_intra, None, None, b.group_idx, b.local_idx, b.pos_in_group, b.slot,
                              b.gate, b.p_top, b.q_top, b.group_count, b.local_count, b.expert_count, b.kept_count, b.p_sum,
                              b.q_sum, stream)
        B.smile_fp8_dispatch(ctx, *self.u8, b.group_idx, b.local_idx, b.slot, *self.xe8, stream)
        B.smile_fp8_gemm(self.up, stream)
        B.smile_fp8_gemm(self.down, stream)
        B.smile_combine(ctx, b.ye, b.group_idx, b.local_idx, b.slot, b.gate, b.y, stream)
        B.smile_aux_loss(ctx, b.group_count, b.local_count, b.p_sum, b.q_sum, b.loss3, stream)
        return self.sum, b.y

    def backward(self, dy, dsum=None, dloss=1.0, stream=None):
        """dy: gradient of y, dsum: that of s from its other uses.  Gradients: ds (of x and of residual), dnorm, and in bwd
        dw_inter, dw_intra, dw1, dw2."""
        b, g, ctx, scratch = self.buf, self.bwd, self.ctx, self.scratch
        B.smile_combine_backward(ctx, dy, b.ye, b.group_idx, b.local_idx, b.slot, b.gate, g.dye, g.dgate, stream)
        B.smile_route_backward(ctx, b.logits_inter, b.logits_intra, None, None, b.group_idx, b.local_idx, g.dgate, b.group_count,
                               b.local_count, dloss, g.dlp, g.dlq, stream)
        B.smile_fp8_pack_rows(g.dye, *scratch.dye8, rows=b.kept_count, stream=stream)
        B.smile_fp8_gemm(self.dup, stream)
        B.smile_fp8_gemm(self.ddown, stream)
        B.smile_fp8_weight_grad(g.dye, *self.h8, g.dw2, scratch.workspace, rows=b.kept_count, stream=stream)
        B.smile_fp8_weight_grad(scratch.dpre, *self.xe8, g.dw1, scratch.workspace, rows=b.kept_count, stream=stream)
        B.smile_dispatch_backward(ctx, g.dxe, b.group_idx, b.local_idx, b.slot, g.dlp, g.dlq, self.w_inter, self.w_intra, g.dx,
                                  stream)
        B.smile_gate_weights_backward(ctx, self.u, g.dlp, g.dlq, g.dw_inter, g.dw_intra, scratch.workspace, stream)
        B.smile_rms_norm_backward(g.dx, self.sum, self.norm_weight, self.rstd, self.ds, self.dnorm, scratch.workspace, dsum=dsum,
                                  stream=stream)
        return self.ds

    def kept_bytes(self):
        """What the forward pass keeps of the experts' part for the backward pass."""
        return sum(t.numel() for pair in (self.xe8, self.h8, self.pre8) for t in pair)

    def packed_bytes(self):
        """The 8-bit weights, in both forms when training."""
        return sum(t.numel() for pair in (self.w1, self.w2, self.w1t, self.w2t) if pair for t in pair)

    def close(self):
        torch.cuda.synchronize()
        self.ctx.close()


def main():
    from . import workloads as wl
    from .runner import GpuLayer
    cfg = wl.CONFIGS["cfg2"]
    layer = GpuLayer(cfg)
    layer.enable_saved_activations()
    layer.prepare_backward(wl.gen_output_grad(cfg))
    T, d = cfg.T, cfg.d_model
    gen = torch.Generator(device="cuda:0").manual_seed(1)
    x, residual, dy = (torch.randn(T, d, device="cuda:0", generator=gen).to(layer.x.dtype) for _ in range(3))
    block = Fp8Block(layer.desc, torch.ones(d, device="cuda:0", dtype=layer.x.dtype), layer.w_inter, layer.w_intra, layer.w1, layer.w2)

    def step16():
        layer.forward()
        layer.backward()

    def step8():
        block.forward(x, residual)
        block.backward(dy)

    def pack():
        block.pack_weights(layer.w1, layer.w2)

    def us(step, times=40):
        start, stop = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        start.record()
        for _ in range(times):
            step()
        stop.record()
        torch.cuda.synchronize()
        return start.elapsed_time(stop) / times * 1e3

    steps = (step16, step8, pack)
    for step in steps:
        us(step, 10)
    t16, t8, t_pack = (sorted(t)[2] for t in zip(*[[us(step) for step in steps] for _ in range(5)]))     # in turn, medians of five
    mib = lambda *tensors: sum(t.numel() * t.element_size() for t in tensors) / 2 ** 20      # noqa: E731
    print(f"{cfg.name}, a training step: 16-bit layer {t16:.0f} us, 8-bit block with its norm {t8:.0f} us, "
          f"and {t_pack:.0f} us after every optimizer step to pack its weights")
    print(f"kept from the forward to the backward pass: {mib(layer.buf.xe, layer.h_save, layer.pre_save):.0f} MiB in 16 bits, "
          f"{block.kept_bytes() / 2 ** 20:.0f} MiB in 8")
    print(f"while the backward pass runs: {mib(layer.bwd.dye, layer.bwd.dxe, layer.bwd_workspace):.0f} MiB in 16 bits, "
          f"{block.scratch.nbytes() / 2 ** 20:.0f} MiB in 8, which a stack of blocks shares; packed weights beside the 16-bit ones: {block.packed_bytes() / 2 ** 20:.0f} MiB")
    block.close()
    layer.close()


if __name__ == "__main__":
    main()
