"""An expert layer without dropped tokens and its training step: every token reaches its k experts, whose rows lie sorted by expert instead of in buffers of a
fixed capacity.

    logits of x (fp32), k experts a token with their weights, pairs sorted by expert, tokens' rows moved there, up-projection with bias and activation,
    down-projection with bias, weighted return, added to the residual stream

the gradients of all of it, with a load-balancing term, and an AdamW step over the experts and the router.  Marshalling only: every step is a library call, no tensor is
allocated after construction (but the value of loss()), and nothing depends on the host: forward, backward and step can be captured into a graph.

    python -m paper_2212_05191_amd.sorted_block     # a training step at the base layer's size, timed, beside the layer with capacity buffers
"""
from __future__ import annotations

import torch

from . import binding as B


class SortedBlock:
    """w_router[N, d], w1[N, F, d], b1[N, F], w2[N, d, F], b2[N, d] in one storage type, for T tokens and k experts each.  The parameters are used, and updated by step(), in
    place.  normalize: weights that add up to one; balance: alpha of the load-balancing term alpha N sum_e f_e P_e; bias[N] float32 (or None) is added to the logits, -inf
    shuts an expert off.  optimizer: bits of AdamW's states (32 or 8), or None.  16-bit parameters have 32-bit masters, from which step() writes them: whoever loads others (a
    checkpoint) calls take_parameters() afterwards, or the next step undoes it."""

    def __init__(self, T, k, w_router, w1, b1, w2, b2, act="gelu", normalize=True, bias=None, balance=0.01, training=True, optimizer=None, weight_decay=0.1, seed=0):
        N, F, d = w1.shape
        st, dev = w1.dtype, w1.device
        code = B._dtype_code(w1)
        rows = T * k
        self.T, self.k, self.N = T, k, N
        self.normalize, self.bias, self.balance = normalize, bias, float(balance)
        self.w_router, self.w1, self.b1, self.w2, self.b2 = w_router, w1, b1, w2, b2
        self.desc = B.make_desc(T, d, F, N, 1, 1, code, act if act != "none" else "relu")   # the router's logits: N columns, and one of zeros
        self.ctx = B.Ctx(self.desc)

        def new(*shape, dtype=st):
            return torch.zeros(shape, dtype=dtype, device=dev)

        i32, f32 = torch.int32, torch.float32
        self.no_column = new(1, d)
        self.logits, self.logits0 = new(T, N, dtype=f32), new(T, 1, dtype=f32)
        self.idx, self.weight, self.p_sum = new(T, k, dtype=i32), new(T, k, dtype=f32), new(N, dtype=f32)
        self.count, self.start, self.pos, self.source = new(N, dtype=i32), new(N + 1, dtype=i32), new(T, k, dtype=i32), new(rows, dtype=i32)
        self.xs, self.h, self.ys, self.y = new(rows, d), new(rows, F), new(rows, d), new(T, d)
        self.pre = new(rows, F) if training and act != "none" else None
        self.up = B.make_linear_args(self.xs, w1, self.h, bias=b1, act=act, start=self.start, pre=self.pre)
        self.down = B.make_linear_args(self.h, w2, self.ys, bias=b2, start=self.start)
        nbytes = max(B.smile_topk_workspace_bytes(T, N), B.smile_sort_experts_workspace_bytes(T, k, N))
        if training:
            self.dys, self.dh, self.dxs, self.dx = new(rows, d), new(rows, F), new(rows, d), new(T, d)
            self.dweight, self.dlogits, self.dlogits0 = new(T, k, dtype=f32), new(T, N, dtype=f32), new(T, 1, dtype=f32)
            self.dw_router, self.no_dw = new(N, d, dtype=f32), new(1, d, dtype=f32)
            self.dw1, self.db1, self.dw2, self.db2 = new(N, F, d), new(N, F), new(N, d, F), new(N, d)
            self.no_slot, self.no_group = torch.full((T,), -1, dtype=i32, device=dev), new(T, dtype=i32)
            self.ddown = B.make_linear_backward_args(self.dys, self.h, w2, dx=self.dh, dw=self.dw2, dbias=self.db2, start=self.start)
            self.dup = B.make_linear_backward_args(self.dh, self.xs, w1, dx=self.dxs, dw=self.dw1, dbias=self.db1, pre=self.pre, act=act, start=self.start)
            nbytes = max(nbytes, B.smile_backward_workspace_bytes(self.desc), *(B.smile_linear_backward_workspace_bytes(a) for a in (self.ddown, self.dup)))
        self.workspace = new(nbytes, dtype=torch.uint8)
        self.optimizers = []
        if training and optimizer:
            experts = [(w1, self.dw1, True), (b1, self.db1, False), (w2, self.dw2, True), (b2, self.db2, False)]
            for i, group in enumerate((experts, [(w_router, self.dw_router, True)])):     # the router's gradient is fp32 whatever the storage type
                tensors = [self._states(p, g, optimizer, weight_decay if decays else 0.0) for p, g, decays in group]
                self.optimizers.append((B.AdamW(tensors, seed=seed + i), tensors, new(1, dtype=i32)))

    @staticmethod
    def _states(param, grad, bits, weight_decay):
        n, dev = param.numel(), param.device
        blocks = -(-n // 128)
        master = param.float().view(-1) if param.dtype != torch.float32 else None
        state = dict(param=param.view(-1), grad=grad.view(-1), master=master, weight_decay=weight_decay)
        if bits == 8:
            return {**state, **{name: torch.zeros(blocks * size, dtype=torch.uint8, device=dev) for name, size in (("m", 128), ("v", 128), ("m_scale", 1), ("v_scale", 1))}}
        return {**state, "m": torch.zeros(n, device=dev), "v": torch.zeros(n, device=dev)}

    def forward(self, x, residual=None, stream=None):
        """x[T, d] -> y[T, d]: the experts' weighted sum, added to the residual stream if that is given."""
        B.smile_gate_logits(self.ctx, x, self.w_router, self.no_column, self.logits, self.logits0, stream)
        B.smile_topk(self.logits, self.idx, self.weight, bias=self.bias, normalize=self.normalize, p_sum=self.p_sum, workspace=self.workspace, stream=stream)
        B.smile_sort_experts(self.idx, self.count, self.start, self.pos, self.source, self.workspace, stream)
        B.smile_sorted_dispatch(x, self.pos, self.xs, stream)
        B.smile_linear(self.up, stream)
        B.smile_linear(self.down, stream)
        B.smile_sorted_combine(self.ys, self.pos, self.y, weight=self.weight, residual=residual, stream=stream)
        return self.y

    def loss(self):
        """The load-balancing term of the last forward pass, on the device."""
        return self.balance * self.N / (self.k * float(self.T) ** 2) * (self.count.float() * self.p_sum).sum()

    def backward(self, x, dy, dloss=1.0, stream=None):
        """dy[T, d]: gradient of y (and that of the residual), dloss: of the load-balancing term.  Gradients: dx, dw_router, dw1, db1, dw2, db2."""
        T, ctx = self.T, self.ctx
        B.smile_sorted_combine_backward(dy, self.ys, self.pos, self.weight, self.dys, self.dweight, stream)
        B.smile_linear_backward(self.ddown, self.workspace, stream)
        B.smile_linear_backward(self.dup, self.workspace, stream)
        B.smile_topk_backward(self.logits, self.idx, self.dweight, self.dlogits, bias=self.bias, normalize=self.normalize, count=self.count,
                              coef=dloss * self.balance * self.N / (self.k * float(T) ** 2), stream=stream)
        B.smile_gate_weights_backward(ctx, x, self.dlogits, self.dlogits0, self.dw_router, self.no_dw, self.workspace, stream)
        # through the router (no token has a row of a capacity buffer here), then through the sorted rows
        B.smile_dispatch_backward(ctx, self.dxs, self.no_group, self.no_group, self.no_slot, self.dlogits, self.dlogits0, self.w_router, self.no_column, self.dx, stream)
        B.smile_sorted_combine(self.dxs, self.pos, self.dx, residual=self.dx, stream=stream)
        return self.dx

    def step(self, lr, stream=None):
        """An AdamW step with the gradients of the last backward pass; lr[1] float32 on the device."""
        for opt, _, count in self.optimizers:
            B.smile_adamw(opt, lr, count, stream)

    def take_parameters(self, new_states=False):
        """The masters from the parameters as they are now; new_states: moments and the count of steps from zero too, as at construction."""
        for _, tensors, count in self.optimizers:
            for t in tensors:
                if t["master"] is not None:
                    t["master"].copy_(t["param"])
                if new_states:
                    for name in ("m", "v", "m_scale", "v_scale"):
                        if name in t:
                            t[name].zero_()
            if new_states:
                count.zero_()

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
    T, d, N, F = cfg.T, cfg.d_model, cfg.N, cfg.d_ff
    st, gen = layer.x.dtype, torch.Generator(device="cuda:0").manual_seed(1)
    normal = lambda *shape, std=1.0: (std * torch.randn(*shape, device="cuda:0", generator=gen)).to(st)      # noqa: E731
    x, residual, dy, lr = normal(T, d), normal(T, d), normal(T, d), torch.full((1,), 1e-4, device="cuda:0")
    blocks = [SortedBlock(T, k, normal(N, d, std=0.02), layer.w1.clone(), normal(N, F, std=0.02), layer.w2.clone(), normal(N, d, std=0.02), optimizer=8) for k in (1, 2)]

    def step16():
        layer.forward()
        layer.backward()

    def pass_of(block):
        def run():
            block.forward(x, residual)
            block.backward(x, dy)
        return run

    def us(step, times=40):
        start, stop = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        start.record()
        for _ in range(times):
            step()
        stop.record()
        torch.cuda.synchronize()
        return start.elapsed_time(stop) / times * 1e3

    steps = [step16, *(pass_of(b) for b in blocks), lambda: blocks[0].step(lr)]
    for step in steps:
        us(step, 10)
    t16, one, two, opt = (sorted(t)[2] for t in zip(*[[us(step) for step in steps] for _ in range(5)]))      # in turn, medians of five
    print(f"{cfg.name}, forward and backward: layer with capacity buffers and one expert a token {t16:.0f} us; sorted, with biases, one expert {one:.0f} us, two {two:.0f} us; "
          f"AdamW step with 8-bit states {opt:.0f} us")
    for b in blocks:
        b.close()
    layer.close()


if __name__ == "__main__":
    main()
