"""Thin ctypes binding of libsmile (include/smile.h): argument marshalling only.

Every step of the layer runs in the HIP kernels of the library; PyTorch is used
for device memory (tensor.data_ptr()) and the current stream.  There is no
fallback: if the built library is missing, load() raises.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsmile.so")
_lib = None

DTYPE = {"f32": 0, "bf16": 1, "f16": 2}
ACT = {"relu": 0, "gelu": 1, "none": 2}   # "none": products of 8-bit operands and of sorted or dense rows only

OK, INVALID_ARG, BAD_SHAPE, UNSUPPORTED, WORKSPACE, HIP_ERROR = range(6)


class SmileError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} (status {status})")


class LayerDesc(C.Structure):
    _fields_ = [("T", C.c_int32), ("d_model", C.c_int32), ("d_ff", C.c_int32), ("n_groups", C.c_int32),
                ("m_local", C.c_int32), ("capacity", C.c_int32), ("dtype", C.c_int32), ("act", C.c_int32),
                ("alpha", C.c_float), ("beta", C.c_float), ("group_capacity", C.c_int32)]


class LayerIO(C.Structure):
    _fields_ = [(k, C.c_void_p) for k in (
        "x", "w_inter", "w_intra", "w1", "b1", "w2", "b2", "bias_inter", "bias_intra",
        "logits_inter", "logits_intra", "group_idx", "local_idx", "pos_in_group", "slot",
        "gate", "p_top", "q_top", "group_count", "local_count", "expert_count", "kept_count",
        "p_sum", "q_sum", "xe", "ye", "y", "loss3", "prof_up_start", "prof_up_stop", "h_save", "pre_save")]


class BackwardIO(C.Structure):
    _fields_ = [(k, C.c_void_p) for k in (
        "x", "w_inter", "w_intra", "w1", "w2", "bias_inter", "bias_intra",
        "logits_inter", "logits_intra", "group_idx", "local_idx", "slot", "gate",
        "group_count", "local_count", "kept_count", "xe", "ye", "h", "pre", "dy",
        "dye", "dgate", "dlp", "dlq", "dxe", "dx", "dw_inter", "dw_intra", "dw1", "dw2")]


class Fp8GemmArgs(C.Structure):
    _fields_ = [(k, C.c_int32) for k in ("N", "C", "K", "Nout", "dtype", "act")] + [(k, C.c_void_p) for k in (
        "x8", "x_scale", "w8", "w_scale", "bias", "rows", "y", "y8", "y_scale", "pre8", "pre_scale", "grad8", "grad_scale")]


class LinearArgs(C.Structure):
    _fields_ = [(k, C.c_int32) for k in ("N", "rows", "K", "F", "dtype", "act")] + [(k, C.c_void_p) for k in (
        "x", "w", "bias", "residual", "start", "y", "pre")]


class LinearBackwardArgs(C.Structure):
    _fields_ = [(k, C.c_int32) for k in ("N", "rows", "K", "F", "dtype", "act")] + [(k, C.c_void_p) for k in (
        "dy", "x", "w", "pre", "start", "dx", "dw", "dbias")]


class AdamWTensor(C.Structure):
    _fields_ = [(k, C.c_void_p) for k in ("param", "grad", "master", "m", "v", "m_scale", "v_scale")] + [("n", C.c_int64), ("weight_decay", C.c_float)]


class AdamWArgs(C.Structure):
    _fields_ = [(k, C.c_int32) for k in ("tensors", "dtype", "grad_dtype", "state_bits", "has_master", "seed")] + [
        (k, C.c_double) for k in ("beta1", "beta2", "eps")] + [("chunks", C.c_int64)]


EXPORTS = (
    "smile_status_string", "smile_version", "smile_capacity", "smile_validate_desc", "smile_workspace_bytes",
    "smile_create", "smile_create_with_workspace", "smile_destroy", "smile_gate_logits", "smile_route_bilevel",
    "smile_route_bilevel_static", "smile_kernel_timing", "smile_kernel_timing_count", "smile_kernel_timing_name",
    "smile_dispatch", "smile_dispatch_hop1", "smile_dispatch_hop2", "smile_expert_ffn", "smile_expert_ffn_up", "smile_expert_ffn_down", "smile_expert_ffn_up_timed", "smile_combine", "smile_aux_loss", "smile_layer_forward",
    "smile_backward_workspace_bytes", "smile_combine_backward", "smile_route_backward", "smile_expert_ffn_backward",
    "smile_dispatch_backward", "smile_gate_weights_backward", "smile_layer_backward",
    "smile_fp8_pitch", "smile_fp8_scale_pitch", "smile_rms_norm", "smile_rms_norm_backward_workspace_bytes",
    "smile_rms_norm_backward", "smile_fp8_pack_rows", "smile_fp8_unpack_rows", "smile_fp8_pack_weights",
    "smile_fp8_dispatch", "smile_fp8_gemm", "smile_fp8_weight_grad_workspace_bytes", "smile_fp8_weight_grad",
    "smile_topk_workspace_bytes", "smile_topk", "smile_topk_backward", "smile_sort_experts_workspace_bytes", "smile_sort_experts",
    "smile_sorted_dispatch", "smile_sorted_combine", "smile_sorted_combine_backward", "smile_linear",
    "smile_linear_backward_workspace_bytes", "smile_linear_backward", "smile_adamw_plan_bytes", "smile_adamw_plan", "smile_adamw",
    "smile_adamw_unpack_states",
)


def load() -> C.CDLL:
    """Load libsmile.so built in-tree by paper_2212_05191_amd.build; raise if it is not there."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2212_05191_amd.build` "
                           "(there is no CPU fallback)")
    lib = C.CDLL(LIB_PATH)
    vp, i32 = C.c_void_p, C.c_int32
    lib.smile_status_string.restype = C.c_char_p
    lib.smile_status_string.argtypes = [i32]
    lib.smile_version.restype = C.c_char_p
    lib.smile_capacity.restype = i32
    lib.smile_capacity.argtypes = [i32, i32, C.c_double]
    lib.smile_validate_desc.argtypes = [C.POINTER(LayerDesc)]
    lib.smile_workspace_bytes.argtypes = [C.POINTER(LayerDesc), C.POINTER(C.c_size_t)]
    lib.smile_create.argtypes = [C.POINTER(LayerDesc), C.POINTER(vp)]
    lib.smile_create_with_workspace.argtypes = [C.POINTER(LayerDesc), vp, C.c_size_t, C.POINTER(vp)]
    lib.smile_destroy.argtypes = [vp]
    lib.smile_gate_logits.argtypes = [vp] * 7
    lib.smile_kernel_timing.argtypes = [vp, C.POINTER(vp), i32]
    lib.smile_kernel_timing_count.argtypes = [vp]
    lib.smile_kernel_timing_count.restype = i32
    lib.smile_kernel_timing_name.argtypes = [vp, i32]
    lib.smile_route_bilevel.argtypes = [vp] * 19
    lib.smile_route_bilevel_static.argtypes = [C.POINTER(LayerDesc)] + [vp] * 18
    lib.smile_dispatch.argtypes = [vp] * 7
    lib.smile_dispatch_hop1.argtypes = [vp, vp, vp, vp, i32, vp, vp]
    lib.smile_dispatch_hop2.argtypes = [vp, vp, vp, vp, vp, vp, i32, vp, vp]
    lib.smile_expert_ffn.argtypes = [vp] * 9
    lib.smile_expert_ffn_up.argtypes = [vp] * 6
    lib.smile_expert_ffn_down.argtypes = [vp] * 6
    lib.smile_expert_ffn_up_timed.argtypes = [vp] * 8
    lib.smile_combine.argtypes = [vp] * 8
    lib.smile_aux_loss.argtypes = [vp] * 7
    lib.smile_layer_forward.argtypes = [vp, C.POINTER(LayerIO), vp]
    lib.smile_backward_workspace_bytes.argtypes = [C.POINTER(LayerDesc), C.POINTER(C.c_size_t)]
    lib.smile_combine_backward.argtypes = [vp] * 10
    lib.smile_route_backward.argtypes = [vp] * 10 + [C.c_float, vp, vp, vp]
    lib.smile_expert_ffn_backward.argtypes = [vp] * 12 + [C.c_size_t, vp]
    lib.smile_dispatch_backward.argtypes = [vp] * 11
    lib.smile_gate_weights_backward.argtypes = [vp] * 7 + [C.c_size_t, vp]
    lib.smile_layer_backward.argtypes = [vp, C.POINTER(BackwardIO), C.c_float, vp, C.c_size_t, vp]
    sz = C.POINTER(C.c_size_t)
    lib.smile_fp8_pitch.argtypes = [i32]
    lib.smile_fp8_scale_pitch.argtypes = [i32]
    lib.smile_rms_norm.argtypes = [i32] * 3 + [vp] * 3 + [C.c_float] + [vp] * 6
    lib.smile_rms_norm_backward_workspace_bytes.argtypes = [i32, i32, sz]
    lib.smile_rms_norm_backward.argtypes = [i32] * 3 + [vp] * 8 + [C.c_size_t, vp]
    lib.smile_fp8_pack_rows.argtypes = [i32] * 4 + [vp] * 5
    lib.smile_fp8_unpack_rows.argtypes = [i32] * 4 + [vp] * 5
    lib.smile_fp8_pack_weights.argtypes = [i32] * 4 + [vp] * 6
    lib.smile_fp8_dispatch.argtypes = [vp] * 9
    lib.smile_fp8_gemm.argtypes = [C.POINTER(Fp8GemmArgs), vp]
    lib.smile_fp8_weight_grad_workspace_bytes.argtypes = [i32] * 4 + [sz]
    lib.smile_fp8_weight_grad.argtypes = [i32] * 5 + [vp] * 6 + [C.c_size_t, vp]
    size = C.c_size_t
    lib.smile_topk_workspace_bytes.argtypes = [i32, i32, sz]
    lib.smile_topk.argtypes = [i32] * 4 + [vp] * 6 + [size, vp]
    lib.smile_topk_backward.argtypes = [i32] * 4 + [vp] * 5 + [C.c_float, vp, vp]
    lib.smile_sort_experts_workspace_bytes.argtypes = [i32] * 3 + [sz]
    lib.smile_sort_experts.argtypes = [i32] * 3 + [vp] * 6 + [size, vp]
    lib.smile_sorted_dispatch.argtypes = [i32] * 5 + [vp] * 4
    lib.smile_sorted_combine.argtypes = [i32] * 5 + [vp] * 6
    lib.smile_sorted_combine_backward.argtypes = [i32] * 5 + [vp] * 7
    lib.smile_linear.argtypes = [C.POINTER(LinearArgs), vp]
    lib.smile_linear_backward_workspace_bytes.argtypes = [C.POINTER(LinearBackwardArgs), sz]
    lib.smile_linear_backward.argtypes = [C.POINTER(LinearBackwardArgs), vp, size, vp]
    lib.smile_adamw_plan_bytes.argtypes = [C.POINTER(AdamWArgs), C.POINTER(AdamWTensor), sz]
    lib.smile_adamw_plan.argtypes = [C.POINTER(AdamWArgs), C.POINTER(AdamWTensor), vp, size]
    lib.smile_adamw.argtypes = [C.POINTER(AdamWArgs), vp, size, vp, vp, vp]
    lib.smile_adamw_unpack_states.argtypes = [C.c_int64, i32] + [vp] * 7
    for name in EXPORTS[3:]:
        getattr(lib, name).restype = i32
    lib.smile_kernel_timing_name.restype = C.c_char_p
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load().smile_status_string(int(status)).decode()


def version() -> str:
    return load().smile_version().decode()


def smile_capacity(T: int, N: int, capacity_factor: float) -> int:
    return int(load().smile_capacity(int(T), int(N), float(capacity_factor)))


def make_desc(T, d_model, d_ff, n_groups, m_local, capacity, dtype="bf16", act="gelu",
              alpha=0.005, beta=0.005, group_capacity=0) -> LayerDesc:
    return LayerDesc(int(T), int(d_model), int(d_ff), int(n_groups), int(m_local), int(capacity),
                     DTYPE[dtype] if isinstance(dtype, str) else int(dtype),
                     ACT[act] if isinstance(act, str) else int(act), float(alpha), float(beta), int(group_capacity))


def smile_validate_desc(desc: LayerDesc) -> int:
    return int(load().smile_validate_desc(C.byref(desc)))


def smile_workspace_bytes(desc: LayerDesc) -> int:
    out = C.c_size_t(0)
    st = load().smile_workspace_bytes(C.byref(desc), C.byref(out))
    if st != OK:
        raise SmileError(st, "smile_workspace_bytes")
    return int(out.value)


def _ptr(t):
    """Device pointer of a torch tensor (None -> NULL); ints pass through."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    assert t.is_contiguous(), "tensors must be dense row-major"
    return t.data_ptr()


_raw_stream = None


def _stream(stream):
    if stream is None:
        global _raw_stream
        if _raw_stream is None:
            import torch
            # the handle itself: building a torch Stream object for it costs more than a small launch
            raw, device = torch._C._cuda_getCurrentRawStream, torch.cuda.current_device
            _raw_stream = lambda: raw(device())      # noqa: E731
        return _raw_stream()
    return stream if isinstance(stream, int) else stream.cuda_stream


def _check(st: int, where: str):
    if st != OK:
        raise SmileError(int(st), where)


class Ctx:
    """Owner of a smile_ctx.  workspace=None: the library allocates; else a uint8 torch tensor."""

    def __init__(self, desc: LayerDesc, workspace=None):
        self.desc = desc
        self._h = C.c_void_p(None)
        self._ws = workspace
        lib = load()
        if workspace is None:
            _check(lib.smile_create(C.byref(desc), C.byref(self._h)), "smile_create")
        else:
            nbytes = workspace.numel() * workspace.element_size()
            _check(lib.smile_create_with_workspace(C.byref(desc), workspace.data_ptr(), nbytes, C.byref(self._h)),
                   "smile_create_with_workspace")

    @property
    def handle(self):
        return self._h

    def close(self):
        if self._h:
            load().smile_destroy(self._h)
            self._h = C.c_void_p(None)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def smile_gate_logits(ctx: Ctx, x, w_inter, w_intra, logits_inter, logits_intra, stream=None):
    _check(load().smile_gate_logits(ctx.handle, _ptr(x), _ptr(w_inter), _ptr(w_intra), _ptr(logits_inter),
                                    _ptr(logits_intra), _stream(stream)), "smile_gate_logits")


def smile_route_bilevel(ctx: Ctx, logits_inter, logits_intra, bias_inter, bias_intra, group_idx, local_idx,
                        pos_in_group, slot, gate, p_top, q_top, group_count, local_count, expert_count,
                        kept_count, p_sum, q_sum, stream=None):
    _check(load().smile_route_bilevel(ctx.handle, _ptr(logits_inter), _ptr(logits_intra), _ptr(bias_inter),
                                      _ptr(bias_intra), _ptr(group_idx), _ptr(local_idx), _ptr(pos_in_group),
                                      _ptr(slot), _ptr(gate), _ptr(p_top), _ptr(q_top), _ptr(group_count),
                                      _ptr(local_count), _ptr(expert_count), _ptr(kept_count), _ptr(p_sum),
                                      _ptr(q_sum), _stream(stream)), "smile_route_bilevel")


def smile_route_bilevel_static(desc: LayerDesc, logits_inter, logits_intra, bias_inter, bias_intra, group_idx,
                               local_idx, pos_in_group, slot, gate, p_top, q_top, group_count, local_count,
                               expert_count, kept_count, p_sum, q_sum, stream=None):
    """smile_route_bilevel without a ctx: the scratch memory is a fixed array inside the library."""
    _check(load().smile_route_bilevel_static(C.byref(desc), _ptr(logits_inter), _ptr(logits_intra),
                                             _ptr(bias_inter), _ptr(bias_intra), _ptr(group_idx), _ptr(local_idx),
                                             _ptr(pos_in_group), _ptr(slot), _ptr(gate), _ptr(p_top), _ptr(q_top),
                                             _ptr(group_count), _ptr(local_count), _ptr(expert_count),
                                             _ptr(kept_count), _ptr(p_sum), _ptr(q_sum), _stream(stream)),
           "smile_route_bilevel_static")


def smile_dispatch(ctx: Ctx, x, group_idx, local_idx, slot, xe, stream=None):
    _check(load().smile_dispatch(ctx.handle, _ptr(x), _ptr(group_idx), _ptr(local_idx), _ptr(slot), _ptr(xe),
                                 _stream(stream)), "smile_dispatch")


def smile_dispatch_hop1(ctx: Ctx, x, group_idx, pos_in_group, group_rows, xg, stream=None):
    _check(load().smile_dispatch_hop1(ctx.handle, _ptr(x), _ptr(group_idx), _ptr(pos_in_group), int(group_rows),
                                      _ptr(xg), _stream(stream)), "smile_dispatch_hop1")


def smile_dispatch_hop2(ctx: Ctx, xg, group_idx, local_idx, pos_in_group, slot, group_rows, xe, stream=None):
    _check(load().smile_dispatch_hop2(ctx.handle, _ptr(xg), _ptr(group_idx), _ptr(local_idx), _ptr(pos_in_group),
                                      _ptr(slot), int(group_rows), _ptr(xe), _stream(stream)), "smile_dispatch_hop2")


def smile_expert_ffn(ctx: Ctx, xe, kept_count, w1, b1, w2, b2, ye, stream=None):
    _check(load().smile_expert_ffn(ctx.handle, _ptr(xe), _ptr(kept_count), _ptr(w1), _ptr(b1), _ptr(w2), _ptr(b2),
                                   _ptr(ye), _stream(stream)), "smile_expert_ffn")


def smile_expert_ffn_up(ctx: Ctx, xe, kept_count, w1, b1, stream=None):
    _check(load().smile_expert_ffn_up(ctx.handle, _ptr(xe), _ptr(kept_count), _ptr(w1), _ptr(b1),
                                      _stream(stream)), "smile_expert_ffn_up")


def smile_expert_ffn_down(ctx: Ctx, kept_count, w2, b2, ye, stream=None):
    _check(load().smile_expert_ffn_down(ctx.handle, _ptr(kept_count), _ptr(w2), _ptr(b2), _ptr(ye),
                                        _stream(stream)), "smile_expert_ffn_down")


def smile_combine(ctx: Ctx, ye, group_idx, local_idx, slot, gate, y, stream=None):
    _check(load().smile_combine(ctx.handle, _ptr(ye), _ptr(group_idx), _ptr(local_idx), _ptr(slot), _ptr(gate),
                                _ptr(y), _stream(stream)), "smile_combine")


def smile_aux_loss(ctx: Ctx, group_count, local_count, p_sum, q_sum, out3, stream=None):
    _check(load().smile_aux_loss(ctx.handle, _ptr(group_count), _ptr(local_count), _ptr(p_sum), _ptr(q_sum),
                                 _ptr(out3), _stream(stream)), "smile_aux_loss")


def smile_layer_forward(ctx: Ctx, io: LayerIO, stream=None):
    _check(load().smile_layer_forward(ctx.handle, C.byref(io), _stream(stream)), "smile_layer_forward")


def torch_dtype(dtype):
    """torch storage type of a desc.dtype code or name."""
    import torch
    code = DTYPE[dtype] if isinstance(dtype, str) else int(dtype)
    return {0: torch.float32, 1: torch.bfloat16, 2: torch.float16}[code]


# ------------------------------------------------------------------ backward pass

def smile_backward_workspace_bytes(desc: LayerDesc) -> int:
    out = C.c_size_t(0)
    _check(load().smile_backward_workspace_bytes(C.byref(desc), C.byref(out)), "smile_backward_workspace_bytes")
    return int(out.value)


def smile_combine_backward(ctx: Ctx, dy, ye, group_idx, local_idx, slot, gate, dye, dgate, stream=None):
    _check(load().smile_combine_backward(ctx.handle, _ptr(dy), _ptr(ye), _ptr(group_idx), _ptr(local_idx), _ptr(slot),
                                         _ptr(gate), _ptr(dye), _ptr(dgate), _stream(stream)), "smile_combine_backward")


def smile_route_backward(ctx: Ctx, logits_inter, logits_intra, bias_inter, bias_intra, group_idx, local_idx, dgate,
                         group_count, local_count, dloss, dlp, dlq, stream=None):
    _check(load().smile_route_backward(ctx.handle, _ptr(logits_inter), _ptr(logits_intra), _ptr(bias_inter),
                                       _ptr(bias_intra), _ptr(group_idx), _ptr(local_idx), _ptr(dgate),
                                       _ptr(group_count), _ptr(local_count), float(dloss), _ptr(dlp), _ptr(dlq),
                                       _stream(stream)), "smile_route_backward")


def smile_expert_ffn_backward(ctx: Ctx, xe, kept_count, w1, w2, dye, dxe, dw1, dw2, workspace, h=None, pre=None,
                              stream=None):
    _check(load().smile_expert_ffn_backward(ctx.handle, _ptr(xe), _ptr(kept_count), _ptr(w1), _ptr(w2), _ptr(dye),
                                            _ptr(h), _ptr(pre), _ptr(dxe), _ptr(dw1), _ptr(dw2), _ptr(workspace),
                                            workspace.numel() * workspace.element_size(), _stream(stream)),
           "smile_expert_ffn_backward")


def smile_dispatch_backward(ctx: Ctx, dxe, group_idx, local_idx, slot, dlp, dlq, w_inter, w_intra, dx, stream=None):
    _check(load().smile_dispatch_backward(ctx.handle, _ptr(dxe), _ptr(group_idx), _ptr(local_idx), _ptr(slot),
                                          _ptr(dlp), _ptr(dlq), _ptr(w_inter), _ptr(w_intra), _ptr(dx),
                                          _stream(stream)), "smile_dispatch_backward")


def smile_gate_weights_backward(ctx: Ctx, x, dlp, dlq, dw_inter, dw_intra, workspace, stream=None):
    _check(load().smile_gate_weights_backward(ctx.handle, _ptr(x), _ptr(dlp), _ptr(dlq), _ptr(dw_inter),
                                              _ptr(dw_intra), _ptr(workspace),
                                              workspace.numel() * workspace.element_size(), _stream(stream)),
           "smile_gate_weights_backward")


def smile_layer_backward(ctx: Ctx, io: BackwardIO, dloss, workspace, stream=None):
    _check(load().smile_layer_backward(ctx.handle, C.byref(io), float(dloss), _ptr(workspace),
                                       workspace.numel() * workspace.element_size(), _stream(stream)),
           "smile_layer_backward")


@dataclass
class BackwardBuffers:
    """Intermediates and results of one backward pass as torch tensors on the GPU."""
    dye: object
    dgate: object
    dlp: object
    dlq: object
    dxe: object
    dx: object
    dw_inter: object
    dw_intra: object
    dw1: object
    dw2: object


def alloc_backward_buffers(desc: LayerDesc, device="cuda:0") -> BackwardBuffers:
    import torch
    T, d, F, n, m, Cap = desc.T, desc.d_model, desc.d_ff, desc.n_groups, desc.m_local, desc.capacity
    N = n * m
    st = torch_dtype(desc.dtype)
    f32 = torch.float32

    def e(shape, dt):
        return torch.empty(shape, dtype=dt, device=device)

    return BackwardBuffers(e((N, Cap, d), st), e((T,), f32), e((T, n), f32), e((T, m), f32), e((N, Cap, d), st),
                           e((T, d), st), e((n, d), f32), e((m, d), f32), e((N, F, d), st), e((N, d, F), st))


def make_backward_io(x, w_inter, w_intra, w1, w2, fwd: "LayerBuffers", dy, bwd: BackwardBuffers, bias_inter=None,
                     bias_intra=None, h=None, pre=None) -> BackwardIO:
    io = BackwardIO()
    for k, v in dict(x=x, w_inter=w_inter, w_intra=w_intra, w1=w1, w2=w2, bias_inter=bias_inter,
                     bias_intra=bias_intra, dy=dy, h=h, pre=pre).items():
        setattr(io, k, _ptr(v))
    for k in ("logits_inter", "logits_intra", "group_idx", "local_idx", "slot", "gate", "group_count", "local_count",
              "kept_count", "xe", "ye"):
        setattr(io, k, _ptr(getattr(fwd, k)))
    for k, v in bwd.__dict__.items():
        setattr(io, k, _ptr(v))
    return io


# ------------------------------------------------------------------ operators in 8 bits

_CODES = {}


def _dtype_code(t) -> int:
    """DTYPE code of a torch tensor's element type."""
    if not _CODES:
        import torch
        _CODES.update({torch.float32: 0, torch.bfloat16: 1, torch.float16: 2})
    code = _CODES.get(t.dtype)
    if code is None:
        raise TypeError(f"storage type {t.dtype} is none of float32, bfloat16, float16")
    return code


def smile_fp8_pitch(K: int) -> int:
    return int(load().smile_fp8_pitch(int(K)))


def smile_fp8_scale_pitch(rows: int) -> int:
    return int(load().smile_fp8_scale_pitch(int(rows)))


def _has_shape(name, t, shape):
    if t is not None and t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, not {tuple(shape)}")


def _check_codes(name, codes, scales, N, rows, K, scaled):
    """Codes [N][rows][K up to a multiple of 128] and scales [N][blocks of K][`scaled` up to a multiple of 16]: the shapes that
    the library takes for granted."""
    if codes is None or scales is None:
        raise ValueError(f"{name}: codes and scales go together")
    blocks = -(-K // 128)
    _has_shape(name, codes, (N, rows, blocks * 128))
    _has_shape(name + " scales", scales, (N, blocks, -(-scaled // 16) * 16))
    for t in (codes, scales):
        if t.element_size() != 1:
            raise TypeError(f"{name} is {t.dtype}, of more than a byte")


def _check_rows8(name, codes, scales, N, rows, K):
    _check_codes(name, codes, scales, N, rows, K, rows)


def _check_weights8(name, codes, scales, N, Nout, K):
    _check_codes(name, codes, scales, N, Nout, K, -(-Nout // 128))


def _check_like(name, t, shape, dtype):
    if t is not None and (t.shape != shape or t.dtype != dtype):
        _has_shape(name, t, shape)
        raise TypeError(f"{name} is {t.dtype}, not {dtype}")


def _f32():
    if not _CODES:
        import torch
        _CODES.update({torch.float32: 0, torch.bfloat16: 1, torch.float16: 2})
    return next(iter(_CODES))


def _check_counts(rows, N):
    if rows is not None:
        import torch
        _check_like("rows", rows, (N,), torch.int32)


def alloc_fp8_rows(N, rows, K, device="cuda:0"):
    """Codes and scales of 8-bit rows [N][rows][K], zeroed."""
    import torch
    pitch = smile_fp8_pitch(K)
    return (torch.zeros((N, rows, pitch), dtype=torch.uint8, device=device),
            torch.zeros((N, pitch // 128, smile_fp8_scale_pitch(rows)), dtype=torch.uint8, device=device))


def alloc_fp8_weights(N, Nout, K, device="cuda:0"):
    """Codes and scales of 8-bit weights [N][Nout][K], zeroed."""
    import torch
    pitch = smile_fp8_pitch(K)
    return (torch.zeros((N, Nout, pitch), dtype=torch.uint8, device=device),
            torch.zeros((N, pitch // 128, smile_fp8_scale_pitch(-(-Nout // 128))), dtype=torch.uint8, device=device))


def smile_rms_norm(x, residual, weight, eps, sum=None, y=None, y8=None, y8_scale=None, rstd=None, stream=None):
    """x[T, d] (+ residual, or None) -> sum, y, 8-bit y, rstd: whichever are given."""
    shape, dtype = x.shape, x.dtype
    T, d = shape
    code = _dtype_code(x)
    _check_like("residual", residual, shape, dtype)
    _check_like("weight", weight, (d,), dtype)
    _check_like("sum", sum, shape, dtype)
    _check_like("y", y, shape, dtype)
    if rstd is not None:
        _check_like("rstd", rstd, (T,), _f32())
    if y8 is not None:
        _check_rows8("y8", y8, y8_scale, 1, T, d)
    _check(load().smile_rms_norm(T, d, code, _ptr(x), _ptr(residual), _ptr(weight), float(eps), _ptr(sum), _ptr(y), _ptr(y8),
                                 _ptr(y8_scale), _ptr(rstd), _stream(stream)), "smile_rms_norm")


def smile_rms_norm_backward_workspace_bytes(T, d) -> int:
    out = C.c_size_t(0)
    _check(load().smile_rms_norm_backward_workspace_bytes(int(T), int(d), C.byref(out)), "smile_rms_norm_backward_workspace_bytes")
    return int(out.value)


def smile_rms_norm_backward(dy, s, weight, rstd, ds, dweight, workspace, dsum=None, stream=None):
    shape, dtype = dy.shape, dy.dtype
    T, d = shape
    code = _dtype_code(dy)
    _check_like("s", s, shape, dtype)
    _check_like("weight", weight, (d,), dtype)
    _check_like("ds", ds, shape, dtype)
    _check_like("dsum", dsum, shape, dtype)
    _check_like("rstd", rstd, (T,), _f32())
    _check_like("dweight", dweight, (d,), _f32())
    _check(load().smile_rms_norm_backward(T, d, code, _ptr(dy), _ptr(dsum), _ptr(s), _ptr(weight), _ptr(rstd), _ptr(ds),
                                          _ptr(dweight), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                          _stream(stream)), "smile_rms_norm_backward")


def _grouped(t):
    """(N, C, K) of a tensor [N, C, K] or [C, K]"""
    shape = t.shape
    return shape if len(shape) == 3 else (1, *shape)


def smile_fp8_pack_rows(src, codes, scales, rows=None, stream=None):
    """src[N, C, K] (or [C, K]) to 8-bit rows; only the first rows[e] of each group."""
    N, cap, K = _grouped(src)
    _check_rows8("codes", codes, scales, N, cap, K)
    _check_counts(rows, N)
    _check(load().smile_fp8_pack_rows(N, cap, K, _dtype_code(src), _ptr(src), _ptr(rows), _ptr(codes), _ptr(scales),
                                      _stream(stream)), "smile_fp8_pack_rows")


def smile_fp8_unpack_rows(codes, scales, dst, rows=None, stream=None):
    """8-bit rows to dst[N, C, K] (or [C, K])."""
    N, cap, K = _grouped(dst)
    _check_rows8("codes", codes, scales, N, cap, K)
    _check_counts(rows, N)
    _check(load().smile_fp8_unpack_rows(N, cap, K, _dtype_code(dst), _ptr(codes), _ptr(scales), _ptr(rows), _ptr(dst),
                                        _stream(stream)), "smile_fp8_unpack_rows")


def smile_fp8_pack_weights(w, codes, scales, codes_t=None, scales_t=None, stream=None):
    """w[N, Nout, K] (or [Nout, K]) to 8-bit weights, and to their transposed form."""
    N, Nout, K = _grouped(w)
    _check_weights8("codes", codes, scales, N, Nout, K)
    if codes_t is not None:
        _check_weights8("codes_t", codes_t, scales_t, N, K, Nout)
    _check(load().smile_fp8_pack_weights(N, Nout, K, _dtype_code(w), _ptr(w), _ptr(codes), _ptr(scales), _ptr(codes_t),
                                         _ptr(scales_t), _stream(stream)), "smile_fp8_pack_weights")


def smile_fp8_dispatch(ctx: Ctx, x8, x_scale, group_idx, local_idx, slot, xe8, xe_scale, stream=None):
    import torch
    d = ctx.desc
    _check_rows8("x8", x8, x_scale, 1, d.T, d.d_model)
    _check_rows8("xe8", xe8, xe_scale, d.n_groups * d.m_local, d.capacity, d.d_model)
    for name, t in (("group_idx", group_idx), ("local_idx", local_idx), ("slot", slot)):
        _check_like(name, t, (d.T,), torch.int32)
    _check(load().smile_fp8_dispatch(ctx.handle, _ptr(x8), _ptr(x_scale), _ptr(group_idx), _ptr(local_idx), _ptr(slot), _ptr(xe8),
                                     _ptr(xe_scale), _stream(stream)), "smile_fp8_dispatch")


def make_fp8_gemm_args(x8, x_scale, w8, w_scale, K, Nout, rows=None, act="none", bias=None, y=None, y8=None, y_scale=None,
                       pre8=None, pre_scale=None, grad8=None, grad_scale=None, dtype=None) -> Fp8GemmArgs:
    """The argument block of smile_fp8_gemm; dtype is that of y and bias, and needed only where neither is given.  The block
    keeps the tensors alive."""
    N, cap = x8.shape[:2]
    _check_rows8("x8", x8, x_scale, N, cap, K)
    _check_weights8("w8", w8, w_scale, N, Nout, K)
    for name, codes, scales in (("y8", y8, y_scale), ("pre8", pre8, pre_scale), ("grad8", grad8, grad_scale)):
        if codes is not None:
            _check_rows8(name, codes, scales, N, cap, Nout)
    if y is not None and _grouped(y) != (N, cap, Nout):
        raise ValueError(f"y has shape {tuple(y.shape)}, not {(N, cap, Nout)}")
    if bias is not None and bias.numel() != N * Nout:
        raise ValueError(f"bias has shape {tuple(bias.shape)}, not {(N, Nout)}")
    _check_counts(rows, N)
    code = _dtype_code(y) if y is not None else _dtype_code(bias) if bias is not None else DTYPE[dtype or "bf16"]
    if bias is not None and _dtype_code(bias) != code:
        raise TypeError(f"bias is {bias.dtype}, of another storage type than y")
    args = Fp8GemmArgs(N, cap, int(K), int(Nout), code, ACT[act])
    tensors = dict(x8=x8, x_scale=x_scale, w8=w8, w_scale=w_scale, bias=bias, rows=rows, y=y, y8=y8, y_scale=y_scale, pre8=pre8,
                   pre_scale=pre_scale, grad8=grad8, grad_scale=grad_scale)
    for k, v in tensors.items():
        setattr(args, k, _ptr(v))
    args.tensors = tensors
    return args


def smile_fp8_gemm(args: Fp8GemmArgs, stream=None):
    _check(load().smile_fp8_gemm(C.byref(args), _stream(stream)), "smile_fp8_gemm")


def smile_fp8_weight_grad_workspace_bytes(N, cap, K, dtype) -> int:
    out = C.c_size_t(0)
    code = DTYPE[dtype] if isinstance(dtype, str) else int(dtype)
    _check(load().smile_fp8_weight_grad_workspace_bytes(int(N), int(cap), int(K), code, C.byref(out)),
           "smile_fp8_weight_grad_workspace_bytes")
    return int(out.value)


def smile_fp8_weight_grad(dy, x8, x_scale, dw, workspace, rows=None, stream=None):
    """dw[N, Nout, K] = dy[N, C, Nout]^T . (8-bit rows [N, C, K]) over the first rows[e] rows of each group."""
    N, cap, Nout = _grouped(dy)
    K = dw.shape[-1]
    if _grouped(dw) != (N, Nout, K):
        raise ValueError(f"dw has shape {tuple(dw.shape)}, not {(N, Nout, K)}")
    _check_rows8("x8", x8, x_scale, N, cap, K)
    if dw.dtype != dy.dtype:
        raise TypeError(f"dw is {dw.dtype}, dy {dy.dtype}")
    _check_counts(rows, N)
    _check(load().smile_fp8_weight_grad(N, cap, Nout, K, _dtype_code(dy), _ptr(dy), _ptr(x8), _ptr(x_scale), _ptr(rows), _ptr(dw),
                                        _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)),
           "smile_fp8_weight_grad")


# ------------------------------------------------------------------ a layer without dropped tokens, and its optimizer

def _nbytes(t):
    return 0 if t is None else t.numel() * t.element_size()


_int32 = _current_device = None     # torch's, once it is imported: looking them up costs as much as a check


def _i32():
    global _int32
    if _int32 is None:
        import torch
        _int32 = torch.int32
    return _int32


def _check_device(*tensors):
    """Tensors of the current device: a kernel would follow any other pointer blindly."""
    global _current_device
    if _current_device is None:
        import torch
        _current_device = torch.cuda.current_device
    here = _current_device()
    for t in tensors:
        if t is not None and t.get_device() != here:
            raise ValueError(f"a tensor is on {t.device}, the current device is cuda:{here}")


def smile_topk_workspace_bytes(T, N) -> int:
    out = C.c_size_t(0)
    _check(load().smile_topk_workspace_bytes(int(T), int(N), C.byref(out)), "smile_topk_workspace_bytes")
    return int(out.value)


def smile_topk(logits, idx, weight, bias=None, normalize=False, p_sum=None, workspace=None, stream=None):
    """logits[T, N] -> the k experts idx[T, k] of each token, their weights, and the column sums of the probabilities."""
    T, N = logits.shape
    k = idx.shape[-1]
    f32 = _f32()
    _check_like("logits", logits, (T, N), f32)
    _check_like("idx", idx, (T, k), _i32())
    _check_like("weight", weight, (T, k), f32)
    _check_like("bias", bias, (N,), f32)
    _check_like("p_sum", p_sum, (N,), f32)
    _check_device(logits, idx, weight, bias, p_sum, workspace)
    _check(load().smile_topk(T, N, k, int(bool(normalize)), _ptr(logits), _ptr(bias), _ptr(idx), _ptr(weight), _ptr(p_sum), _ptr(workspace),
                             _nbytes(workspace), _stream(stream)), "smile_topk")


def smile_topk_backward(logits, idx, dweight, dlogits, bias=None, normalize=False, count=None, coef=0.0, stream=None):
    """Gradient of the logits from that of the weights and coef * count for each column of p_sum."""
    T, N = logits.shape
    k = idx.shape[-1]
    f32 = _f32()
    _check_like("logits", logits, (T, N), f32)
    _check_like("idx", idx, (T, k), _i32())
    _check_like("dweight", dweight, (T, k), f32)
    _check_like("dlogits", dlogits, (T, N), f32)
    _check_like("bias", bias, (N,), f32)
    _check_like("count", count, (N,), _i32())
    _check_device(logits, idx, dweight, dlogits, bias, count)
    _check(load().smile_topk_backward(T, N, k, int(bool(normalize)), _ptr(logits), _ptr(bias), _ptr(idx), _ptr(dweight), _ptr(count), float(coef),
                                      _ptr(dlogits), _stream(stream)), "smile_topk_backward")


def smile_sort_experts_workspace_bytes(T, k, N) -> int:
    out = C.c_size_t(0)
    _check(load().smile_sort_experts_workspace_bytes(int(T), int(k), int(N), C.byref(out)), "smile_sort_experts_workspace_bytes")
    return int(out.value)


def smile_sort_experts(idx, count, start, pos, source, workspace=None, stream=None):
    """The pairs of idx[T, k] sorted by expert: count[N], start[N + 1], pos[T, k] (the pair's row or -1), source[T * k] (the row's pair or -1)."""
    T, k = idx.shape
    N, i32 = count.shape[0], _i32()
    for name, t, shape in (("idx", idx, (T, k)), ("count", count, (N,)), ("start", start, (N + 1,)), ("pos", pos, (T, k)), ("source", source, (T * k,))):
        _check_like(name, t, shape, i32)
    _check_device(idx, count, start, pos, source, workspace)
    _check(load().smile_sort_experts(T, k, N, _ptr(idx), _ptr(count), _ptr(start), _ptr(pos), _ptr(source), _ptr(workspace), _nbytes(workspace),
                                     _stream(stream)), "smile_sort_experts")


def _check_pairs(pos, T, weight=None, dweight=None):
    k = pos.shape[-1]
    _check_like("pos", pos, (T, k), _i32())
    _check_like("weight", weight, (T, k), _f32())
    _check_like("dweight", dweight, (T, k), _f32())
    return k


def smile_sorted_dispatch(x, pos, xs, stream=None):
    """Row t of x[T, d] to the rows pos[t, :] of xs[R, d]."""
    T, d = x.shape
    k, R = _check_pairs(pos, T), xs.shape[0]
    _check_like("xs", xs, (R, d), x.dtype)
    _check_device(x, pos, xs)
    _check(load().smile_sorted_dispatch(T, k, d, R, _dtype_code(x), _ptr(x), _ptr(pos), _ptr(xs), _stream(stream)), "smile_sorted_dispatch")


def smile_sorted_combine(ys, pos, y, weight=None, residual=None, stream=None):
    """y[T, d] = residual + the weighted sum of each token's rows of ys[R, d]."""
    (R, d), T = ys.shape, pos.shape[0]
    k = _check_pairs(pos, T, weight)
    _check_like("y", y, (T, d), ys.dtype)
    _check_like("residual", residual, (T, d), ys.dtype)
    _check_device(ys, pos, y, weight, residual)
    _check(load().smile_sorted_combine(T, k, d, R, _dtype_code(ys), _ptr(ys), _ptr(pos), _ptr(weight), _ptr(residual), _ptr(y), _stream(stream)),
           "smile_sorted_combine")


def smile_sorted_combine_backward(dy, ys, pos, weight, dys, dweight, stream=None):
    """Gradients of smile_sorted_combine: dys[R, d] and dweight[T, k] (ys and dweight None: without the latter)."""
    (T, d), R = dy.shape, dys.shape[0]
    k = _check_pairs(pos, T, weight, dweight)
    _check_like("ys", ys, (R, d), dy.dtype)
    _check_like("dys", dys, (R, d), dy.dtype)
    _check_device(dy, ys, pos, weight, dys, dweight)
    _check(load().smile_sorted_combine_backward(T, k, d, R, _dtype_code(dy), _ptr(dy), _ptr(ys), _ptr(pos), _ptr(weight), _ptr(dys), _ptr(dweight),
                                                _stream(stream)), "smile_sorted_combine_backward")


def _linear_shapes(x, w, start):
    rows, K = x.shape
    N, F = _grouped(w)[:2]
    if _grouped(w)[2] != K:
        raise ValueError(f"w has shape {tuple(w.shape)}, not {(N, F, K)}")
    if start is not None:
        _check_like("start", start, (N + 1,), _i32())
    return N, rows, K, F


def _like_grouped(name, t, shape, dtype):
    """t of a shape that may leave out a first extent of 1"""
    if t is not None and tuple(t.shape) != shape and not (shape[0] == 1 and tuple(t.shape) == shape[1:]):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, not {shape}")
    if t is not None and t.dtype != dtype:
        raise TypeError(f"{name} is {t.dtype}, not {dtype}")


def make_linear_args(x, w, y, bias=None, act="none", residual=None, start=None, pre=None) -> LinearArgs:
    """The argument block of smile_linear: x[rows, K], w[N, F, K] (or [F, K]), y[rows, F], bias[N, F], residual and pre like y, start[N + 1].  The block
    keeps the tensors alive."""
    N, rows, K, F = _linear_shapes(x, w, start)
    dtype = x.dtype
    _like_grouped("w", w, (N, F, K), dtype)
    _like_grouped("bias", bias, (N, F), dtype)
    for name, t in (("y", y), ("residual", residual), ("pre", pre)):
        _check_like(name, t, (rows, F), dtype)
    args = LinearArgs(N, rows, K, F, _dtype_code(x), ACT[act])
    tensors = dict(x=x, w=w, bias=bias, residual=residual, start=start, y=y, pre=pre)
    for name, t in tensors.items():
        setattr(args, name, _ptr(t))
    args.tensors = tensors
    return args


def smile_linear(args: LinearArgs, stream=None):
    _check_device(*args.tensors.values())
    _check(load().smile_linear(C.byref(args), _stream(stream)), "smile_linear")


def make_linear_backward_args(dy, x, w, dx=None, dw=None, dbias=None, pre=None, act="none", start=None) -> LinearBackwardArgs:
    """The argument block of smile_linear_backward; shapes as in make_linear_args.  x and w give the shapes and are always passed."""
    N, rows, K, F = _linear_shapes(x, w, start)
    dtype = dy.dtype
    for name, t, shape in (("dy", dy, (rows, F)), ("x", x, (rows, K)), ("pre", pre, (rows, F)), ("dx", dx, (rows, K))):
        _check_like(name, t, shape, dtype)
    for name, t, shape in (("w", w, (N, F, K)), ("dw", dw, (N, F, K)), ("dbias", dbias, (N, F))):
        _like_grouped(name, t, shape, dtype)
    args = LinearBackwardArgs(N, rows, K, F, _dtype_code(dy), ACT[act])
    tensors = dict(dy=dy, x=x, w=w, pre=pre, start=start, dx=dx, dw=dw, dbias=dbias)
    for name, t in tensors.items():
        setattr(args, name, _ptr(t))
    args.tensors = tensors
    return args


def smile_linear_backward_workspace_bytes(args: LinearBackwardArgs) -> int:
    out = C.c_size_t(0)
    _check(load().smile_linear_backward_workspace_bytes(C.byref(args), C.byref(out)), "smile_linear_backward_workspace_bytes")
    return int(out.value)


def smile_linear_backward(args: LinearBackwardArgs, workspace=None, stream=None):
    _check_device(*args.tensors.values(), workspace)
    _check(load().smile_linear_backward(C.byref(args), _ptr(workspace), _nbytes(workspace), _stream(stream)), "smile_linear_backward")


class AdamW:
    """The tensors of an optimizer step and its plan on their device.  tensors: dicts of param, grad, m, v, and master, m_scale, v_scale or None, all flat or of
    one shape, with weight_decay; they share their types.  States in uint8 (with scales) make an 8-bit optimizer, in float32 a 32-bit one; zeros are new states."""

    def __init__(self, tensors, beta1=0.9, beta2=0.999, eps=1e-8, seed=0):
        import torch
        first = tensors[0]
        eight = first["m"].dtype == torch.uint8
        state = torch.uint8 if eight else torch.float32
        self.tensors = [dict(t) for t in tensors]          # kept alive
        block = (AdamWTensor * len(tensors))()
        device = first["param"].device
        for i, t in enumerate(self.tensors):
            n = t["param"].numel()
            padded = -(-n // 128) * 128
            sizes = dict(param=n, grad=n, master=n, m=padded if eight else n, v=padded if eight else n, m_scale=padded // 128, v_scale=padded // 128)
            types = dict(param=first["param"].dtype, grad=first["grad"].dtype, master=torch.float32, m=state, v=state, m_scale=torch.uint8, v_scale=torch.uint8)
            for name, size in sizes.items():
                x = t.get(name)
                if (x is None) != (first.get(name) is None):
                    raise ValueError(f"{name} is given for some tensors only")
                if x is None:
                    continue
                if x.dtype != types[name]:
                    raise TypeError(f"{name} of tensor {i} is {x.dtype}, not {types[name]}")
                if x.device != device:
                    raise ValueError(f"{name} of tensor {i} is on {x.device}, not {device}")
                if x.numel() != size and not (name.endswith("_scale") and x.numel() >= size):
                    raise ValueError(f"{name} of tensor {i} has {x.numel()} elements, not {size}")
                setattr(block[i], name, _ptr(x))
            block[i].n, block[i].weight_decay = n, float(t.get("weight_decay", 0.0))
        self.args = AdamWArgs(len(tensors), _dtype_code(first["param"]), _dtype_code(first["grad"]), 8 if eight else 32,
                              int(first.get("master") is not None), int(seed), float(beta1), float(beta2), float(eps), 0)
        out = C.c_size_t(0)
        _check(load().smile_adamw_plan_bytes(C.byref(self.args), block, C.byref(out)), "smile_adamw_plan_bytes")
        host = torch.empty(out.value + 256, dtype=torch.uint8)
        at = -host.data_ptr() % 256
        host = host[at:at + out.value]
        _check(load().smile_adamw_plan(C.byref(self.args), block, host.data_ptr(), out.value), "smile_adamw_plan")
        self.plan = host.to(device)


def smile_adamw(opt: AdamW, lr, step, stream=None):
    """One step in place; lr[1] float32 and step[1] int32 on the device.  step is the number of steps made, and goes up by one."""
    _check_like("lr", lr, (1,), _f32())
    _check_like("step", step, (1,), _i32())
    _check_device(opt.plan, lr, step)
    _check(load().smile_adamw(C.byref(opt.args), opt.plan.data_ptr(), _nbytes(opt.plan), _ptr(lr), _ptr(step), _stream(stream)), "smile_adamw")


def smile_adamw_unpack_states(m, m_scale, v, v_scale, m_value, v_value, stream=None):
    """8-bit states (flat, of whole blocks) as values: float32 or bfloat16."""
    import torch
    n = m.numel()
    for name, t, size in (("m", m, n), ("v", v, n), ("m_value", m_value, n), ("v_value", v_value, n)):
        if t.numel() != size:
            raise ValueError(f"{name} has {t.numel()} elements, not {size}")
    for name, t in (("m", m), ("v", v), ("m_scale", m_scale), ("v_scale", v_scale)):
        if t.dtype != torch.uint8:
            raise TypeError(f"{name} is {t.dtype}, not {torch.uint8}")
    for name, t in (("m_scale", m_scale), ("v_scale", v_scale)):
        if t.numel() * 128 < n:
            raise ValueError(f"{name} has {t.numel()} elements, of {-(-n // 128)} blocks")
    if v_value.dtype != m_value.dtype:
        raise TypeError(f"v_value is {v_value.dtype}, not {m_value.dtype}")
    _check_device(m, m_scale, v, v_scale, m_value, v_value)
    _check(load().smile_adamw_unpack_states(n, _dtype_code(m_value), _ptr(m), _ptr(m_scale), _ptr(v), _ptr(v_scale), _ptr(m_value), _ptr(v_value),
                                            _stream(stream)), "smile_adamw_unpack_states")


# ------------------------------------------------------------------ device buffers for one layer

@dataclass
class LayerBuffers:
    """All intermediates/outputs of one forward pass as torch tensors on the GPU."""
    logits_inter: object
    logits_intra: object
    group_idx: object
    local_idx: object
    pos_in_group: object
    slot: object
    gate: object
    p_top: object
    q_top: object
    group_count: object
    local_count: object
    expert_count: object
    kept_count: object
    p_sum: object
    q_sum: object
    xe: object
    ye: object
    y: object
    loss3: object


def alloc_buffers(desc: LayerDesc, device="cuda:0") -> LayerBuffers:
    import torch
    T, d, n, m, Cap = desc.T, desc.d_model, desc.n_groups, desc.m_local, desc.capacity
    N = n * m
    st = torch_dtype(desc.dtype)
    f32, i32 = torch.float32, torch.int32

    def e(shape, dt):
        return torch.empty(shape, dtype=dt, device=device)

    return LayerBuffers(
        e((T, n), f32), e((T, m), f32), e((T,), i32), e((T,), i32), e((T,), i32), e((T,), i32),
        e((T,), f32), e((T,), f32), e((T,), f32), e((n,), i32), e((max(m, 4),), i32)[:m], e((N,), i32),
        e((N,), i32), e((n,), f32), e((m,), f32), e((N, Cap, d), st), e((N, Cap, d), st), e((T, d), st),
        e((4,), f32)[:3])


def make_io(x, w_inter, w_intra, w1, w2, buf: LayerBuffers, b1=None, b2=None, bias_inter=None,
            bias_intra=None) -> LayerIO:
    io = LayerIO()
    for k, v in dict(x=x, w_inter=w_inter, w_intra=w_intra, w1=w1, b1=b1, w2=w2, b2=b2,
                     bias_inter=bias_inter, bias_intra=bias_intra).items():
        setattr(io, k, _ptr(v))
    for k, v in buf.__dict__.items():
        setattr(io, k, _ptr(v))
    io.h_save = None
    io.pre_save = None
    return io
