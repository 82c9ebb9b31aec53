"""Python binding over libpf.so: argument marshalling only.

Every function has the name and the semantics of the C entry point it wraps (see
``include/pf.h``).  Tensors are torch CUDA tensors; torch is used for device memory and the
current stream, nothing else.  Outputs and workspaces that the caller does not pass come from
torch's caching allocator (the C library itself never allocates).  The marshalling is native
(``csrc/pf_python.cpp``, module ``_pf_native``): the functions here only give it names and
defaults.  ``lib()`` is the C library itself through ctypes.
"""
from __future__ import annotations

import ctypes
import math
import os

import torch

PF_F32, PF_BF16 = 0, 1
PF_ACT_NONE, PF_ACT_RELU = 0, 1
PF_GRAD_ACCUMULATE, PF_GRAD_F32 = 1, 2
PF_ROPE_HALVES, PF_ROPE_PAIRS = 0, 1
PF_STATE_F32, PF_STATE_8BIT = 0, 1
_PKG = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_PKG, "libpf.so")
_lib = None
_native = None


class PfError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {pf_status_string(status)} ({status})")


def lib() -> ctypes.CDLL:
    """The loaded C library; raises if it has not been built (no fallback path exists)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise ImportError(
                f"{_LIB_PATH} is missing: build it with `python -m paper_2103_03936_b200.build` "
                "(there is no CPU or PyTorch fallback)")
        L = ctypes.CDLL(_LIB_PATH)
        i64, vp, sz, ci = ctypes.c_int64, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int
        L.pf_status_string.restype = ctypes.c_char_p
        L.pf_status_string.argtypes = [ci]
        L.pf_version.restype = ci
        L.pf_last_device_status.restype = ci
        L.pf_launch_count.restype = ctypes.c_longlong
        L.pf_lowrank_linear_workspace.restype = sz
        L.pf_lowrank_linear_workspace.argtypes = [i64, i64, i64, i64, ci, ci]
        L.pf_lowrank_linear_fwd.restype = ci
        L.pf_lowrank_linear_fwd.argtypes = [vp, i64, vp, i64, vp, i64, vp, i64, vp, i64,
                                            i64, i64, i64, i64, ci, vp, sz, vp]
        L.pf_lowrank_linear_fwd_act.restype = ci
        L.pf_lowrank_linear_fwd_act.argtypes = [vp, i64, vp, i64, vp, i64, vp, ci, vp, i64, vp, i64,
                                                i64, i64, i64, i64, ci, vp, sz, vp]
        L.pf_bias_act_bwd_workspace.restype = sz
        L.pf_bias_act_bwd_workspace.argtypes = [i64, i64]
        L.pf_bias_act_bwd.restype = ci
        L.pf_bias_act_bwd.argtypes = [vp, i64, vp, i64, vp, i64, i64, ci, ci, vp, sz, vp]
        L.pf_lowrank_linear_fwd_static.restype = ci
        L.pf_lowrank_linear_fwd_static.argtypes = [vp, i64, vp, i64, vp, i64, vp, i64, vp, i64,
                                                   i64, i64, i64, i64, ci, vp]
        L.pf_static_scratch_bytes.restype = sz
        L.pf_lowrank_linear_bwd.restype = ci
        L.pf_lowrank_linear_bwd.argtypes = [vp, i64, vp, i64, vp, i64, vp, i64, vp, i64,
                                            vp, i64, vp, i64, vp, i64,
                                            i64, i64, i64, i64, ci, vp, sz, vp]
        L.pf_lowrank_linear_bwd_ex.restype = ci
        L.pf_lowrank_linear_bwd_ex.argtypes = [vp, i64, vp, i64, vp, i64, vp, i64, vp, i64,
                                               vp, i64, vp, i64, vp, i64, i64, i64, i64, i64, ci, ctypes.c_uint, vp, sz, vp]
        L.pf_lowrank_linear_grouped_workspace.restype = sz
        L.pf_lowrank_linear_grouped_workspace.argtypes = [ci, i64, i64, i64, i64, ci, ci]
        L.pf_lowrank_linear_grouped_fwd.restype = ci
        L.pf_lowrank_linear_grouped_fwd.argtypes = [ci] + [vp, i64, i64] * 5 + [i64, i64, i64, i64, ci, vp, sz, vp]
        L.pf_lowrank_linear_grouped_bwd.restype = ci
        L.pf_lowrank_linear_grouped_bwd.argtypes = [ci] + [vp, i64, i64] * 8 + [i64, i64, i64, i64, ci, vp, sz, vp]
        L.pf_lowrank_conv_workspace.restype = sz
        L.pf_lowrank_conv_workspace.argtypes = [ci] * 12
        L.pf_lowrank_conv_fwd.restype = ci
        L.pf_lowrank_conv_fwd.argtypes = [vp] * 5 + [ci] * 11 + [vp, sz, vp]
        L.pf_lowrank_conv_bwd.restype = ci
        L.pf_lowrank_conv_bwd.argtypes = [vp] * 8 + [ci] * 11 + [vp, sz, vp]
        L.pf_lowrank_conv_bwd_ex.restype = ci
        L.pf_lowrank_conv_bwd_ex.argtypes = [vp] * 8 + [ci] * 11 + [ctypes.c_uint, vp, sz, vp]
        L.pf_pack_factor_grads.restype = ci
        L.pf_pack_factor_grads.argtypes = [vp, vp, ci, ci, vp, i64, vp, vp, sz, vp]
        L.pf_unpack_factor_grads.restype = ci
        L.pf_unpack_factor_grads.argtypes = [vp, i64, vp, vp, ci, ci, vp, vp, sz, vp]
        L.pf_expert_rows.restype = i64
        L.pf_expert_rows.argtypes = [i64, ci, ci, i64]
        L.pf_expert_sort.restype = ci
        L.pf_expert_sort.argtypes = [vp, i64, ci, ci, i64, vp, vp, vp, vp, vp, sz, vp]
        L.pf_expert_sort_workspace.restype = sz
        L.pf_expert_sort_workspace.argtypes = [i64, ci, ci]
        sizes = [i64, ci, i64, i64, ci, vp]
        L.pf_expert_dispatch_fwd.restype = ci
        L.pf_expert_dispatch_fwd.argtypes = [vp, i64, vp, vp, vp, i64] + sizes
        L.pf_expert_dispatch_bwd.restype = ci
        L.pf_expert_dispatch_bwd.argtypes = [vp, i64, vp, vp, i64] + sizes
        L.pf_expert_combine_fwd.restype = ci
        L.pf_expert_combine_fwd.argtypes = [vp, i64, vp, vp, vp, i64] + sizes
        L.pf_expert_combine_bwd.restype = ci
        L.pf_expert_combine_bwd.argtypes = [vp, i64, vp, vp, vp, vp, i64, vp, i64, vp] + sizes
        heads = [i64, ci, ci, ci, ci, ci, ctypes.c_double, ci]
        L.pf_qk_norm_rope_fwd.restype = ci
        L.pf_qk_norm_rope_fwd.argtypes = [vp, i64, i64] * 2 + [vp] * 4 + [vp, i64, i64] * 2 + heads + [vp]
        L.pf_qk_norm_rope_bwd_workspace.restype = sz
        L.pf_qk_norm_rope_bwd_workspace.argtypes = [i64, ci, ci, ci]
        L.pf_qk_norm_rope_bwd.restype = ci
        L.pf_qk_norm_rope_bwd.argtypes = [vp, i64, i64] * 2 + [vp] * 4 + [vp, i64, i64] * 4 + [vp, vp] + heads + [ctypes.c_uint, vp, sz, vp]
        L.pf_adamw_step.restype = ci
        L.pf_adamw_step.argtypes = [vp] * 8 + [ci] * 4 + [vp] * 3
        _lib = L
    return _lib


def _load_native():
    """The marshalling module; raises if it has not been built."""
    global _native
    lib()
    path = os.path.join(_PKG, "_pf_native.so")
    if not os.path.exists(path):
        raise ImportError(f"{path} is missing: build it with `python -m paper_2103_03936_b200.build`")
    from . import _pf_native
    _pf_native.set_error(PfError)
    _native = _pf_native
    return _native


def pf_status_string(status: int) -> str:
    return lib().pf_status_string(int(status)).decode()


def pf_version() -> int:
    return int(lib().pf_version())


def pf_launch_count() -> int:
    return int(lib().pf_launch_count())


def pf_last_device_status() -> int:
    return int(lib().pf_last_device_status())


def pf_lowrank_linear_workspace(m, k, n, r, dtype, is_bwd) -> int:
    return int(lib().pf_lowrank_linear_workspace(m, k, n, r, dtype, int(bool(is_bwd))))


def pf_lowrank_linear_fwd(x, U, V, *, y=None, T_stash=None, want_stash=False, workspace=None,
                          stream=None, prepare=False):
    """y = (x U) V^T.  Returns y, or (y, T_stash) when a stash is requested.
    With prepare=True nothing is launched: returns (call, outputs) where call() issues the
    C call with the arguments marshalled once (fixed buffers and stream)."""
    n = _native or _load_native()
    return n.linear_fwd(x, U, V, None, 0, y, T_stash, want_stash, workspace, stream, prepare, False)


def pf_lowrank_linear_fwd_act(x, U, V, *, bias=None, act=PF_ACT_NONE, y=None, T_stash=None, want_stash=False,
                              workspace=None, stream=None, prepare=False):
    """y = act((x U) V^T + bias); bias [n] in x's dtype or None, act PF_ACT_NONE / PF_ACT_RELU.
    Otherwise as pf_lowrank_linear_fwd."""
    n = _native or _load_native()
    return n.linear_fwd(x, U, V, bias, act, y, T_stash, want_stash, workspace, stream, prepare, True)


def pf_bias_act_bwd(y, dY, *, act=PF_ACT_RELU, want_dbias=True, dbias=None, workspace=None, stream=None):
    """Backward of y = act(z + bias): dY [m, n] becomes dZ IN PLACE (zeroed where y <= 0 for PF_ACT_RELU);
    returns dbias [n] (column sums of dZ) or None."""
    n = _native or _load_native()
    return n.bias_act_bwd(y, dY, act, want_dbias, dbias, workspace, stream)


def pf_static_scratch_bytes() -> int:
    return int(lib().pf_static_scratch_bytes())


def pf_lowrank_linear_fwd_static(x, U, V, *, y, T_stash=None, stream=None):
    """y = (x U) V^T for callers that cannot allocate: the scratch is a fixed array inside the
    library, so the caller passes inputs and outputs only (y is required; nothing is allocated
    here either).  Raises PfError(PF_ERR_WORKSPACE) when the problem does not fit the array.
    Calls on one device share that array: do not let two of them overlap on the GPU."""
    n = _native or _load_native()
    return n.linear_fwd_static(x, U, V, y, T_stash, stream)


def pf_lowrank_linear_bwd(x, U, V, dY, *, T_stash=None, need_dX=True, dX=None, dU=None, dV=None,
                          accumulate=False, grads_f32=False, workspace=None, stream=None, prepare=False):
    """Returns (dX or None, dU, dV) for upstream gradient dY (prepare: see the forward).
    accumulate: dU and dV (required then) are added to; grads_f32: dU and dV are fp32 tensors."""
    n = _native or _load_native()
    return n.linear_bwd(x, U, V, dY, T_stash, need_dX, dX, dU, dV, accumulate, grads_f32, workspace, stream, prepare)


def pf_lowrank_linear_grouped_workspace(groups, m, k, n, r, dtype, is_bwd) -> int:
    return int(lib().pf_lowrank_linear_grouped_workspace(groups, m, k, n, r, dtype, int(bool(is_bwd))))


def pf_lowrank_linear_grouped_fwd(x, U, V, *, y=None, T_stash=None, want_stash=False, workspace=None,
                                  stream=None, prepare=False):
    """y[g] = (x[g] U[g]) V[g]^T for U [G, k, r], V [G, n, r] and x [G, m, k] or one shared x [m, k].
    Returns y [G, m, n], or (y, T_stash [G, m, r]) when a stash is requested."""
    n = _native or _load_native()
    return n.grouped_fwd(x, U, V, y, T_stash, want_stash, workspace, stream, prepare)


def pf_lowrank_linear_grouped_bwd(x, U, V, dY, *, T_stash=None, need_dX=True, dX=None, dU=None, dV=None,
                                  workspace=None, stream=None, prepare=False):
    """Returns (dX or None, dU [G, k, r], dV [G, n, r]).  dX is [G, m, k] when every group has its own
    x and ONE [m, k] matrix (the sum over the groups) when x [m, k] is shared."""
    n = _native or _load_native()
    return n.grouped_bwd(x, U, V, dY, T_stash, need_dX, dX, dU, dV, workspace, stream, prepare)


def pf_lowrank_conv_workspace(N, H, W, C, R, O, kh, kw, stride, pad, dtype, is_bwd) -> int:
    return int(lib().pf_lowrank_conv_workspace(N, H, W, C, R, O, kh, kw, stride, pad, dtype,
                                               int(bool(is_bwd))))


def pf_lowrank_conv_fwd(x, U, V, *, stride=1, pad=1, y=None, T_stash=None, want_stash=False,
                        workspace=None, stream=None, prepare=False):
    """NHWC factorized convolution.  Returns y, or (y, T_stash) when a stash is requested."""
    n = _native or _load_native()
    return n.conv_fwd(x, U, V, stride, pad, y, T_stash, want_stash, workspace, stream, prepare)


def pf_lowrank_conv_bwd(x, U, V, dY, *, stride=1, pad=1, T_stash=None, need_dX=True, dX=None,
                        dU=None, dV=None, accumulate=False, grads_f32=False, workspace=None, stream=None,
                        prepare=False):
    """Returns (dX or None, dU, dV) for upstream gradient dY [N, Ho, Wo, O].
    accumulate / grads_f32: as in pf_lowrank_linear_bwd."""
    n = _native or _load_native()
    return n.conv_bwd(x, U, V, dY, stride, pad, T_stash, need_dX, dX, dU, dV, accumulate, grads_f32, workspace, stream,
                      prepare)


def pf_pack_factor_grads(grads, *, flat=None, stream=None, prepare=False):
    """Copies the tensors of `grads`, in order and tightly, into one flat buffer.
    Returns (flat, offsets) with offsets a python list of count+1 element offsets."""
    if len(grads) == 0:
        offs = (ctypes.c_int64 * 1)()
        st = lib().pf_pack_factor_grads(None, None, 0, PF_BF16, flat.data_ptr() if flat is not None else None,
                                        flat.numel() if flat is not None else 0, offs, None, 0, None)
        if st != 0:
            raise PfError(st, "pf_pack_factor_grads")
        return flat, [0]
    n = _native or _load_native()
    return n.pack(grads, flat, stream, prepare)


def pf_unpack_factor_grads(flat, grads, *, stream=None):
    """The inverse of pf_pack_factor_grads: tensor i of `grads` (contiguous CUDA tensors of flat's
    dtype, overwritten) receives its slice of `flat`.  Returns the list of count+1 element offsets."""
    if len(grads) == 0:
        return [0]
    n = _native or _load_native()
    return n.unpack(flat, grads, stream)


def _fit(ints, longs=()) -> bool:
    """Whether numbers fit the C types of a size query, which ctypes would cut them to."""
    return all(abs(v) < 1 << 31 for v in ints) and all(abs(v) < 1 << 63 for v in longs)


def pf_expert_rows(tokens, k, experts, capacity=0) -> int:
    if not _fit((k, experts), (tokens, capacity)):
        return 0
    return int(lib().pf_expert_rows(tokens, k, experts, capacity))


def pf_expert_sort_workspace(tokens, k, experts) -> int:
    if not _fit((k, experts), (tokens,)):
        return 0
    return int(lib().pf_expert_sort_workspace(tokens, k, experts))


def pf_expert_sort(ids, experts, *, capacity=0, slots=None, sources=None, counts=None, offsets=None, workspace=None, stream=None, prepare=False):
    """Rows of a layer's experts for the assignments ids [tokens, k] (int32).  Returns (slots [tokens, k], sources [rows],
    counts [experts], offsets [experts + 1]), all int32; rows = experts * capacity, or tokens * k without a capacity."""
    n = _native or _load_native()
    return n.expert_sort(ids, experts, capacity, slots, sources, counts, offsets, workspace, stream, prepare)


def pf_expert_dispatch_fwd(x, slots, sources, *, xs=None, stream=None, prepare=False):
    """Tokens' rows x [tokens, width] in their experts' rows xs [rows, width] (rows without a token are zero); with a capacity
    xs.view(experts, capacity, width) is what pf_lowrank_linear_grouped_fwd takes."""
    n = _native or _load_native()
    return n.expert_dispatch_fwd(x, slots, sources, xs, stream, prepare)


def pf_expert_dispatch_bwd(dxs, slots, *, dx=None, stream=None, prepare=False):
    """dx [tokens, width]: for each token the sum of its experts' rows of dxs [rows, width]."""
    n = _native or _load_native()
    return n.expert_combine_fwd(dxs, slots, None, dx, stream, prepare, True)


def pf_expert_combine_fwd(ys, slots, weights=None, *, y=None, stream=None, prepare=False):
    """y [tokens, width]: for each token the sum of its experts' rows of ys [rows, width] times weights [tokens, k] (float32)."""
    n = _native or _load_native()
    return n.expert_combine_fwd(ys, slots, weights, y, stream, prepare, False)


def pf_expert_combine_bwd(ys, slots, sources, weights, dy, *, need_dys=True, dys=None, need_dweights=True, dweights=None, stream=None,
                          prepare=False):
    """Returns (dys [rows, width] or None, dweights [tokens, k] float32 or None) for the upstream gradient dy [tokens, width]."""
    n = _native or _load_native()
    return n.expert_combine_bwd(ys, slots, sources, weights, dy, need_dys, dys, need_dweights, dweights, stream, prepare)


def pf_qk_norm_rope_fwd(q, k, wq, wk, inv_freq, *, positions=None, style=PF_ROPE_HALVES, eps=1e-6, q_out=None, k_out=None, stream=None,
                        prepare=False):
    """Root-mean-square norm of each head of q [tokens, q_heads, dim] and k [tokens, k_heads, dim] (either may be None; any strides of
    tokens and heads), times wq, wk [dim] or None, its first 2 * len(inv_freq) elements rotated by positions [tokens] (int64;
    None: 0, 1, ...) times inv_freq (float32).  Returns (q_out, k_out)."""
    n = _native or _load_native()
    return n.qk_fwd(q, k, wq, wk, inv_freq, positions, style, eps, q_out, k_out, stream, prepare)


def pf_qk_norm_rope_bwd_workspace(tokens, q_heads, k_heads, dim) -> int:
    if not _fit((q_heads, k_heads, dim), (tokens,)):
        return 0
    return int(lib().pf_qk_norm_rope_bwd_workspace(tokens, q_heads, k_heads, dim))


def pf_qk_norm_rope_bwd(q, k, wq, wk, inv_freq, dq_out, dk_out, *, positions=None, style=PF_ROPE_HALVES, eps=1e-6, dq=None, dk=None,
                        need_dw=True, dwq=None, dwk=None, accumulate=False, grads_f32=False, workspace=None, stream=None, prepare=False):
    """Returns (dq, dk, dwq, dwk) for the gradients of pf_qk_norm_rope_fwd's outputs; dwq and dwk are None where there is no weight
    or need_dw=False.  accumulate: dwq and dwk (required then) are added to; grads_f32: they are float32."""
    n = _native or _load_native()
    return n.qk_bwd(q, k, wq, wk, inv_freq, positions, style, eps, dq_out, dk_out, dq, dk, need_dw, dwq, dwk, accumulate, grads_f32,
                    workspace, stream, prepare)


def pf_adamw_scalars(*, lr, betas=(0.9, 0.999), step, grad_scale=1.0, seed=0):
    """The five values that replace lr, step, grad_scale and seed of a pf_adamw_step with scalars=: a float32 tensor on the host
    (the seed's bits in the last), to be copied into the device tensor that the step reads."""
    if step < 1 or not 0 <= seed < 1 << 32:
        raise ValueError("need a step from 1 on and a seed of 0 .. 2^32 - 1")
    if not all(0 <= b < 1 for b in betas) or not (math.isfinite(lr) and math.isfinite(grad_scale)):
        raise ValueError("need betas of 0 .. 1 (without 1), and a finite lr and grad_scale")
    t = torch.tensor([lr, 1 - betas[0] ** step, 1 - betas[1] ** step, grad_scale, 0], dtype=torch.float32)
    t.view(torch.int32)[4] = seed - (1 << 32) if seed >= 1 << 31 else seed
    return t


def pf_adamw_step(params, grads, m, v, *, masters=None, m_scales=None, v_scales=None, lr=1e-3, betas=(0.9, 0.999), eps=1e-8,
                  weight_decay=0.01, step=1, grad_scale=1.0, seed=0, scalars=None, stream=None, prepare=False):
    """One AdamW step in place over lists of contiguous CUDA tensors.  m and v are float32, or float8_e4m3fn and float8_e5m2 with
    m_scales and v_scales (float32, one for each 256 elements of a tensor); masters (float32) go with bfloat16 parameters.
    scalars: a float32 CUDA tensor with the values of pf_adamw_scalars, read when the step runs.  Returns None
    (prepare=True: (call, None))."""
    if len(params) == 0:
        return ((lambda: None), None) if prepare else None
    n = _native or _load_native()
    return n.adamw_step(params, grads, m, v, masters, m_scales, v_scales, lr, betas[0], betas[1], eps, weight_decay, step, grad_scale, seed,
                        scalars, stream, prepare)
