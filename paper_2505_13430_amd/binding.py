"""Thin ctypes binding of libqzo.so (include/qzo.h): argument marshalling only.

Every function has the name of the C entry point it calls and takes torch CUDA
tensors for device memory.  PyTorch supplies memory and streams; every step of
the QZO path runs in the library's HIP kernels.  There is no fallback: if the
library has not been built, loading raises.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libqzo.so")
_lib = None

QZO_OK = 0
QZO_ERR_ARG, QZO_ERR_SHAPE, QZO_ERR_ALIGN, QZO_ERR_WORKSPACE = -1, -2, -3, -4
QZO_ERR_NONFINITE, QZO_ERR_HIP, QZO_ERR_UNSUPPORTED = -5, -6, -7
MAX_GROUPS = 2048               # of qzo_paged_attention_shared and qzo_answer_shared

EXPORTS = [
    "qzo_model_create", "qzo_model_destroy", "qzo_model_scale_count", "qzo_workspace_bytes",
    "qzo_forward_loss", "qzo_step", "qzo_model_apply_update",
    "qzo_model_dense_count", "qzo_model_joint_table_bytes", "qzo_model_enable_joint", "qzo_step_joint",
    "qzo_linear_scratch_bytes", "qzo_dequant_gemm", "qzo_dequant_gemm_static", "qzo_dequant_gemm_zp", "qzo_apply_update",
    "qzo_rtn_quantize", "qzo_rtn_quantize_asym", "qzo_repack_kmajor",
    "qzo_int4_expand", "qzo_int4_scratch_bytes", "qzo_int4_gemm_expanded", "qzo_model_set_int4_path",
    "qzo_nf4_expand", "qzo_nf4_scratch_bytes", "qzo_nf4_gemm",
    "qzo_codebook_scratch_bytes", "qzo_codebook_gemm", "qzo_apply_update_channel",
    "qzo_cache_plan", "qzo_qk_norm_rope", "qzo_paged_attention_scratch_bytes", "qzo_paged_attention",
    "qzo_cache_fork_scratch_bytes", "qzo_cache_fork", "qzo_cache_compact", "qzo_cache_copy", "qzo_beam_select_scratch_bytes", "qzo_beam_select",
    "qzo_paged_attention_shared_scratch_bytes", "qzo_paged_attention_shared",
    "qzo_answer_workspace_bytes", "qzo_answer", "qzo_answer_shared_workspace_bytes", "qzo_answer_shared",
    "qzo_debug_philox", "qzo_debug_normal_pairs", "qzo_debug_normals", "qzo_debug_dequant", "qzo_debug_dequant_zp",
    "qzo_debug_forward", "qzo_debug_bf16_gemm", "qzo_debug_reduce_norm", "qzo_debug_fused_linear", "qzo_debug_attention_slices",
    "qzo_debug_attention_linear",
    "qzo_debug_mfma_rate",
    "qzo_profile_begin", "qzo_profile_collect", "qzo_profile_stride",
    "qzo_last_error",
]


class QzoError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__(f"qzo status {status}: {msg}")
        self.status = status


class qzo_model_config(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("arch", C.c_uint32), ("n_layers", C.c_uint32),
                ("d_model", C.c_uint32), ("n_heads", C.c_uint32), ("d_ffn", C.c_uint32),
                ("vocab", C.c_uint32), ("max_seq", C.c_uint32), ("group_size", C.c_uint32),
                ("quant", C.c_uint32), ("norm_eps", C.c_float), ("rope_theta", C.c_float),
                ("scale_fp16", C.c_uint32), ("act_order", C.c_uint32)]


class qzo_buf(C.Structure):
    _fields_ = [("ptr_dev", C.c_void_p), ("bytes", C.c_uint64)]


class qzo_cache(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("type", C.c_uint32), ("n_blocks", C.c_uint32), ("block", C.c_uint32),
                ("kv_heads", C.c_uint32), ("head_dim", C.c_uint32), ("k_dev", C.c_void_p), ("v_dev", C.c_void_p),
                ("k_scale_dev", C.c_void_p), ("v_scale_dev", C.c_void_p)]


def lib():
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -c 'import __graft_entry__ as g; g.build()'`")
        _lib = C.CDLL(LIB_PATH)
        _lib.qzo_last_error.restype = C.c_char_p
        for name in EXPORTS[:-1]:
            getattr(_lib, name).restype = C.c_int
        # called once or more per layer and token: arguments converted by declared types
        u32, u64, i32, p, f, d = C.c_uint32, C.c_uint64, C.c_int32, C.c_void_p, C.c_float, C.c_double
        _lib.qzo_cache_plan.argtypes = [p, p, u32, u32, u32, u32, u32] + [p] * 9
        _lib.qzo_qk_norm_rope.argtypes = [p, u64, u32, u32, u32, u32, p, p, f, f, p, u32, p, p, p, u64, p]
        _lib.qzo_paged_attention_scratch_bytes.argtypes = [u32, u32, u32, u32, p]
        _lib.qzo_answer.argtypes = [p, p, u32, u32, p, p, u32, p, p, p, p, p, u64, p, p]
        _lib.qzo_paged_attention.argtypes = [p, u64, u32, u32, u32, p, p, u32, p, p, f, p, u64, p, u64, p]
        _lib.qzo_cache_fork_scratch_bytes.argtypes = [u32, u32, u32, p]
        _lib.qzo_cache_fork.argtypes = [p, u32, u32, u32, u32, p, p, p, p, u32, p, p, p, p, u64, p]
        _lib.qzo_cache_compact.argtypes = [u32, u32, u32, u32, p, p, p, p, p, p, p, u64, p]
        _lib.qzo_cache_copy.argtypes = [p, u32, p, u32, p, p]
        _lib.qzo_beam_select_scratch_bytes.argtypes = [u32, u32, u32, p]
        _lib.qzo_beam_select.argtypes = [p, u64, u32, u32, u32, i32, d, p, p, p, p, u32, p, p, p, p, p, u64, p]
        _lib.qzo_paged_attention_shared_scratch_bytes.argtypes = [u32, u32, u32, u32, u32, p]
        _lib.qzo_paged_attention_shared.argtypes = [p, u64, u32, u32, u32, p, p, u32, p, p, u32, p, p, f, p, u64, p, u64, p]
        _lib.qzo_answer_shared_workspace_bytes.argtypes = [p, u32, u32, p]
        _lib.qzo_answer_shared.argtypes = [p, p, u32, u32, p, p, u32, p, p, p, p, u32, p, p, p, u64, p, p]
    return _lib


def _check(status):
    if status != QZO_OK:
        raise QzoError(status, lib().qzo_last_error().decode())


def _ptr(t):
    if t is None:
        return C.c_void_p(0)
    assert t.is_cuda and t.is_contiguous(), "device tensors must be contiguous CUDA tensors"
    return C.c_void_p(t.data_ptr())


def _stream(stream):
    s = torch.cuda.current_stream() if stream is None else stream
    return C.c_void_p(s.cuda_stream)


def make_config(shape: dict) -> qzo_model_config:
    return qzo_model_config(C.sizeof(qzo_model_config), 0 if shape["arch"] == "llama" else 1,
                            shape["n_layers"], shape["d_model"], shape["n_heads"], shape["d_ffn"],
                            shape["vocab"], shape["max_seq"], shape.get("group", 128), shape.get("quant", 0),
                            shape.get("norm_eps", 1e-5), shape.get("rope_theta", 10000.0),
                            int(shape.get("scale_fp16", 0)), int(shape.get("act_order", 0)))


def qzo_model_scale_count(shape: dict) -> int:
    cfg = make_config(shape)
    out = C.c_uint64(0)
    _check(lib().qzo_model_scale_count(C.byref(cfg), C.byref(out)))
    return out.value


def qzo_model_create(shape: dict, tensors, scale_arena):
    cfg = make_config(shape)
    bufs = (qzo_buf * len(tensors))(*[qzo_buf(t.data_ptr(), t.numel() * t.element_size())
                                      for t in tensors])
    handle = C.c_void_p(0)
    _check(lib().qzo_model_create(C.byref(cfg), bufs, C.c_uint32(len(tensors)), _ptr(scale_arena),
                                  C.c_uint64(scale_arena.numel()), C.byref(handle)))
    return handle


def qzo_model_destroy(model):
    _check(lib().qzo_model_destroy(model))


def qzo_workspace_bytes(model, batch, seq) -> int:
    out = C.c_uint64(0)
    _check(lib().qzo_workspace_bytes(model, C.c_uint32(batch), C.c_uint32(seq), C.byref(out)))
    return out.value


def qzo_forward_loss(model, tokens, seed, eps, sign, workspace, loss_out, stream=None):
    B, S = tokens.shape
    _check(lib().qzo_forward_loss(model, _ptr(tokens), C.c_uint32(B), C.c_uint32(S),
                                  C.c_uint64(seed), C.c_float(eps), C.c_int(sign), _ptr(workspace),
                                  C.c_uint64(workspace.numel() * workspace.element_size()),
                                  _ptr(loss_out), _stream(stream)))


def qzo_step(model, tokens, seed, eps, eta, clip, workspace, result, stream=None):
    """result: 8 x 4-byte device tensor receiving qzo_step_result."""
    B, S = tokens.shape
    _check(lib().qzo_step(model, _ptr(tokens), C.c_uint32(B), C.c_uint32(S), C.c_uint64(seed),
                          C.c_float(eps), C.c_float(eta), C.c_float(clip), _ptr(workspace),
                          C.c_uint64(workspace.numel() * workspace.element_size()), _ptr(result),
                          _stream(stream)))


def qzo_model_dense_count(shape: dict) -> int:
    cfg = make_config(shape)
    out = C.c_uint64(0)
    _check(lib().qzo_model_dense_count(C.byref(cfg), C.byref(out)))
    return out.value


def qzo_model_joint_table_bytes(shape: dict) -> int:
    cfg = make_config(shape)
    out = C.c_uint64(0)
    _check(lib().qzo_model_joint_table_bytes(C.byref(cfg), C.byref(out)))
    return out.value


def qzo_model_enable_joint(model, dense_master, table):
    """table: uint8 device tensor of qzo_model_joint_table_bytes bytes, kept alive by the caller."""
    assert dense_master.dtype == torch.float32
    _check(lib().qzo_model_enable_joint(model, _ptr(dense_master), C.c_uint64(dense_master.numel()),
                                        _ptr(table), C.c_uint64(table.numel() * table.element_size())))


def qzo_step_joint(model, tokens, seed, eps, eta, eta_dense, clip, workspace, result, stream=None):
    B, S = tokens.shape
    _check(lib().qzo_step_joint(model, _ptr(tokens), C.c_uint32(B), C.c_uint32(S), C.c_uint64(seed),
                                C.c_float(eps), C.c_float(eta), C.c_float(eta_dense), C.c_float(clip),
                                _ptr(workspace), C.c_uint64(workspace.numel() * workspace.element_size()),
                                _ptr(result), _stream(stream)))


def read_step_result(result) -> dict:
    """Host copy of a qzo_step_result (synchronises)."""
    raw = result.cpu()
    f = raw.view(torch.float32)
    i = raw.view(torch.int32)
    return dict(loss_plus=float(f[0]), loss_minus=float(f[1]), d=float(f[2]),
                d_clipped=float(f[3]), status=int(i[4]))


def qzo_model_apply_update(model, seed, eta, d_clipped, stream=None):
    _check(lib().qzo_model_apply_update(model, C.c_uint64(seed), C.c_float(eta),
                                        C.c_float(d_clipped), _stream(stream)))


def qzo_linear_scratch_bytes(M, N, K, with_sumsq) -> int:
    out = C.c_uint64(0)
    _check(lib().qzo_linear_scratch_bytes(C.c_uint32(M), C.c_uint32(N), C.c_uint32(K), C.c_int(int(with_sumsq)),
                                          C.byref(out)))
    return out.value


_scratch = {}


def scratch_for(device, nbytes):
    """Device-memory plumbing for the single-linear calls: one cached uint8 tensor per device, grown
    on demand (torch allocations are 256-byte aligned).  Calls that use it must not overlap."""
    t = _scratch.get(device)
    if t is None or t.numel() < nbytes:
        t = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)
        _scratch[device] = t
    return t


def _scratch_args(scratch):
    if scratch is None:
        return C.c_void_p(0), C.c_uint64(0)
    return _ptr(scratch), C.c_uint64(scratch.numel() * scratch.element_size())


def qzo_dequant_gemm(x, q, s, row_base, seed, eps, sign, y, sumsq=None, group=128, stream=None, scratch="auto"):
    M, K = x.shape
    N = q.shape[0]
    if isinstance(scratch, str):
        scratch = scratch_for(x.device, qzo_linear_scratch_bytes(M, N, K, sumsq is not None)) if K % 128 == 0 and K else None
    _check(lib().qzo_dequant_gemm(_ptr(x), _ptr(q), _ptr(s), C.c_uint32(row_base), C.c_uint32(M),
                                  C.c_uint32(N), C.c_uint32(K), C.c_uint32(group), C.c_uint64(seed),
                                  C.c_float(eps), C.c_int(sign), _ptr(y), _ptr(sumsq),
                                  *_scratch_args(scratch), _stream(stream)))


def qzo_dequant_gemm_static(x, q, s, row_base, seed, eps, sign, y, sumsq=None, group=128, stream=None):
    M, K = x.shape
    N = q.shape[0]
    _check(lib().qzo_dequant_gemm_static(_ptr(x), _ptr(q), _ptr(s), C.c_uint32(row_base), C.c_uint32(M),
                                         C.c_uint32(N), C.c_uint32(K), C.c_uint32(group), C.c_uint64(seed),
                                         C.c_float(eps), C.c_int(sign), _ptr(y), _ptr(sumsq), _stream(stream)))


def qzo_dequant_gemm_zp(x, q, s, zp, row_base, seed, eps, sign, y, sumsq=None, group=128, stream=None,
                        scratch="auto", scale_fp16=None):
    """s: bf16 or fp16 scales (scale_fp16 defaults to the tensor's dtype)."""
    if scale_fp16 is None:
        scale_fp16 = s.dtype == torch.float16
    M, K = x.shape
    N = q.shape[0]
    if isinstance(scratch, str):
        scratch = scratch_for(x.device, qzo_linear_scratch_bytes(M, N, K, sumsq is not None)) if K % 128 == 0 and K else None
    _check(lib().qzo_dequant_gemm_zp(_ptr(x), _ptr(q), _ptr(s), _ptr(zp), C.c_uint32(int(scale_fp16)),
                                     C.c_uint32(row_base), C.c_uint32(M), C.c_uint32(N), C.c_uint32(K), C.c_uint32(group),
                                     C.c_uint64(seed), C.c_float(eps), C.c_int(sign), _ptr(y),
                                     _ptr(sumsq), *_scratch_args(scratch), _stream(stream)))


def qzo_repack_kmajor(qweight, qzeros, scales, zero_add, q, zp, s, group=128, stream=None):
    K, N = qweight.shape[0] * 8, qweight.shape[1]
    _check(lib().qzo_repack_kmajor(_ptr(qweight), _ptr(qzeros), _ptr(scales), C.c_uint32(N),
                                   C.c_uint32(K), C.c_uint32(group), C.c_uint32(zero_add),
                                   C.c_uint32(int(s.dtype == torch.float16)), _ptr(q),
                                   _ptr(zp), _ptr(s), _stream(stream)))


def qzo_apply_update(s, row_base, seed, eta, d_clipped, stream=None):
    n_rows, G = s.shape
    _check(lib().qzo_apply_update(_ptr(s), C.c_uint32(n_rows), C.c_uint32(G), C.c_uint32(row_base),
                                  C.c_uint64(seed), C.c_float(eta), C.c_float(d_clipped),
                                  C.c_uint32(int(s.dtype == torch.float16)), _stream(stream)))


def qzo_rtn_quantize(w, q, s, group=128, stream=None):
    N, K = w.shape
    _check(lib().qzo_rtn_quantize(_ptr(w), C.c_uint32(N), C.c_uint32(K), C.c_uint32(group), _ptr(q),
                                  _ptr(s), _stream(stream)))


def qzo_rtn_quantize_asym(w, q, zp, s, group=128, stream=None):
    """s: bf16 or fp16 output tensor; its dtype selects the scale's storage type."""
    N, K = w.shape
    _check(lib().qzo_rtn_quantize_asym(_ptr(w), C.c_uint32(N), C.c_uint32(K), C.c_uint32(group),
                                       C.c_uint32(int(s.dtype == torch.float16)), _ptr(q), _ptr(zp), _ptr(s),
                                       _stream(stream)))


def qzo_debug_normals(seed, stream_id, row0, out, stream=None):
    n_rows, G = out.shape
    _check(lib().qzo_debug_normals(C.c_uint64(seed), C.c_uint32(stream_id), C.c_uint32(row0),
                                   C.c_uint32(n_rows), C.c_uint32(G), _ptr(out), _stream(stream)))


def qzo_debug_philox(seed, ctr, out, stream=None):
    _check(lib().qzo_debug_philox(C.c_uint64(seed), _ptr(ctr), C.c_uint32(ctr.shape[0]), _ptr(out),
                                  _stream(stream)))


def qzo_debug_normal_pairs(words, out, stream=None):
    _check(lib().qzo_debug_normal_pairs(_ptr(words), C.c_uint32(words.numel()), _ptr(out),
                                        _stream(stream)))


def qzo_debug_dequant(q, s, row_base, seed, eps, sign, w_eff, group=128, stream=None):
    N, K = w_eff.shape
    _check(lib().qzo_debug_dequant(_ptr(q), _ptr(s), C.c_uint32(row_base), C.c_uint32(N),
                                   C.c_uint32(K), C.c_uint32(group), C.c_uint64(seed),
                                   C.c_float(eps), C.c_int(sign), _ptr(w_eff), _stream(stream)))


def qzo_int4_expand(q, s, zp, row_base, seed, eps, sign, se_out, w_out, g_idx=None, stream=None):
    N, K = q.shape[0], q.shape[1] * 2
    _check(lib().qzo_int4_expand(_ptr(q), _ptr(s), _ptr(zp), _ptr(g_idx), C.c_uint32(row_base), C.c_uint32(N),
                                 C.c_uint32(K), C.c_uint32(128), C.c_uint64(seed), C.c_float(eps), C.c_int(sign),
                                 _ptr(se_out), _ptr(w_out), _stream(stream)))


def qzo_int4_scratch_bytes(N, K) -> int:
    out = C.c_uint64(0)
    _check(lib().qzo_int4_scratch_bytes(C.c_uint32(N), C.c_uint32(K), C.byref(out)))
    return out.value


def qzo_int4_gemm_expanded(x, q, s, zp, g_idx, row_base, seed, eps, sign, y, scratch, stream=None):
    M, K = x.shape
    N = q.shape[0]
    _check(lib().qzo_int4_gemm_expanded(_ptr(x), _ptr(q), _ptr(s), _ptr(zp), _ptr(g_idx), C.c_uint32(row_base),
                                        C.c_uint32(M), C.c_uint32(N), C.c_uint32(K), C.c_uint32(128),
                                        C.c_uint64(seed), C.c_float(eps), C.c_int(sign), _ptr(y), _ptr(scratch),
                                        C.c_uint64(scratch.numel() * scratch.element_size()), _stream(stream)))


def qzo_nf4_expand(q, s, row_base, seed, eps, sign, se_out, w_out, stream=None):
    N, K = q.shape[0], q.shape[1] * 2
    _check(lib().qzo_nf4_expand(_ptr(q), _ptr(s), C.c_uint32(row_base), C.c_uint32(N), C.c_uint32(K),
                                C.c_uint32(64), C.c_uint64(seed), C.c_float(eps), C.c_int(sign),
                                _ptr(se_out), _ptr(w_out), _stream(stream)))


def qzo_nf4_scratch_bytes(N, K) -> int:
    out = C.c_uint64(0)
    _check(lib().qzo_nf4_scratch_bytes(C.c_uint32(N), C.c_uint32(K), C.byref(out)))
    return out.value


def qzo_nf4_gemm(x, q, s, row_base, seed, eps, sign, y, scratch, stream=None):
    M, K = x.shape
    N = q.shape[0]
    _check(lib().qzo_nf4_gemm(_ptr(x), _ptr(q), _ptr(s), C.c_uint32(row_base), C.c_uint32(M), C.c_uint32(N),
                              C.c_uint32(K), C.c_uint32(64), C.c_uint64(seed), C.c_float(eps), C.c_int(sign),
                              _ptr(y), _ptr(scratch), C.c_uint64(scratch.numel() * scratch.element_size()),
                              _stream(stream)))


def qzo_model_set_int4_path(model, mode: int):
    _check(lib().qzo_model_set_int4_path(model, C.c_int(mode)))


def qzo_debug_bf16_gemm(x, w, y, pipe=2, stream=None):
    M, K = x.shape
    N = w.shape[0]
    _check(lib().qzo_debug_bf16_gemm(_ptr(x), _ptr(w), C.c_uint32(M), C.c_uint32(N), C.c_uint32(K),
                                     C.c_int(pipe), _ptr(y), _stream(stream)))


def qzo_debug_reduce_norm(part, bias, resid, gain, norm_bias, eps, joined, y, out, xsum=None, stream=None) -> bool:
    """Returns whether the reduction and the norm ran as one launch."""
    slices, M, N = part.shape
    done = C.c_uint32(0)
    _check(lib().qzo_debug_reduce_norm(_ptr(part), C.c_uint32(slices), C.c_uint32(M), C.c_uint32(N), _ptr(bias),
                                       _ptr(resid), _ptr(gain), _ptr(norm_bias), C.c_float(eps), C.c_int(int(joined)),
                                       _ptr(y), _ptr(out), _ptr(xsum), C.byref(done), _stream(stream)))
    return bool(done.value)


def qzo_debug_fused_linear(x, q, s, zp, row_base, seed, eps, sign, y, passes=1, nf4=False, epilogue=0, bias=None, resid=None,
                           rope=None, head_dim=0, height=0, stream=None) -> int:
    """Returns the height of the output tiles, in units of 32 tokens; of two launches, + 65536 times the second one's.
    rope [seq, head_dim / 2, 2]."""
    N, K, mt = q.shape[0], x.shape[1], C.c_uint32(height)
    assert x.shape[0] % passes == 0 and y.shape == (x.shape[0], N // 2 if epilogue == 16 else N)
    _check(lib().qzo_debug_fused_linear(_ptr(x), _ptr(q), _ptr(s), _ptr(zp), C.c_int(int(nf4)), C.c_uint32(row_base),
                                        C.c_uint32(x.shape[0] // passes), C.c_uint32(passes), C.c_uint32(N), C.c_uint32(K),
                                        C.c_uint64(seed & 0xFFFFFFFFFFFFFFFF), C.c_float(eps), C.c_int(sign), C.c_uint32(epilogue),
                                        _ptr(bias), _ptr(resid), _ptr(rope), C.c_uint32(0 if rope is None else rope.shape[0]),
                                        C.c_uint32(head_dim), C.byref(mt), _ptr(y), _stream(stream)))
    return mt.value


def qzo_debug_attention_slices(part, rope, n_heads, joined, qkv, out, stream=None) -> bool:
    """part [slices, batch, seq, 3 d].  Returns whether the attention added up the slices itself."""
    slices, B, S, d3 = part.shape
    done = C.c_uint32(0)
    _check(lib().qzo_debug_attention_slices(_ptr(part), C.c_uint32(slices), C.c_uint32(B), C.c_uint32(S), C.c_uint32(n_heads),
                                            C.c_uint32(d3 // 3 // n_heads), _ptr(rope), C.c_int(int(joined)), _ptr(qkv),
                                            _ptr(out), C.byref(done), _stream(stream)))
    return bool(done.value)


def qzo_debug_attention_linear(qkv, n_heads, passes, rope, packed, att, xsum, q, s, zp, row_base, seed, eps, sign, part, y,
                               stream=None) -> int:
    """qkv [passes, batch, seq, 3 n_heads 128].  Returns the number of K slices in part."""
    _, B, S, _ = qkv.shape
    slices = C.c_uint32(0)
    assert att.numel() >= 128 * 128 * n_heads and xsum.numel() >= 128 * n_heads and y.shape == (passes * B * S, q.shape[0])
    _check(lib().qzo_debug_attention_linear(
        _ptr(qkv), C.c_uint32(B), C.c_uint32(S), C.c_uint32(n_heads), C.c_uint32(passes), _ptr(rope), C.c_int(int(packed)), _ptr(att),
        _ptr(xsum), _ptr(q), _ptr(s), _ptr(zp), C.c_int(int(s.dtype == torch.float16)), C.c_uint32(q.shape[0]), C.c_uint32(row_base),
        C.c_uint64(seed & 0xFFFFFFFFFFFFFFFF), C.c_float(eps), C.c_int(sign), _ptr(part), C.c_uint64(part.numel()),
        C.byref(slices), _ptr(y), _stream(stream)))
    return slices.value


def qzo_debug_dequant_zp(q, s, zp, row_base, seed, eps, sign, w_eff, group=128, stream=None):
    N, K = w_eff.shape
    _check(lib().qzo_debug_dequant_zp(_ptr(q), _ptr(s), _ptr(zp), C.c_uint32(int(s.dtype == torch.float16)),
                                      C.c_uint32(row_base), C.c_uint32(N),
                                      C.c_uint32(K), C.c_uint32(group), C.c_uint64(seed),
                                      C.c_float(eps), C.c_int(sign), _ptr(w_eff), _stream(stream)))


def qzo_debug_forward(model, tokens, seed, eps, sign, workspace, loss_out, hidden_out, stream=None):
    B, S = tokens.shape
    _check(lib().qzo_debug_forward(model, _ptr(tokens), C.c_uint32(B), C.c_uint32(S),
                                   C.c_uint64(seed), C.c_float(eps), C.c_int(sign), _ptr(workspace),
                                   C.c_uint64(workspace.numel() * workspace.element_size()),
                                   _ptr(loss_out), _ptr(hidden_out), _stream(stream)))


PROFILE_KINDS = {"w4a16_gemm": 0, "lmhead_ce": 1, "attention": 2, "scale_update": 3, "embed": 4, "expand": 5}


def qzo_profile_stride(stride: int):
    _check(lib().qzo_profile_stride(C.c_uint32(stride)))


def qzo_debug_mfma_rate(iters: int, random_operands: bool, sink, stream=None) -> int:
    """Launches the matrix-pipe rate probe; returns the number of workgroups (8 wavefronts each)."""
    wgs = C.c_uint32(0)
    assert sink.numel() >= 512 * 512
    _check(lib().qzo_debug_mfma_rate(C.c_uint32(iters), C.c_int(int(random_operands)), _ptr(sink),
                                     C.byref(wgs), _stream(stream)))
    return wgs.value


def qzo_profile_begin(max_records: int):
    _check(lib().qzo_profile_begin(C.c_uint32(max_records)))


def qzo_profile_collect(kind: int) -> dict:
    ms, n, work = C.c_double(0), C.c_uint64(0), C.c_double(0)
    _check(lib().qzo_profile_collect(C.c_uint32(kind), C.byref(ms), C.byref(n), C.byref(work)))
    return dict(total_ms=ms.value, launches=n.value, work=work.value)


def qzo_codebook_scratch_bytes(M, N, with_sumsq) -> int:
    out = C.c_uint64(0)
    _check(lib().qzo_codebook_scratch_bytes(C.c_uint32(M), C.c_uint32(N), C.c_int(int(with_sumsq)), C.byref(out)))
    return out.value


def qzo_codebook_gemm(x, codes, codebook, c, row_base, seed, eps, sign, y, sumsq=None, stream=None,
                      scratch="auto"):
    M, K = x.shape
    N = codes.shape[0]
    if isinstance(scratch, str):
        scratch = scratch_for(x.device, qzo_codebook_scratch_bytes(M, N, sumsq is not None))
    _check(lib().qzo_codebook_gemm(_ptr(x), _ptr(codes), _ptr(codebook), _ptr(c), C.c_uint32(row_base),
                                   C.c_uint32(M), C.c_uint32(N), C.c_uint32(K), C.c_uint64(seed),
                                   C.c_float(eps), C.c_int(sign), _ptr(y), _ptr(sumsq),
                                   *_scratch_args(scratch), _stream(stream)))


def qzo_apply_update_channel(c, row_base, seed, eta, d_clipped, stream=None):
    _check(lib().qzo_apply_update_channel(_ptr(c), C.c_uint32(c.numel()), C.c_uint32(row_base),
                                          C.c_uint64(seed), C.c_float(eta), C.c_float(d_clipped),
                                          _stream(stream)))


# The calls below are made once or more per layer and token: their checks are written for few attribute reads.
def _rows(t, at):
    """Address and row stride of a bf16 matrix on device `at` whose rows are contiguous."""
    ld, step = t.stride()
    n, width = t.shape
    assert t.dtype is torch.bfloat16 and t.get_device() == at and (step == 1 or width == 1), \
        "a bf16 matrix on the current device is needed, its rows contiguous"
    return t.data_ptr(), (ld if n > 1 else width)


def _at(t, dtype, at):
    """Address of a contiguous tensor of that type on device `at`; None: null."""
    if t is None:
        return None
    assert t.dtype is dtype and t.get_device() == at and t.is_contiguous(), f"a contiguous tensor of {dtype} on the current device is needed"
    return t.data_ptr()


def _room(t, at):
    """Address and bytes of memory on device `at` that a call may use; None: null."""
    if t is None:
        return None, 0
    assert t.get_device() == at and t.is_contiguous(), "scratch and workspace are contiguous tensors on the current device"
    return t.data_ptr(), t.numel() * t.element_size()


def _stream_of(stream, at):
    return torch._C._cuda_getCurrentRawStream(at) if stream is None else stream.cuda_stream


def make_cache(k, v, k_scale=None, v_scale=None) -> qzo_cache:
    """k, v: bf16 or float8_e4m3fn [n_blocks, kv_heads, block, head_dim]; e4m3: fp32 scales [kv_heads].  Holds its tensors."""
    n_blocks, kv_heads, block, dh = k.shape
    at, kind = k.get_device(), k.dtype
    assert at >= 0 and k.shape == v.shape and (kind is torch.bfloat16 or kind is torch.float8_e4m3fn)
    assert (k_scale is None or k_scale.numel() == kv_heads) and (v_scale is None or v_scale.numel() == kv_heads)
    c = qzo_cache(C.sizeof(qzo_cache), kind is not torch.bfloat16, n_blocks, block, kv_heads, dh, _at(k, kind, at), _at(v, kind, at),
                  _at(k_scale, torch.float32, at), _at(v_scale, torch.float32, at))
    c.tensors, c.device = (k, v, k_scale, v_scale), at
    return c


def qzo_cache_plan(cached, added, block, tables, free, before, lengths, starts, slots, positions, after, stream=None):
    """int32 tensors; tables [n_seq, max_blocks], free [n_blocks], slots and positions [max_tokens], before and after: a
    qzo_cache_state of four int32 (free blocks, tokens, status, blocks taken)."""
    at, i32, (n, most), tokens = torch.cuda.current_device(), torch.int32, tables.shape, slots.numel()
    assert cached.numel() == added.numel() == lengths.numel() == n == starts.numel() - 1 and positions.numel() == tokens
    assert before.numel() == after.numel() == 4
    _check(lib().qzo_cache_plan(_at(cached, i32, at), _at(added, i32, at), n, block, free.numel(), most, tokens, _at(tables, i32, at),
                                _at(free, i32, at), _at(before, i32, at), _at(lengths, i32, at), _at(starts, i32, at), _at(slots, i32, at),
                                _at(positions, i32, at), _at(after, i32, at), _stream_of(stream, at)))


def qzo_qk_norm_rope(qkv, q_heads, kv_heads, out, q_gain=None, k_gain=None, eps=1e-6, theta=10000.0, positions=None, seq=0, cache=None,
                     slots=None, stream=None):
    """qkv bf16 [tokens, (q_heads + 2 kv_heads) head_dim]; out bf16 [tokens, the heads of q (and of k without a cache)], it may be
    a column range of qkv's own rows from the first on (in place).  Rows may be strided."""
    at, (T, width) = torch.cuda.current_device(), qkv.shape
    x, ldx = _rows(qkv, at)
    y, ldy = _rows(out, at)
    dh = width // (q_heads + 2 * kv_heads)
    T2, wide = out.shape
    assert width == (q_heads + 2 * kv_heads) * dh and T2 == T and wide >= (q_heads if cache is not None else q_heads + kv_heads) * dh
    assert (q_gain is None or q_gain.numel() == dh) and (k_gain is None or k_gain.numel() == dh)
    assert (positions is None or positions.numel() >= T) and (slots is None or slots.numel() >= T) and (cache is None or cache.device == at)
    if T == 0:
        return                                  # an empty tensor has no address
    _check(lib().qzo_qk_norm_rope(x, ldx, T, q_heads, kv_heads, dh, _at(q_gain, torch.bfloat16, at), _at(k_gain, torch.bfloat16, at), eps, theta,
                                  _at(positions, torch.int32, at), seq, None if cache is None else C.addressof(cache),
                                  _at(slots, torch.int32, at), y, ldy, _stream_of(stream, at)))


def qzo_paged_attention_scratch_bytes(n_rows, n_seq, q_heads, head_dim) -> int:
    out = C.c_uint64(0)
    _check(lib().qzo_paged_attention_scratch_bytes(n_rows, n_seq, q_heads, head_dim, C.addressof(out)))
    return out.value


_stream_scratch = {}


def _scratch_of_stream(device, stream, handle, nbytes, kind=None):
    """Address and bytes of the scratch of the calls of a kind on one stream, which do not overlap.  A captured graph keeps the address it was captured
    with and may be replayed on any stream beside any other: it is given scratch of its own."""
    captured = torch.cuda.is_current_stream_capturing()
    if stream is not None:                     # a stream may be captured without being the current one
        with torch.cuda.stream(stream):
            captured = captured or torch.cuda.is_current_stream_capturing()
    assert not captured, "a captured call needs scratch of its own: pass scratch"
    kept = _stream_scratch.get((device, handle, kind))
    if kept is None or kept[1] < nbytes:
        with torch.cuda.stream(stream):        # what is outgrown is used again on this stream only
            t = torch.zeros(nbytes, dtype=torch.uint8, device=device)
        kept = _stream_scratch[device, handle, kind] = t.data_ptr(), nbytes, t
    return kept[:2]


def qzo_paged_attention(q, cache, tables, lengths, out, scale, starts=None, scratch="auto", stream=None):
    """q, out bf16 [rows, q_heads head_dim], rows may be strided; tables int32 [n_seq, max_blocks], lengths int32 [n_seq], starts
    int32 [n_seq + 1] or None: a row per sequence.  scratch: uint8, its first 2048 bytes zero before its first call; "auto": one
    for all calls on the stream."""
    at, i32, (rows, width), (n, most), dh = torch.cuda.current_device(), torch.int32, q.shape, tables.shape, cache.head_dim
    x, ldx = _rows(q, at)
    y, ldy = _rows(out, at)
    heads = width // dh
    assert q.shape == out.shape and heads * dh == width and cache.device == at
    assert lengths.numel() == n and (starts is None or starts.numel() == n + 1)
    if rows == 0:
        return
    st = _stream_of(stream, at)
    if isinstance(scratch, str):
        room = _scratch_of_stream(at, stream, st, qzo_paged_attention_scratch_bytes(rows, n, heads, dh))
    else:
        room = _room(scratch, at)
    _check(lib().qzo_paged_attention(x, ldx, rows, n, heads, C.addressof(cache), _at(tables, i32, at), most, _at(lengths, i32, at),
                                     _at(starts, i32, at), scale, y, ldy, *room, st))


def qzo_paged_attention_shared_scratch_bytes(n_rows, n_seq, q_heads, kv_heads, head_dim) -> int:
    out = C.c_uint64(0)
    _check(lib().qzo_paged_attention_shared_scratch_bytes(n_rows, n_seq, q_heads, kv_heads, head_dim, C.addressof(out)))
    return out.value


def qzo_paged_attention_shared(q, cache, tables, lengths, group_starts, shared, out, scale, starts=None, scratch="auto", stream=None):
    """qzo_paged_attention of sequences whose groups begin alike: group_starts int32 [n_groups + 1], shared int32 [n_groups], the tokens that
    a group's sequences have in common."""
    at, i32, (rows, width), (n, most), dh = torch.cuda.current_device(), torch.int32, q.shape, tables.shape, cache.head_dim
    x, ldx = _rows(q, at)
    y, ldy = _rows(out, at)
    heads, groups = width // dh, shared.numel()
    assert q.shape == out.shape and heads * dh == width and cache.device == at
    assert lengths.numel() == n and (starts is None or starts.numel() == n + 1) and group_starts.numel() == groups + 1
    if rows == 0:
        return
    st = _stream_of(stream, at)
    if isinstance(scratch, str):
        room = _scratch_of_stream(at, stream, st, qzo_paged_attention_shared_scratch_bytes(rows, n, heads, cache.kv_heads, dh), "shared")
    else:
        room = _room(scratch, at)
    _check(lib().qzo_paged_attention_shared(x, ldx, rows, n, heads, C.addressof(cache), _at(tables, i32, at), most, _at(lengths, i32, at),
                                            _at(starts, i32, at), groups, _at(group_starts, i32, at), _at(shared, i32, at), scale, y, ldy, *room, st))


def qzo_cache_fork_scratch_bytes(n_seq, n_blocks, max_blocks) -> int:
    out = C.c_uint64(0)
    _check(lib().qzo_cache_fork_scratch_bytes(n_seq, n_blocks, max_blocks, C.addressof(out)))
    return out.value


def _fork_room(scratch, at, stream, st, n, n_blocks, most):
    # the marks in it are one pool's: kept apart by the number of its blocks
    if isinstance(scratch, str):
        return _scratch_of_stream(at, stream, st, qzo_cache_fork_scratch_bytes(n, n_blocks, most), ("fork", n_blocks))
    return _room(scratch, at)


def qzo_cache_fork(parents, block, lengths, tables, free, state, copies, group_starts=None, shared=None, scratch="auto", stream=None):
    """int32 tensors, in place: lengths [n_seq], tables [n_seq, max_blocks], free [n_blocks], state a qzo_cache_state; copies [n_seq, 4] receives
    a qzo_block_copy a row, state[3] of them.  group_starts [n_groups + 1], shared [n_groups]: None, or what it tells of the groups."""
    at, i32, (n, most), groups = torch.cuda.current_device(), torch.int32, tables.shape, 0 if shared is None else shared.numel()
    assert parents.numel() == lengths.numel() == n and state.numel() == 4 and copies.numel() >= 4 * n
    assert (group_starts is None) == (shared is None) and (shared is None or group_starts.numel() == groups + 1)
    st = _stream_of(stream, at)
    room = _fork_room(scratch, at, stream, st, n, free.numel(), most)
    _check(lib().qzo_cache_fork(_at(parents, i32, at), n, block, free.numel(), most, _at(lengths, i32, at), _at(tables, i32, at), _at(free, i32, at),
                                _at(state, i32, at), groups, _at(group_starts, i32, at) if groups else None, _at(shared, i32, at) if groups else None,
                                _at(copies, i32, at), *room, st))


def qzo_cache_compact(block, lengths, tables, free, new_tables, state, copies, scratch="auto", stream=None):
    """int32 tensors as for qzo_cache_fork; new_tables may be tables; copies [at least n_blocks // 2, 4]."""
    at, i32, (n, most) = torch.cuda.current_device(), torch.int32, tables.shape
    assert lengths.numel() == n and new_tables.shape == tables.shape and state.numel() == 4 and copies.numel() >= free.numel() // 2 * 4
    st = _stream_of(stream, at)
    room = _fork_room(scratch, at, stream, st, n, free.numel(), most)
    _check(lib().qzo_cache_compact(n, block, free.numel(), most, _at(lengths, i32, at), _at(tables, i32, at), _at(new_tables, i32, at), _at(free, i32, at),
                                   _at(state, i32, at), _at(copies, i32, at), *room, st))


def qzo_cache_copy(cache, copies, layers=1, count=None, stream=None):
    """copies int32 [n, 4], a qzo_block_copy a row, with count only the first count[3] of them: count is the qzo_cache_state that came with the
    list, or one number.  cache: of layer 0, the other layers' pools behind it."""
    at = torch.cuda.current_device()
    assert cache.device == at and copies.shape[-1] == 4
    n, where = copies.numel() // 4, _at(count, torch.int32, at)
    if where is not None and count.numel() == 4:
        where += 12                             # n_taken
    if n:
        _check(lib().qzo_cache_copy(C.addressof(cache), layers, _at(copies, torch.int32, at), n, where, _stream_of(stream, at)))


def qzo_beam_select_scratch_bytes(n_groups, width, vocab) -> int:
    out = C.c_uint64(0)
    _check(lib().qzo_beam_select_scratch_bytes(n_groups, width, vocab, C.addressof(out)))
    return out.value


def qzo_beam_select(logits, width, scores, counts, ended, history, parents, chosen, tokens, added, end_token=-1, length_penalty=0.0, scratch="auto",
                    stream=None):
    """logits bf16 [n_groups * width, vocab], rows may be strided; scores fp32, counts, ended, parents, chosen, tokens, added int32 [rows]; history
    int32 [rows, max_history] or None."""
    at, i32, (rows, vocab) = torch.cuda.current_device(), torch.int32, logits.shape
    x, ld = _rows(logits, at)
    assert rows % width == 0 and scores.numel() == counts.numel() == ended.numel() == parents.numel() == chosen.numel() == tokens.numel() == added.numel() == rows
    most = 0 if history is None else history.numel() // rows
    assert history is None or history.shape == (rows, most)
    st = _stream_of(stream, at)
    if isinstance(scratch, str):
        room = _scratch_of_stream(at, stream, st, qzo_beam_select_scratch_bytes(rows // width, width, vocab), "beams")
    else:
        room = _room(scratch, at)
    _check(lib().qzo_beam_select(x, ld, rows // width, width, vocab, end_token, length_penalty, _at(scores, torch.float32, at), _at(counts, i32, at),
                                 _at(ended, i32, at), _at(history, i32, at) if most else None, most, _at(parents, i32, at), _at(chosen, i32, at),
                                 _at(tokens, i32, at), _at(added, i32, at), *room, st))


def qzo_answer_workspace_bytes(model, n_tokens, n_seq, shared=False) -> int:
    out = C.c_uint64(0)
    call = lib().qzo_answer_shared_workspace_bytes if shared else lib().qzo_answer_workspace_bytes
    _check(call(model, C.c_uint32(n_tokens), C.c_uint32(n_seq), C.byref(out)))
    return out.value


def qzo_answer(model, tokens, cache, tables, lengths, starts, slots, positions, workspace, logits, stream=None, group_starts=None, shared=None):
    """tokens int32 [n_tokens]; cache: of layer 0, the other layers' pools behind it; logits bf16 [n_seq, vocab].  With group_starts [n_groups + 1] and
    shared [n_groups] it is qzo_answer_shared, whose workspace it then needs."""
    i32, (n, most) = torch.int32, tables.shape
    assert lengths.numel() == n and starts.numel() == n + 1 and slots.numel() >= tokens.numel() <= positions.numel() and logits.shape[0] == n
    at = torch.cuda.current_device()
    assert cache.device == at and (group_starts is None) == (shared is None)
    args = [model, _at(tokens, i32, at), tokens.numel(), n, C.addressof(cache), _at(tables, i32, at), most, _at(lengths, i32, at),
            _at(starts, i32, at), _at(slots, i32, at), _at(positions, i32, at)]
    rest = [*_room(workspace, at), _at(logits, torch.bfloat16, at), _stream_of(stream, at)]
    if shared is None:
        _check(lib().qzo_answer(*args, *rest))
        return
    assert group_starts.numel() == shared.numel() + 1
    _check(lib().qzo_answer_shared(*args, shared.numel(), _at(group_starts, i32, at), _at(shared, i32, at), *rest))
