"""ctypes binding over the C ABI in include/hidet_mi355x.h -- argument marshalling only.

Every function here has the name of the C entry point it forwards to.  Tensors are torch tensors on
the GPU; torch is used for device memory and the current HIP stream, nothing else.  There is no
fallback: if libhidet_mi355x.so has not been built, or a call returns a non-zero status, an
exception is raised.
"""
import ctypes
import importlib.machinery
import importlib.util
import os
import sys

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libhidet_mi355x.so")
HOST_CALLS_PATH = os.path.join(HERE, "_host_calls.so")

HIDET_F32, HIDET_F16, HIDET_BF16 = 0, 1, 2
HIDET_CONV_GATHER, HIDET_CONV_BATCHED, HIDET_CONV_IMAGES, HIDET_CONV_PATCH_64, HIDET_CONV_PATCH_128 = 0, 1, 2, 3, 4
HIDET_BIAS_NONE, HIDET_BIAS_PER_COL, HIDET_BIAS_PER_ROW = 0, 1, 2
HIDET_ACT_NONE, HIDET_ACT_RELU = 0, 1
HIDET_MAP_PLAIN, HIDET_MAP_HEAD_SPLIT = 0, 1
HIDET_PROLOGUE_NONE, HIDET_PROLOGUE_RELU = 0, 1
HIDET_REDUCE_SUM, HIDET_REDUCE_MAX, HIDET_REDUCE_MEAN = 0, 1, 2
HIDET_ROPE_PLAIN, HIDET_ROPE_LINEAR, HIDET_ROPE_BASE, HIDET_ROPE_BANDS = 0, 1, 2, 3

_DTYPES = {torch.float32: HIDET_F32, torch.float16: HIDET_F16, torch.bfloat16: HIDET_BF16}

_i32, _i64, _vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p


class hidet_epilogue_t(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_uint32),
        ("alpha", ctypes.c_float),
        ("bias", _vp),
        ("bias_axis", _i32),
        ("act", _i32),
        ("residual", _vp),
        ("ld_residual", _i64),
        ("batch_stride_residual", _i64),
        ("out_map", _i32),
        ("prologue", _i32),
        ("map_seq", _i64),
        ("map_head_dim", _i64),
    ]


class hidet_config_info_t(ctypes.Structure):
    _fields_ = [(n, _i32) for n in ("block_m", "block_n", "block_k", "waves_m", "waves_n", "mfma", "is_f32", "schedule",
                                    "stages", "lds_bytes", "waves_k")]


class hidet_row_schedule_t(ctypes.Structure):
    _fields_ = [(n, _i32) for n in ("form", "threads_per_row", "chunks_per_thread", "workgroup_size")] + [
        ("workgroups", _i64), ("launches", _i64)]


class hidet_heads_t(ctypes.Structure):
    _fields_ = [("data", _vp), ("stride_batch", _i64), ("stride_head", _i64), ("stride_row", _i64)]


class hidet_attention_options_t(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("causal", _i32), ("scale", ctypes.c_float), ("softcap", ctypes.c_float),
                ("window", _i64), ("slopes", _vp), ("ranges", _vp)]


class hidet_cache_t(ctypes.Structure):
    _fields_ = [("struct_size", ctypes.c_uint32), ("dtype", _i32), ("k", _vp), ("v", _vp)] + [
        (n, _i64) for n in ("num_pages", "page_size", "heads", "head_dim", "stride_page", "stride_slot", "stride_head")] + [
        ("tables", _vp), ("table_width", _i64), ("table_stride", _i64), ("lengths", _vp), ("seqs", _i64)]


class HidetError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__("%s: status %d (%s)" % (where, status, lib().hidet_status_string(status).decode()))


EXPORTS = (
    "hidet_gemm", "hidet_batched_gemm", "hidet_conv2d_implicit_gemm", "hidet_gemm_cfg", "hidet_batched_gemm_cfg",
    "hidet_conv2d_implicit_gemm_cfg", "hidet_config_count", "hidet_config_info", "hidet_tune_gemm", "hidet_tune_conv2d",
    "hidet_tune_last_times", "hidet_tune_clear", "hidet_tune_save", "hidet_tune_load", "hidet_taskmap_count",
    "hidet_taskmap_info", "hidet_taskmap_tasks", "hidet_block_task", "hidet_status_string", "hidet_version",
    "hidet_kernel_launch_count", "hidet_probe_stream_bandwidth",
    "hidet_probe_mfma_peak", "hidet_probe_scratch_bytes", "hidet_probe_launch_floor", "hidet_splitk_workspace_bytes", "hidet_batched_gemm_splitk",
    "hidet_conv2d_implicit_gemm_splitk", "hidet_tune_gemm_splitk", "hidet_tune_conv2d_splitk", "hidet_reduce_rows",
    "hidet_softmax_rows", "hidet_host_div", "hidet_conv2d_splitk_workspace_bytes", "hidet_static_scratch_bytes",
    "hidet_batched_gemm_splitk_static", "hidet_conv2d_pack_weights", "hidet_conv2d_implicit_gemm_packed",
    "hidet_tune_conv2d_packed", "hidet_row_schedule", "hidet_conv2d_untuned_config",
    "hidet_gemm_untuned_config", "hidet_conv2d_patch_rows", "hidet_conv2d_untuned_form", "hidet_attention",
    "hidet_attention_workspace_bytes", "hidet_attention_backward", "hidet_attention_backward_workspace_bytes",
    "hidet_attention_ranges", "hidet_rope", "hidet_rope_frequencies", "hidet_cache_append", "hidet_cache_attention",
    "hidet_cache_attention_workspace_bytes",
)

_lib = None


def lib():
    """The loaded shared library.  Raises if it has not been built (python -m paper_2210_09603_amd.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("HIP extension missing: %s (build it with `python -m paper_2210_09603_amd.build`)" % LIB_PATH)
        L = ctypes.CDLL(LIB_PATH)
        ep = ctypes.POINTER(hidet_epilogue_t)
        gemm_args = [_i32, _i32, _i32, _i32, _i64, _i64, _i64, _vp, _i64, _vp, _i64, _vp, _i64, ep, _vp]
        bgemm_args = [_i32, _i32, _i32, _i32, _i64, _i64, _i64, _i64, _vp, _i64, _i64, _vp, _i64, _i64, _vp, _i64, _i64,
                      ep, _vp]
        conv_args = [_i32, _i32] + [_i64] * 11 + [_vp, _vp, _vp, ep, _vp]
        L.hidet_gemm.argtypes = gemm_args
        L.hidet_gemm_cfg.argtypes = [_i32] + gemm_args
        L.hidet_batched_gemm.argtypes = bgemm_args
        L.hidet_batched_gemm_cfg.argtypes = [_i32] + bgemm_args
        L.hidet_conv2d_implicit_gemm.argtypes = conv_args
        L.hidet_conv2d_implicit_gemm_cfg.argtypes = [_i32] + conv_args
        tune_tail = [_i32, ctypes.POINTER(_i32), ctypes.POINTER(ctypes.c_float)]
        L.hidet_tune_gemm.argtypes = bgemm_args + tune_tail
        L.hidet_tune_conv2d.argtypes = conv_args + tune_tail
        L.hidet_splitk_workspace_bytes.argtypes = [_i64, _i64, _i64, _i32]
        L.hidet_splitk_workspace_bytes.restype = _i64
        L.hidet_conv2d_splitk_workspace_bytes.argtypes = [_i64, _i64, _i64, _i64, _i32]
        L.hidet_conv2d_splitk_workspace_bytes.restype = _i64
        L.hidet_static_scratch_bytes.restype = _i64
        L.hidet_batched_gemm_splitk_static.argtypes = [_i32, _i32] + bgemm_args
        ws_args = [_vp, _i64, _vp]  # workspace, bytes, stream (replaces the trailing stream argument)
        L.hidet_batched_gemm_splitk.argtypes = [_i32, _i32] + bgemm_args[:-1] + ws_args
        L.hidet_conv2d_implicit_gemm_splitk.argtypes = [_i32, _i32] + conv_args[:-1] + ws_args
        tune_tail_sk = [_i32, ctypes.POINTER(_i32), ctypes.POINTER(_i32), ctypes.POINTER(ctypes.c_float)]
        L.hidet_conv2d_pack_weights.argtypes = [_i32, _i64, _i64, _i64, _i64, _vp, _vp, _vp]
        L.hidet_conv2d_implicit_gemm_packed.argtypes = [_i32, _i32] + conv_args[:-1] + ws_args
        L.hidet_tune_conv2d_packed.argtypes = conv_args[:-1] + ws_args + tune_tail_sk
        L.hidet_tune_gemm_splitk.argtypes = bgemm_args[:-1] + ws_args + tune_tail_sk
        L.hidet_tune_conv2d_splitk.argtypes = conv_args[:-1] + ws_args + tune_tail_sk
        L.hidet_host_div.argtypes = [_i64, _i32, ctypes.POINTER(_i32)]
        L.hidet_reduce_rows.argtypes = [_i32, _i32, _i32, _i64, _i64, _vp, _i64, _vp, _vp]
        L.hidet_softmax_rows.argtypes = [_i32, _i64, _i64, _vp, _i64, _vp, _i64, _vp]
        L.hidet_conv2d_untuned_config.argtypes = [_i32] + [_i64] * 11 + [_i32, ctypes.POINTER(_i32)]
        L.hidet_conv2d_untuned_form.argtypes = [_i32] + [_i64] * 11 + [ctypes.POINTER(_i32)]
        L.hidet_conv2d_patch_rows.argtypes = [_i32] + [_i64] * 11 + [ctypes.POINTER(_i32)]
        L.hidet_gemm_untuned_config.argtypes = [_i32, _i32, _i32] + [_i64] * 4 + [ctypes.POINTER(_i32)]
        L.hidet_row_schedule.argtypes = [_i32, _i32, _i64, _i64, ctypes.POINTER(hidet_row_schedule_t)]
        L.hidet_tune_last_times.argtypes = [ctypes.POINTER(ctypes.c_float), _i32]
        L.hidet_tune_clear.restype = None
        L.hidet_tune_save.argtypes = [ctypes.c_char_p]
        L.hidet_tune_load.argtypes = [ctypes.c_char_p]
        L.hidet_config_info.argtypes = [_i32, ctypes.POINTER(hidet_config_info_t)]
        L.hidet_taskmap_info.argtypes = [_i32, ctypes.c_char_p, _i32] + [ctypes.POINTER(_i32)] * 4
        L.hidet_taskmap_tasks.argtypes = [_i32, _i32, ctypes.POINTER(_i32), _i32]
        L.hidet_block_task.argtypes = [_i32] * 4 + [ctypes.POINTER(_i32)] * 2
        L.hidet_probe_mfma_peak.argtypes = [_i32, _i32, _vp, _i64, _vp, _i64, _vp, ctypes.POINTER(ctypes.c_float),
                                            ctypes.POINTER(ctypes.c_float)]
        L.hidet_probe_scratch_bytes.restype = _i64
        L.hidet_probe_launch_floor.argtypes = [_vp, _i32, ctypes.POINTER(ctypes.c_float)]
        L.hidet_probe_stream_bandwidth.argtypes = [_vp, _i64, _i32, _vp, ctypes.POINTER(ctypes.c_float)]
        hp, op, cp = ctypes.POINTER(hidet_heads_t), ctypes.POINTER(hidet_attention_options_t), ctypes.POINTER(hidet_cache_t)
        L.hidet_attention.argtypes = [_i32] + [_i64] * 6 + [hp] * 4 + [_vp, op, _vp, _i64, _vp]
        L.hidet_attention_workspace_bytes.argtypes = [_i64] * 6
        L.hidet_attention_workspace_bytes.restype = _i64
        L.hidet_attention_backward.argtypes = [_i32] + [_i64] * 6 + [hp] * 5 + [_vp] + [hp] * 3 + [op, _vp, _i64, _vp]
        L.hidet_attention_backward_workspace_bytes.argtypes = [_i64] * 6
        L.hidet_attention_backward_workspace_bytes.restype = _i64
        L.hidet_attention_ranges.argtypes = [_i64] * 3 + [_vp, _vp, _i32, _i64, _vp, _vp]
        L.hidet_rope.argtypes = [_i32] + [_i64] * 5 + [hp, hp, _vp, _vp, _i64, _i64, _i32, _i32, ctypes.c_float, _vp]
        f64 = ctypes.c_double
        L.hidet_rope_frequencies.argtypes = [_i64, f64, _i32, f64, f64, f64, f64, ctypes.POINTER(f64)]
        L.hidet_cache_append.argtypes = [cp, _i64, _i64, hp, hp, _vp, _vp]
        L.hidet_cache_attention.argtypes = [cp, _i64, _i64, _i64, hp, hp, _vp, _vp, op, _vp, _i64, _vp]
        L.hidet_cache_attention_workspace_bytes.argtypes = [cp, _i64, _i64, _i64]
        L.hidet_cache_attention_workspace_bytes.restype = _i64
        L.hidet_status_string.argtypes = [_i32]
        L.hidet_status_string.restype = ctypes.c_char_p
        L.hidet_version.restype = ctypes.c_char_p
        L.hidet_kernel_launch_count.restype = ctypes.c_int64
        _lib = L
    return _lib


# The plain form of a call goes through an extension module that reads the tensors itself (csrc/host_calls.cpp).  A
# negative answer means that the arguments are not of that form and that nothing was called.
_host_calls = None


def built_for():
    """What an extension module has to have been compiled for to read this process's tensors."""
    return "torch %s, Python %d.%d" % (torch.__version__, sys.version_info[0], sys.version_info[1])


def _host_module():
    if not os.path.exists(HOST_CALLS_PATH):
        raise RuntimeError("host extension missing: %s (build it with `python -m paper_2210_09603_amd.build`)" % HOST_CALLS_PATH)
    loader = importlib.machinery.ExtensionFileLoader("_host_calls", HOST_CALLS_PATH)
    module = importlib.util.module_from_spec(importlib.util.spec_from_loader("_host_calls", loader))
    loader.exec_module(module)
    if module.built_for != built_for():
        raise RuntimeError("host extension %s was built for %s, this is %s (run `python -m paper_2210_09603_amd.build`)"
                           % (HOST_CALLS_PATH, module.built_for, built_for()))
    return module


def _of_the_process():
    """What tells a forked process, the current device and its current stream."""
    c = torch._C
    unavailable = lambda *a: None  # (a torch without the GPU: the general path says so)
    return (getattr(c, "_cuda_isInBadFork", unavailable), getattr(c, "_cuda_getDevice", unavailable),
            getattr(c, "_cuda_getCurrentRawStream", unavailable))


def _load_host_calls(L):
    entry = (L.hidet_gemm_cfg, L.hidet_batched_gemm_cfg, L.hidet_conv2d_implicit_gemm_cfg,
             L.hidet_conv2d_implicit_gemm_packed, L.hidet_softmax_rows, L.hidet_reduce_rows)
    return _host_module().Calls(tuple(ctypes.cast(f, _vp).value for f in entry), hidet_epilogue_t, *_of_the_process())


def _load_attention_calls(L):
    entry = (L.hidet_attention, L.hidet_attention_backward, L.hidet_attention_ranges, L.hidet_rope, L.hidet_cache_append,
             L.hidet_cache_attention)
    return _host_module().AttentionCalls(tuple(ctypes.cast(f, _vp).value for f in entry), hidet_cache_t, *_of_the_process())


def _calls():
    global _host_calls
    if _host_calls is None:
        _host_calls = _load_host_calls(lib())
    return _host_calls


_attention_calls = None


def _attn():
    global _attention_calls
    if _attention_calls is None:
        _attention_calls = _load_attention_calls(lib())
    return _attention_calls


def _check(status, where):
    if status != 0:
        raise HidetError(status, where)


# The helpers of the general path hand plain integers to ctypes (argtypes converts them), read each shape and stride tuple
# once and take the current stream's handle without building a Stream object.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream):
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is not None and torch.cuda.is_initialized():
        return _raw_stream(torch._C._cuda_getDevice())
    return torch.cuda.current_stream().cuda_stream


def _dtype(t):
    d = _DTYPES.get(t.dtype)
    if d is None:
        raise TypeError("unsupported dtype %s" % t.dtype)
    return d


def _ptr(t):
    return t.data_ptr() if t is not None else None


def _ld(t):
    """Leading dimension of a 2-D (or the last two dims of a 3-D) row-major tensor, in elements."""
    n, s = t.shape, t.stride()
    if s[-1] != 1 and n[-1] > 1:
        raise ValueError("innermost dimension must be contiguous")
    return s[-2] if n[-2] > 1 else max(n[-1], 1)


def make_epilogue(alpha=1.0, bias=None, bias_axis=HIDET_BIAS_NONE, residual=None, relu=False, batched=False,
                  head_split=None, relu_input=False):
    """Build a hidet_epilogue_t (returns None for the identity epilogue).  head_split=(seq, head_dim) selects the
    [b][h][s][f] output index map; the residual (if any) is then a dense tensor of that shape.  A 3-D residual
    advances by its own batch stride (`batched` is accepted for older callers and ignored).  relu_input: the fused
    prologue, ReLU on the activation operand (A of a GEMM, x of a convolution) as it is loaded."""
    if alpha == 1.0 and bias is None and residual is None and not relu and head_split is None and not relu_input:
        return None
    e = hidet_epilogue_t()
    e.struct_size = ctypes.sizeof(hidet_epilogue_t)
    e.alpha = alpha
    # the struct holds raw device addresses: keep the tensors alive as long as it lives (an asynchronous kernel
    # reads them after the call has returned)
    e._keep = (bias, residual)
    e.bias = bias.data_ptr() if bias is not None else None
    e.bias_axis = bias_axis if bias is not None else HIDET_BIAS_NONE
    e.act = HIDET_ACT_RELU if relu else HIDET_ACT_NONE
    e.prologue = HIDET_PROLOGUE_RELU if relu_input else HIDET_PROLOGUE_NONE
    if head_split is not None:
        e.out_map = HIDET_MAP_HEAD_SPLIT
        e.map_seq, e.map_head_dim = head_split
    if residual is not None:
        e.residual = residual.data_ptr()
        if head_split is None:
            e.ld_residual = _ld(residual)
            e.batch_stride_residual = residual.stride(0) if (residual.dim() == 3 and residual.shape[0] > 1) else 0
    return e


def _epi_ref(e):
    return ctypes.byref(e) if e is not None else None


def _gemm_dims(A, B, transA, transB):
    a, b = A.shape, B.shape
    M, K = (a[-1], a[-2]) if transA else (a[-2], a[-1])
    Kb, N = (b[-1], b[-2]) if transB else (b[-2], b[-1])
    if K != Kb:
        raise ValueError("inner dimensions differ: %d vs %d" % (K, Kb))
    return M, N, K


def hidet_gemm(A, B, C, transA=False, transB=False, epilogue=None, stream=None, config=-1):
    """C[M,N] = epilogue(op(A) . op(B)); A, B, C are 2-D GPU tensors (row-major, any leading dimension)."""
    st = (_host_calls or _calls()).gemm(A, B, C, transA, transB, epilogue, stream, config)
    if st < 0:
        _gemm(A, B, C, transA, transB, epilogue, stream, config)
    else:
        _check(st, "hidet_gemm")


def _gemm(A, B, C, transA, transB, epilogue, stream, config):
    M, N, K = _gemm_dims(A, B, transA, transB)
    if epilogue is not None and epilogue.out_map == HIDET_MAP_HEAD_SPLIT:
        want = (M // epilogue.map_seq, N // epilogue.map_head_dim, epilogue.map_seq, epilogue.map_head_dim)
        if tuple(C.shape) != want or not C.is_contiguous():
            raise ValueError("C must be a dense tensor of shape %s" % (want,))
        st = lib().hidet_gemm_cfg(config, _dtype(A), _dtype(C), int(transA), int(transB), M, N, K, _ptr(A), _ld(A), _ptr(B),
                                  _ld(B), _ptr(C), N, _epi_ref(epilogue), _stream(stream))
        _check(st, "hidet_gemm")
        return
    if C.shape != (M, N):
        raise ValueError("C has shape %s, expected %s" % (tuple(C.shape), (M, N)))
    st = lib().hidet_gemm_cfg(config, _dtype(A), _dtype(C), int(transA), int(transB), M, N, K, _ptr(A), _ld(A), _ptr(B),
                              _ld(B), _ptr(C), _ld(C), _epi_ref(epilogue), _stream(stream))
    _check(st, "hidet_gemm")


def _bstride(t):
    n = t.shape
    return t.stride(0) if n[0] > 1 else n[-2] * _ld(t)


def hidet_batched_gemm(A, B, C, transA=False, transB=False, epilogue=None, stream=None, config=-1):
    """Batched form: A, B, C are 3-D GPU tensors [batch, rows, cols]."""
    st = (_host_calls or _calls()).batched_gemm(A, B, C, transA, transB, epilogue, stream, config)
    if st < 0:
        _batched_gemm(A, B, C, transA, transB, epilogue, stream, config)
    else:
        _check(st, "hidet_batched_gemm")


def _batched_gemm(A, B, C, transA, transB, epilogue, stream, config):
    M, N, K = _gemm_dims(A, B, transA, transB)
    batch = A.shape[0]
    if B.shape[0] != batch or C.shape != (batch, M, N):
        raise ValueError("batch/shape mismatch")
    st = lib().hidet_batched_gemm_cfg(config, _dtype(A), _dtype(C), int(transA), int(transB), batch, M, N, K, _ptr(A),
                                      _ld(A), _bstride(A), _ptr(B), _ld(B), _bstride(B), _ptr(C), _ld(C), _bstride(C),
                                      _epi_ref(epilogue), _stream(stream))
    _check(st, "hidet_batched_gemm")


def _conv_args(x, w, y, stride, pad):
    for t in (x, w, y):
        if not t.is_contiguous():
            raise ValueError("conv tensors must be dense NCHW / OIHW")
    Nb, IC, H, W = x.shape
    OC, IC2, KH, KW = w.shape
    if IC != IC2:
        raise ValueError("channel mismatch")
    return [_dtype(x), _dtype(y), Nb, IC, H, W, OC, KH, KW, stride[0], stride[1], pad[0], pad[1], _ptr(x), _ptr(w), _ptr(y)]


def conv_out_shape(x_shape, w_shape, stride, pad):
    Nb, _, H, W = x_shape
    OC, _, KH, KW = w_shape
    return (Nb, OC, (H + 2 * pad[0] - KH) // stride[0] + 1, (W + 2 * pad[1] - KW) // stride[1] + 1)


def hidet_conv2d_implicit_gemm(x, w, y, stride=(1, 1), pad=(0, 0), epilogue=None, stream=None, config=-1):
    """y = epilogue(conv2d(x, w)), NCHW / OIHW / NCHW dense GPU tensors; bias (if any) is per output channel."""
    st = (_host_calls or _calls()).conv2d(x, w, y, stride, pad, epilogue, stream, config)
    if st < 0:
        _conv2d(x, w, y, stride, pad, epilogue, stream, config)
    else:
        _check(st, "hidet_conv2d_implicit_gemm")


def _conv2d(x, w, y, stride, pad, epilogue, stream, config):
    if y.shape != conv_out_shape(x.shape, w.shape, stride, pad):
        raise ValueError("y has the wrong shape")
    st = lib().hidet_conv2d_implicit_gemm_cfg(config, *_conv_args(x, w, y, stride, pad), _epi_ref(epilogue),
                                              _stream(stream))
    _check(st, "hidet_conv2d_implicit_gemm")


def hidet_tune_gemm(A, B, C, transA=False, transB=False, epilogue=None, stream=None, iters=10):
    """Enumerate the schedule space on this (possibly batched) problem; returns (best_config, best_us)."""
    if A.dim() == 2:
        A, B, C = A.unsqueeze(0), B.unsqueeze(0), C.unsqueeze(0)
    M, N, K = _gemm_dims(A, B, transA, transB)
    batch = A.shape[0]
    best, us = _i32(-1), ctypes.c_float(0.0)
    st = lib().hidet_tune_gemm(_dtype(A), _dtype(C), int(transA), int(transB), batch, M, N, K, _ptr(A), _ld(A),
                               _bstride(A), _ptr(B), _ld(B), _bstride(B), _ptr(C), _ld(C), _bstride(C),
                               _epi_ref(epilogue), _stream(stream), iters, ctypes.byref(best), ctypes.byref(us))
    _check(st, "hidet_tune_gemm")
    return best.value, us.value


def hidet_tune_conv2d(x, w, y, stride=(1, 1), pad=(0, 0), epilogue=None, stream=None, iters=10):
    best, us = _i32(-1), ctypes.c_float(0.0)
    st = lib().hidet_tune_conv2d(*_conv_args(x, w, y, stride, pad), _epi_ref(epilogue), _stream(stream), iters,
                                 ctypes.byref(best), ctypes.byref(us))
    _check(st, "hidet_tune_conv2d")
    return best.value, us.value


def hidet_splitk_workspace_bytes(batch, M, N, k_slices):
    return lib().hidet_splitk_workspace_bytes(batch, M, N, k_slices)


def hidet_conv2d_splitk_workspace_bytes(y_shape, k_slices):
    """Workspace bytes of the K-parallel convolution that produces y [Nb, OC, OH, OW]."""
    Nb, OC, OH, OW = y_shape
    return lib().hidet_conv2d_splitk_workspace_bytes(Nb, OC, OH, OW, k_slices)


def hidet_static_scratch_bytes():
    return lib().hidet_static_scratch_bytes()


def hidet_batched_gemm_splitk_static(A, B, C, k_slices=0, transA=False, transB=False, epilogue=None, stream=None, config=-1):
    """hidet_batched_gemm_splitk with the library's static scratch array as the workspace (allocates nothing)."""
    if A.dim() == 2:
        A, B, C = A.unsqueeze(0), B.unsqueeze(0), C.unsqueeze(0)
    M, N, K = _gemm_dims(A, B, transA, transB)
    batch = A.shape[0]
    if B.shape[0] != batch or C.shape != (batch, M, N):
        raise ValueError("batch/shape mismatch")
    st = lib().hidet_batched_gemm_splitk_static(config, k_slices, _dtype(A), _dtype(C), int(transA), int(transB), batch, M, N,
                                                K, _ptr(A), _ld(A), _bstride(A), _ptr(B), _ld(B), _bstride(B), _ptr(C),
                                                _ld(C), _bstride(C), _epi_ref(epilogue), _stream(stream))
    _check(st, "hidet_batched_gemm_splitk_static")


def _ws(workspace):
    """(pointer, bytes) of a workspace tensor (any dtype, contiguous) or (NULL, 0)."""
    if workspace is None:
        return None, 0
    return _ptr(workspace), workspace.numel() * workspace.element_size()


def hidet_batched_gemm_splitk(A, B, C, workspace, k_slices=0, transA=False, transB=False, epilogue=None, stream=None,
                              config=-1):
    """K-parallel form of hidet_batched_gemm (2-D tensors are taken as batch 1); workspace is a GPU tensor."""
    if A.dim() == 2:
        A, B, C = A.unsqueeze(0), B.unsqueeze(0), C.unsqueeze(0)
    M, N, K = _gemm_dims(A, B, transA, transB)
    batch = A.shape[0]
    if B.shape[0] != batch or C.shape != (batch, M, N):
        raise ValueError("batch/shape mismatch")
    wp, wb = _ws(workspace)
    st = lib().hidet_batched_gemm_splitk(config, k_slices, _dtype(A), _dtype(C), int(transA), int(transB), batch, M, N, K,
                                         _ptr(A), _ld(A), _bstride(A), _ptr(B), _ld(B), _bstride(B), _ptr(C), _ld(C),
                                         _bstride(C), _epi_ref(epilogue), wp, wb, _stream(stream))
    _check(st, "hidet_batched_gemm_splitk")


def hidet_conv2d_implicit_gemm_splitk(x, w, y, workspace, k_slices=0, stride=(1, 1), pad=(0, 0), epilogue=None,
                                      stream=None, config=-1):
    """K-parallel form of hidet_conv2d_implicit_gemm; workspace is a GPU tensor."""
    if y.shape != conv_out_shape(x.shape, w.shape, stride, pad):
        raise ValueError("y has the wrong shape")
    wp, wb = _ws(workspace)
    st = lib().hidet_conv2d_implicit_gemm_splitk(config, k_slices, *_conv_args(x, w, y, stride, pad), _epi_ref(epilogue),
                                                 wp, wb, _stream(stream))
    _check(st, "hidet_conv2d_implicit_gemm_splitk")


def hidet_conv2d_pack_weights(w, w_packed=None, stream=None):
    """OIHW weights -> the tap-major order [OC][KH][KW][IC] of the packed convolution; returns the packed tensor."""
    if not w.is_contiguous():
        raise ValueError("weights must be dense OIHW")
    OC, IC, KH, KW = w.shape
    if w_packed is None:
        w_packed = torch.empty((OC, KH, KW, IC), dtype=w.dtype, device=w.device)
    if w_packed.numel() != w.numel() or not w_packed.is_contiguous() or w_packed.dtype != w.dtype:
        raise ValueError("w_packed must be a dense tensor of the same dtype and element count")
    _check(lib().hidet_conv2d_pack_weights(_dtype(w), OC, IC, KH, KW, _ptr(w), _ptr(w_packed), _stream(stream)),
           "hidet_conv2d_pack_weights")
    return w_packed


def _packed_conv_args(x, w_packed, y, stride, pad):
    for t in (x, w_packed, y):
        if not t.is_contiguous():
            raise ValueError("conv tensors must be dense")
    Nb, IC, H, W = x.shape
    OC, KH, KW, IC2 = w_packed.shape
    if IC != IC2:
        raise ValueError("channel mismatch")
    if y.shape != conv_out_shape(x.shape, (OC, IC, KH, KW), stride, pad):
        raise ValueError("y has the wrong shape")
    return [_dtype(x), _dtype(y), Nb, IC, H, W, OC, KH, KW, stride[0], stride[1], pad[0], pad[1], _ptr(x), _ptr(w_packed),
            _ptr(y)]


def hidet_conv2d_implicit_gemm_packed(x, w_packed, y, stride=(1, 1), pad=(0, 0), epilogue=None, stream=None, config=-1,
                                      k_slices=0, workspace=None):
    """The convolution from weights repacked by hidet_conv2d_pack_weights ([OC][KH][KW][IC])."""
    st = -1
    if workspace is None:
        st = (_host_calls or _calls()).conv2d_packed(x, w_packed, y, stride, pad, epilogue, stream, config, k_slices)
    if st < 0:
        _conv2d_packed(x, w_packed, y, stride, pad, epilogue, stream, config, k_slices, workspace)
    else:
        _check(st, "hidet_conv2d_implicit_gemm_packed")


def _conv2d_packed(x, w_packed, y, stride, pad, epilogue, stream, config, k_slices, workspace):
    wp, wb = _ws(workspace)
    st = lib().hidet_conv2d_implicit_gemm_packed(config, k_slices, *_packed_conv_args(x, w_packed, y, stride, pad),
                                                 _epi_ref(epilogue), wp, wb, _stream(stream))
    _check(st, "hidet_conv2d_implicit_gemm_packed")


def hidet_tune_conv2d_packed(x, w_packed, y, workspace=None, stride=(1, 1), pad=(0, 0), epilogue=None, stream=None, iters=10):
    best, sl, us = _i32(-1), _i32(1), ctypes.c_float(0.0)
    wp, wb = _ws(workspace)
    st = lib().hidet_tune_conv2d_packed(*_packed_conv_args(x, w_packed, y, stride, pad), _epi_ref(epilogue), wp, wb,
                                        _stream(stream), iters, ctypes.byref(best), ctypes.byref(sl), ctypes.byref(us))
    _check(st, "hidet_tune_conv2d_packed")
    return best.value, sl.value, us.value


def hidet_tune_gemm_splitk(A, B, C, workspace, transA=False, transB=False, epilogue=None, stream=None, iters=10):
    """Enumerate configurations x slice counts; returns (best_config, best_slices, best_us)."""
    if A.dim() == 2:
        A, B, C = A.unsqueeze(0), B.unsqueeze(0), C.unsqueeze(0)
    M, N, K = _gemm_dims(A, B, transA, transB)
    batch = A.shape[0]
    best, sl, us = _i32(-1), _i32(1), ctypes.c_float(0.0)
    wp, wb = _ws(workspace)
    st = lib().hidet_tune_gemm_splitk(_dtype(A), _dtype(C), int(transA), int(transB), batch, M, N, K, _ptr(A), _ld(A),
                                      _bstride(A), _ptr(B), _ld(B), _bstride(B), _ptr(C), _ld(C), _bstride(C),
                                      _epi_ref(epilogue), wp, wb, _stream(stream), iters, ctypes.byref(best),
                                      ctypes.byref(sl), ctypes.byref(us))
    _check(st, "hidet_tune_gemm_splitk")
    return best.value, sl.value, us.value


def hidet_tune_conv2d_splitk(x, w, y, workspace, stride=(1, 1), pad=(0, 0), epilogue=None, stream=None, iters=10):
    best, sl, us = _i32(-1), _i32(1), ctypes.c_float(0.0)
    wp, wb = _ws(workspace)
    st = lib().hidet_tune_conv2d_splitk(*_conv_args(x, w, y, stride, pad), _epi_ref(epilogue), wp, wb, _stream(stream),
                                        iters, ctypes.byref(best), ctypes.byref(sl), ctypes.byref(us))
    _check(st, "hidet_tune_conv2d_splitk")
    return best.value, sl.value, us.value


def _rows_view(t):
    """[..., cols] tensor whose leading axes collapse to one row axis with a single stride -> (rows, cols, ld)."""
    if t.dim() < 1:
        raise ValueError("need at least one axis")
    if t.dim() == 1:
        return 1, t.shape[0], max(t.shape[0], 1)
    v = t if t.dim() == 2 else (t.view(-1, t.shape[-1]) if t.is_contiguous() else None)
    if v is None:
        raise ValueError("leading axes must be collapsible (pass a 2-D view)")
    return v.shape[0], v.shape[1], _ld(v)


def hidet_reduce_rows(x, y, op=HIDET_REDUCE_SUM, stream=None):
    """y[i] = reduce over the last axis of x; y has one element per row, dtype of x or float32."""
    st = (_host_calls or _calls()).reduce_rows(x, y, op, stream)
    if st < 0:
        _reduce_rows(x, y, op, stream)
    else:
        _check(st, "hidet_reduce_rows")


def _reduce_rows(x, y, op, stream):
    rows, cols, ld = _rows_view(x)
    if y.numel() != rows or not y.is_contiguous():
        raise ValueError("y must be a dense tensor with one element per row")
    st = lib().hidet_reduce_rows(_dtype(x), _dtype(y), op, rows, cols, _ptr(x), ld, _ptr(y), _stream(stream))
    _check(st, "hidet_reduce_rows")


def hidet_softmax_rows(x, y, stream=None):
    """y = softmax of x along the last axis (same shape and dtype; y may be x itself)."""
    st = (_host_calls or _calls()).softmax_rows(x, y, stream)
    if st < 0:
        _softmax_rows(x, y, stream)
    else:
        _check(st, "hidet_softmax_rows")


def _softmax_rows(x, y, stream):
    if x.shape != y.shape or x.dtype != y.dtype:
        raise ValueError("x and y must agree in shape and dtype")
    rows, cols, ldx = _rows_view(x)
    _, _, ldy = _rows_view(y)
    st = lib().hidet_softmax_rows(_dtype(x), rows, cols, _ptr(x), ldx, _ptr(y), ldy, _stream(stream))
    _check(st, "hidet_softmax_rows")


# ---- attention, its positions and its cache ---------------------------------------------------------------------------
# These run on the device that their tensors are on, whichever is current: on `stream`, or on that device's current stream.
def _on(tensors, stream):
    """(context that makes the tensors' device current, stream handle)."""
    device = None
    for t in tensors:
        if t is None:
            continue
        if t.device.type != "cuda":
            raise ValueError("tensors must be on the GPU")
        if device is None:
            device = t.device
        elif t.device != device:
            raise ValueError("tensors are on different devices")
    if stream is not None:
        return torch.cuda.device(device), stream.cuda_stream
    return torch.cuda.device(device), torch.cuda.current_stream(device).cuda_stream


def _heads(t):
    """hidet_heads_t of a [batch, heads, rows, head_dim] tensor, or of [rows, heads, head_dim]."""
    s = t.stride()
    if s[-1] != 1 and t.shape[-1] > 1:
        raise ValueError("the last dimension must be contiguous")
    if t.dim() == 4:
        return hidet_heads_t(t.data_ptr(), s[0], s[1], s[2])
    return hidet_heads_t(t.data_ptr(), 0, s[1], s[0])


def _whole32(t, shape, what):
    """Address of a dense int32 tensor of that shape, or None."""
    if t is None:
        return None
    if t.dtype != torch.int32 or tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise ValueError("%s must be a dense int32 tensor of shape %s" % (what, tuple(shape)))
    return t.data_ptr()


def _float32(t, shape, what):
    if t is None:
        return None
    if t.dtype != torch.float32 or tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise ValueError("%s must be a dense float32 tensor of shape %s" % (what, tuple(shape)))
    return t.data_ptr()


def _dense_ws(workspace):
    """_ws() of a workspace that is checked: all of its bytes are written to."""
    if workspace is not None and not workspace.is_contiguous():
        raise ValueError("the workspace must be a dense tensor")
    return _ws(workspace)


def _options(scale, head_dim, causal, window, softcap, slopes, ranges, heads, ranges_shape):
    o = hidet_attention_options_t()
    o.struct_size = ctypes.sizeof(hidet_attention_options_t)
    o.causal, o.window, o.softcap = int(causal), window, softcap
    o.scale = head_dim ** -0.5 if scale is None else scale
    o.slopes = _float32(slopes, (heads,), "slopes")
    o.ranges = _whole32(ranges, ranges_shape, "ranges")
    return o


def _attention_shapes(q, k, v, *like_q):
    if q.dim() != 4 or k.dim() != 4 or k.shape != v.shape or k.shape[0] != q.shape[0] or k.shape[3] != q.shape[3]:
        raise ValueError("need q [batch, heads, seq_q, head_dim] and k, v [batch, kv_heads, seq_k, head_dim]")
    for t in like_q:
        if t.shape != q.shape:
            raise ValueError("expected shape %s, got %s" % (tuple(q.shape), tuple(t.shape)))
    for t in (k, v) + like_q:
        if t.dtype != q.dtype:
            raise ValueError("tensors must agree in dtype")
    batch, heads, seq_q, dim = q.shape
    return batch, heads, k.shape[1], seq_q, k.shape[2], dim


def hidet_attention(q, k, v, out, lse=None, scale=None, causal=False, window=0, softcap=0.0, slopes=None, ranges=None,
                    workspace=None, stream=None):
    """out = softmax(scores(q, k)) . v; q, out [batch, heads, seq_q, head_dim], k, v [batch, kv_heads, seq_k, head_dim], any
    strides with a contiguous last dimension.  scale: head_dim ** -0.5 if None.  lse [batch, heads, seq_q] float32 is written where
    given.  ranges [batch, seq_q, 2] int32 (hidet_attention_ranges) stands in for causal and window."""
    st = (_attention_calls or _attn()).attention(q, k, v, out, lse, scale, causal, window, softcap, slopes, ranges, workspace, stream)
    if st < 0:
        _attention(q, k, v, out, lse, scale, causal, window, softcap, slopes, ranges, workspace, stream)
    else:
        _check(st, "hidet_attention")


def _attention(q, k, v, out, lse, scale, causal, window, softcap, slopes, ranges, workspace, stream):
    sizes = _attention_shapes(q, k, v, out)
    batch, heads, _, seq_q, _, dim = sizes
    o = _options(scale, dim, causal, window, softcap, slopes, ranges, heads, (batch, seq_q, 2))
    wp, wb = _dense_ws(workspace)
    device, handle = _on((q, k, v, out, lse, slopes, ranges, workspace), stream)
    with device:
        st = lib().hidet_attention(_dtype(q), *sizes, _heads(q), _heads(k), _heads(v), _heads(out),
                                   _float32(lse, (batch, heads, seq_q), "lse"), o, wp, wb, handle)
    _check(st, "hidet_attention")


def hidet_attention_workspace_bytes(q, k):
    """Workspace bytes of hidet_attention on these tensors (0: none is wanted)."""
    return lib().hidet_attention_workspace_bytes(q.shape[0], q.shape[1], k.shape[1], q.shape[2], k.shape[2], q.shape[3])


def hidet_attention_backward(grad_out, q, k, v, out, lse, grad_q, grad_k, grad_v, workspace, scale=None, causal=False, window=0,
                             softcap=0.0, slopes=None, ranges=None, stream=None):
    """Writes the gradients of q, k and v from that of out, with the options, out and lse of the forward call."""
    st = (_attention_calls or _attn()).attention_backward(grad_out, q, k, v, out, lse, grad_q, grad_k, grad_v, workspace, scale,
                                                            causal, window, softcap, slopes, ranges, stream)
    if st < 0:
        _attention_backward(grad_out, q, k, v, out, lse, grad_q, grad_k, grad_v, workspace, scale, causal, window, softcap, slopes, ranges,
                            stream)
    else:
        _check(st, "hidet_attention_backward")


def _attention_backward(grad_out, q, k, v, out, lse, grad_q, grad_k, grad_v, workspace, scale, causal, window, softcap, slopes,
                        ranges, stream):
    sizes = _attention_shapes(q, k, v, grad_out, out, grad_q)
    batch, heads, _, seq_q, _, dim = sizes
    for t in (grad_k, grad_v):
        if t.shape != k.shape or t.dtype != q.dtype:
            raise ValueError("grad_k and grad_v must agree with k in shape and dtype")
    o = _options(scale, dim, causal, window, softcap, slopes, ranges, heads, (batch, seq_q, 2))
    wp, wb = _dense_ws(workspace)
    device, handle = _on((grad_out, q, k, v, out, lse, grad_q, grad_k, grad_v, slopes, ranges, workspace), stream)
    with device:
        st = lib().hidet_attention_backward(_dtype(q), *sizes, _heads(grad_out), _heads(q), _heads(k), _heads(v), _heads(out),
                                            _float32(lse, (batch, heads, seq_q), "lse"), _heads(grad_q), _heads(grad_k),
                                            _heads(grad_v), o, wp, wb, handle)
    _check(st, "hidet_attention_backward")


def hidet_attention_backward_workspace_bytes(q, k):
    """Workspace bytes of hidet_attention_backward on these tensors."""
    return lib().hidet_attention_backward_workspace_bytes(q.shape[0], q.shape[1], k.shape[1], q.shape[2], k.shape[2], q.shape[3])


def hidet_attention_ranges(ranges, keys=None, documents=None, prefix=None, causal=False, window=0, stream=None):
    """Fills ranges [batch, seq_q, 2] (int32) with the keys that every query sees: documents [batch, keys] int32 (runs of equal
    numbers, negative: padding), prefix [batch] int32; `keys`: their number, the documents' or seq_q if None."""
    if keys is None:
        keys = (ranges if documents is None else documents).shape[1]
    st = (_attention_calls or _attn()).attention_ranges(ranges, keys, documents, prefix, causal, window, stream)
    if st < 0:
        _attention_ranges(ranges, keys, documents, prefix, causal, window, stream)
    else:
        _check(st, "hidet_attention_ranges")


def _attention_ranges(ranges, keys, documents, prefix, causal, window, stream):
    if ranges.dim() != 3:
        raise ValueError("ranges must be [batch, seq_q, 2]")
    batch, seq_q, _ = ranges.shape
    device, handle = _on((ranges, documents, prefix), stream)
    with device:
        st = lib().hidet_attention_ranges(batch, seq_q, keys, _whole32(documents, (batch, keys), "documents"),
                                          _whole32(prefix, (batch,), "prefix"), int(causal), window,
                                          _whole32(ranges, (batch, seq_q, 2), "ranges"), handle)
    _check(st, "hidet_attention_ranges")


def hidet_rope(x, y, frequencies, positions=None, first_position=0, interleaved=False, inverse=False, amplitude=1.0, stream=None):
    """y = x [batch, heads, seq, head_dim] with its first 2 * len(frequencies) elements turned (y may be x); frequencies: float64 on
    the GPU; positions: int32 [batch, seq] or [seq], or first_position, first_position + 1, ...  inverse: the backward pass."""
    st = (_attention_calls or _attn()).rope(x, y, frequencies, positions, first_position, interleaved, inverse, amplitude, stream)
    if st < 0:
        _rope(x, y, frequencies, positions, first_position, interleaved, inverse, amplitude, stream)
    else:
        _check(st, "hidet_rope")


def _rope(x, y, frequencies, positions, first_position, interleaved, inverse, amplitude, stream):
    if x.dim() != 4 or x.shape != y.shape or x.dtype != y.dtype:
        raise ValueError("x and y must be [batch, heads, seq, head_dim] and agree in shape and dtype")
    batch, heads, seq, dim = x.shape
    if frequencies.dtype != torch.float64 or frequencies.dim() != 1 or not frequencies.is_contiguous():
        raise ValueError("frequencies must be a dense float64 vector")
    pp, ps = None, 0
    if positions is not None:
        if positions.dtype != torch.int32 or tuple(positions.shape) not in ((batch, seq), (seq,)) or (
                seq > 1 and positions.stride(-1) != 1):
            raise ValueError("positions must be int32 of shape %s or %s with contiguous rows" % ((batch, seq), (seq,)))
        pp, ps = positions.data_ptr(), positions.stride(0) if positions.dim() == 2 else 0
    device, handle = _on((x, y, frequencies, positions), stream)
    with device:
        st = lib().hidet_rope(_dtype(x), batch, heads, seq, dim, 2 * frequencies.shape[0], _heads(x), _heads(y),
                              frequencies.data_ptr(), pp, ps, first_position, int(interleaved), int(inverse), amplitude, handle)
    _check(st, "hidet_rope")


def hidet_rope_frequencies(rotary_dim, base=10000.0, scaling=HIDET_ROPE_PLAIN, factor=1.0, low_turns=1.0, high_turns=4.0,
                           original_length=8192.0):
    """The frequencies of hidet_rope as a float64 CPU tensor of rotary_dim / 2 elements."""
    out = torch.empty(max(rotary_dim, 0) // 2, dtype=torch.float64)
    _check(lib().hidet_rope_frequencies(rotary_dim, base, scaling, factor, low_turns, high_turns, original_length,
                                        ctypes.cast(out.data_ptr(), ctypes.POINTER(ctypes.c_double))), "hidet_rope_frequencies")
    return out


def make_cache(k_pages, v_pages, tables, lengths):
    """hidet_cache_t over k_pages, v_pages [pages, page_size, kv_heads, head_dim] (the same strides), tables [seqs, width] int32 and
    lengths [seqs] int32, all on one device.  It holds their addresses: they are to be filled in place."""
    if k_pages.dim() != 4 or k_pages.shape != v_pages.shape or k_pages.dtype != v_pages.dtype or k_pages.stride() != v_pages.stride():
        raise ValueError("k_pages and v_pages must be [pages, page_size, kv_heads, head_dim] and agree in shape, dtype and strides")
    if k_pages.stride(3) != 1 and k_pages.shape[3] > 1:
        raise ValueError("the last dimension must be contiguous")
    if tables.dim() != 2 or tables.dtype != torch.int32 or (tables.shape[1] > 1 and tables.stride(1) != 1):
        raise ValueError("tables must be int32 [seqs, width] with contiguous rows")
    c = hidet_cache_t()
    c.struct_size = ctypes.sizeof(hidet_cache_t)
    c._keep = (k_pages, v_pages, tables, lengths)  # (the structure holds raw addresses)
    one = k_pages.is_cuda and all(t.device == k_pages.device for t in c._keep)
    c._device = k_pages.device.index if one else -1  # (of the calls that need no look at each tensor)
    c.dtype = _dtype(k_pages)
    c.k, c.v = k_pages.data_ptr(), v_pages.data_ptr()
    c.num_pages, c.page_size, c.heads, c.head_dim = k_pages.shape
    c.stride_page, c.stride_slot, c.stride_head, _ = k_pages.stride()
    c.seqs, c.table_width = tables.shape
    c.tables, c.table_stride = tables.data_ptr(), max(tables.stride(0), tables.shape[1]) if tables.shape[0] <= 1 else tables.stride(0)
    c.lengths = _whole32(lengths, (tables.shape[0],), "lengths")
    return c


def _new_tokens(cache, tensors, starts):
    for t in tensors:
        if t.dim() != 3 or t.shape != tensors[0].shape or t.shape[2] != cache.head_dim:
            raise ValueError("need tensors [tokens, heads, %d] of one shape" % cache.head_dim)
        if _dtype(t) != cache.dtype:
            raise ValueError("tensors must have the cache's dtype")
    return _whole32(starts, (cache.seqs + 1,), "starts")


def hidet_cache_append(cache, k, v, starts, max_new, stream=None):
    """Writes the new tokens' k and v [tokens, kv_heads, head_dim] into the pages of `cache` (make_cache): rows starts[s] to
    starts[s + 1] are the last positions of sequence s; starts [seqs + 1] int32; at most max_new of each sequence."""
    st = (_attention_calls or _attn()).cache_append(cache, k, v, starts, max_new, stream)
    if st < 0:
        _cache_append(cache, k, v, starts, max_new, stream)
    else:
        _check(st, "hidet_cache_append")


def _cache_append(cache, k, v, starts, max_new, stream):
    sp = _new_tokens(cache, (k, v), starts)
    if k.shape[1] != cache.heads:
        raise ValueError("the cache has %d heads" % cache.heads)
    device, handle = _on((k, v, starts) + cache._keep, stream)
    with device:
        st = lib().hidet_cache_append(cache, k.shape[0], max_new, _heads(k), _heads(v), sp, handle)
    _check(st, "hidet_cache_append")


def hidet_cache_attention(cache, q, out, starts, max_new, scale=None, window=0, softcap=0.0, slopes=None, lse=None, workspace=None,
                          stream=None):
    """Attention of the new tokens' q [tokens, heads, head_dim] over their sequences' keys in `cache` up to their own position; rows
    of `out` behind the last sequence stay as they are.  lse [tokens, heads] float32 is written where given."""
    st = (_attention_calls or _attn()).cache_attention(cache, q, out, starts, max_new, scale, window, softcap, slopes, lse, workspace, stream)
    if st < 0:
        _cache_attention(cache, q, out, starts, max_new, scale, window, softcap, slopes, lse, workspace, stream)
    else:
        _check(st, "hidet_cache_attention")


def _cache_attention(cache, q, out, starts, max_new, scale, window, softcap, slopes, lse, workspace, stream):
    sp = _new_tokens(cache, (q, out), starts)
    tokens, heads, dim = q.shape
    o = _options(scale, dim, True, window, softcap, slopes, None, heads, None)
    wp, wb = _dense_ws(workspace)
    device, handle = _on((q, out, lse, slopes, starts, workspace) + cache._keep, stream)
    with device:
        st = lib().hidet_cache_attention(cache, heads, tokens, max_new, _heads(q), _heads(out), _float32(lse, (tokens, heads), "lse"), sp,
                                         o, wp, wb, handle)
    _check(st, "hidet_cache_attention")


def hidet_cache_attention_workspace_bytes(cache, q, max_new, window=0):
    """Workspace bytes of hidet_cache_attention for queries like q (0: none is wanted)."""
    return lib().hidet_cache_attention_workspace_bytes(cache, q.shape[1], max_new, window)


def hidet_conv2d_untuned_config(dtype, x_shape, w_shape, stride=(1, 1), pad=(0, 0), packed=False):
    """The configuration of a convolution (x NCHW, w OIHW) that names none, with nothing tuned; runs nothing."""
    (Nb, IC, H, W), (OC, _, KH, KW), config = x_shape, w_shape, _i32(-1)
    _check(lib().hidet_conv2d_untuned_config(dtype, Nb, IC, H, W, OC, KH, KW, stride[0], stride[1], pad[0], pad[1], int(packed),
                                             ctypes.byref(config)), "hidet_conv2d_untuned_config")
    return config.value


def hidet_conv2d_untuned_form(dtype, x_shape, w_shape, stride=(1, 1), pad=(0, 0)):
    """The form (HIDET_CONV_) of such a convolution that names no configuration, with nothing tuned; runs nothing."""
    (Nb, IC, H, W), (OC, _, KH, KW), form = x_shape, w_shape, _i32(-1)
    _check(lib().hidet_conv2d_untuned_form(dtype, Nb, IC, H, W, OC, KH, KW, stride[0], stride[1], pad[0], pad[1], ctypes.byref(form)),
           "hidet_conv2d_untuned_form")
    return form.value


def hidet_conv2d_patch_rows(dtype, x_shape, w_shape, stride=(1, 1), pad=(0, 0)):
    """Rows of the tiles on which such a convolution runs from a patch of the input in LDS; 0: it does not."""
    (Nb, IC, H, W), (OC, _, KH, KW), rows = x_shape, w_shape, _i32(0)
    _check(lib().hidet_conv2d_patch_rows(dtype, Nb, IC, H, W, OC, KH, KW, stride[0], stride[1], pad[0], pad[1], ctypes.byref(rows)),
           "hidet_conv2d_patch_rows")
    return rows.value


def hidet_gemm_untuned_config(dtype, M, N, K, batch=1, transA=False, transB=False):
    """The configuration of a GEMM on dense operands that names none, with nothing tuned; runs nothing."""
    config = _i32(-1)
    _check(lib().hidet_gemm_untuned_config(dtype, int(transA), int(transB), batch, M, N, K, ctypes.byref(config)),
           "hidet_gemm_untuned_config")
    return config.value


def hidet_row_schedule(dtype, softmax, rows, cols):
    """How a row softmax (or reduction) of this size is cut, as a dict; runs nothing."""
    out = hidet_row_schedule_t()
    _check(lib().hidet_row_schedule(dtype, int(softmax), rows, cols, ctypes.byref(out)), "hidet_row_schedule")
    return {n: getattr(out, n) for n, _ in out._fields_}


def hidet_tune_last_times():
    n = lib().hidet_config_count()
    buf = (ctypes.c_float * n)()
    lib().hidet_tune_last_times(buf, n)
    return list(buf)


def hidet_tune_clear():
    lib().hidet_tune_clear()


def hidet_tune_save(path):
    _check(lib().hidet_tune_save(path.encode()), "hidet_tune_save")


def hidet_tune_load(path):
    _check(lib().hidet_tune_load(path.encode()), "hidet_tune_load")


def hidet_config_count():
    return lib().hidet_config_count()


def hidet_config_info(config):
    info = hidet_config_info_t()
    _check(lib().hidet_config_info(config, ctypes.byref(info)), "hidet_config_info")
    return {n: getattr(info, n) for n, _ in hidet_config_info_t._fields_}


def hidet_taskmap_count():
    return lib().hidet_taskmap_count()


def hidet_taskmap_info(index):
    buf = ctypes.create_string_buffer(256)
    w, s0, s1, t = _i32(), _i32(), _i32(), _i32()
    _check(lib().hidet_taskmap_info(index, buf, 256, ctypes.byref(w), ctypes.byref(s0), ctypes.byref(s1), ctypes.byref(t)),
           "hidet_taskmap_info")
    return dict(expr=buf.value.decode(), workers=w.value, shape=(s0.value, s1.value), tasks=t.value)


def hidet_taskmap_tasks(index, worker):
    info = hidet_taskmap_info(index)
    buf = (_i32 * (2 * info["tasks"]))()
    _check(lib().hidet_taskmap_tasks(index, worker, buf, info["tasks"]), "hidet_taskmap_tasks")
    return [(buf[2 * q], buf[2 * q + 1]) for q in range(info["tasks"])]


def hidet_block_task(tiles_m, tiles_n, group, w):
    i, j = _i32(), _i32()
    _check(lib().hidet_block_task(tiles_m, tiles_n, group, w, ctypes.byref(i), ctypes.byref(j)), "hidet_block_task")
    return i.value, j.value


def hidet_probe_launch_floor(iters=1000, stream=None):
    """Microseconds per launch of an empty kernel (back-to-back launches on one stream)."""
    us = ctypes.c_float(0.0)
    _check(lib().hidet_probe_launch_floor(_stream(stream), iters, ctypes.byref(us)), "hidet_probe_launch_floor")
    return us.value


def hidet_probe_mfma_peak(sample, mfma=16, stream=None):
    """MFMA-only ceiling on operands taken from `sample` (a GPU tensor of the input dtype); returns (TFLOP/s, sclk MHz)."""
    n = lib().hidet_probe_scratch_bytes()
    scratch = torch.empty(n, dtype=torch.uint8, device=sample.device)
    tf, mhz = ctypes.c_float(0.0), ctypes.c_float(0.0)
    flat = sample.reshape(-1)
    st = lib().hidet_probe_mfma_peak(_dtype(sample), mfma, _ptr(flat), flat.numel() * flat.element_size(), _ptr(scratch), n,
                                     _stream(stream), ctypes.byref(tf), ctypes.byref(mhz))
    _check(st, "hidet_probe_mfma_peak")
    return tf.value, mhz.value


def hidet_probe_stream_bandwidth(buffer, mode, stream=None):
    """GB/s of a plain read (mode 0), write (1) or copy (2) kernel walking over `buffer` (a GPU tensor, ideally 1 GiB)."""
    out = ctypes.c_float(0.0)
    flat = buffer.reshape(-1)
    _check(lib().hidet_probe_stream_bandwidth(_ptr(flat), flat.numel() * flat.element_size(), mode, _stream(stream),
                                              ctypes.byref(out)), "hidet_probe_stream_bandwidth")
    return out.value


def hidet_version():
    return lib().hidet_version().decode()


def hidet_kernel_launch_count():
    return int(lib().hidet_kernel_launch_count())
