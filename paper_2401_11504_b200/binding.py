"""Thin Python binding over the C ABI of libtemplora.so (include/templora.h).

Argument marshalling only: every step of the path runs in the library's CUDA
kernels.  torch provides device memory and streams.  The functions carry the
names of the C entry points.  There is no CPU fallback: importing this module
without the compiled library raises.
"""
import ctypes as C
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtemplora.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_CUDA, ERR_TIMEOUT = range(6)
F32, BF16 = 0, 1

EXPORTS = [
    "templora_workspace_bytes", "templora_update_block_workspace_bytes", "templora_linear_fwd",
    "templora_linear_bwd", "templora_adamw_step", "templora_decode_fwd", "templora_update_block",
    "templora_status_string", "templora_read_device_status", "templora_set_kernel_path",
    "templora_timing_enable", "templora_timing_read", "templora_decode_fwd_noalloc",
    "templora_decode_block_workspace_bytes", "templora_decode_block_fwd", "templora_update_block_batched",
    "templora_set_stream_sm_limit", "templora_selftest_bounded_wait", "templora_lr_at_step",
    "templora_update_block_warmup", "templora_swiglu_fwd", "templora_swiglu_bwd", "templora_rmsnorm_fwd",
    "templora_rmsnorm_bwd", "templora_decode_fwd_noalloc_status", "templora_update_mlp",
    "templora_update_mlp_workspace_bytes", "templora_sm_partition_create", "templora_sm_partition_destroy",
    "templora_update_attn_in", "templora_attention_workspace_bytes", "templora_attention_fwd", "templora_attention_bwd",
    "templora_kv_cache_append_workspace_bytes", "templora_kv_cache_append",
    "templora_attention_decode_workspace_bytes", "templora_attention_decode_fwd",
    "templora_kv_cache_weigh_workspace_bytes", "templora_kv_cache_weigh", "templora_kv_cache_evict_workspace_bytes",
    "templora_kv_cache_evict", "templora_sample",
]
NOALLOC_SCRATCH_BYTES = 8 << 20
(KIND_TC_MAIN, KIND_TC_SKINNY, KIND_TC_DECODE, KIND_REDUCE, KIND_ADAMW, KIND_SIMT, KIND_DECODE_FINISH, KIND_DROPOUT,
 KIND_TC_DROPOUT_TERM, KIND_BLOCK_OPS, KIND_ATTENTION, KIND_KV_CACHE, KIND_SAMPLE) = range(13)
N_KINDS = 13


class SmPartition(C.Structure):
    """templora_sm_partition_t: two streams whose kernels run on disjoint groups of SMs."""
    _fields_ = [("handle", C.c_void_p), ("stream_first", C.c_void_p), ("stream_rest", C.c_void_p),
                ("sms_first", C.c_int32), ("sms_rest", C.c_int32)]


class LinearDesc(C.Structure):
    _fields_ = [("d_in", C.c_int32), ("d_out", C.c_int32), ("r", C.c_int32), ("s", C.c_float),
                ("dtype", C.c_int32), ("W0", C.c_void_p), ("A", C.c_void_p), ("B", C.c_void_p),
                ("dropout_p", C.c_float), ("input_group", C.c_int32), ("dropout_seed", C.c_uint64),
                ("dropout_offset", C.c_uint64)]


class ParamDesc(C.Structure):
    _fields_ = [("n", C.c_int64), ("master", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p),
                ("work", C.c_void_p), ("grad", C.c_void_p)]


class AttentionDesc(C.Structure):
    """templora_attn_t: head layout, score modifications and masks of an attention call."""
    _fields_ = [("n_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int32),
                ("scale", C.c_float), ("softcap", C.c_float), ("causal", C.c_int32), ("window", C.c_int32),
                ("slopes", C.c_void_p), ("n_docs", C.c_int32), ("doc_offsets", C.c_void_p), ("prefix_lens", C.c_void_p)]


class AttentionIo(C.Structure):
    """templora_attn_io_t: the tensors of an attention call and their row strides in elements."""
    _fields_ = [("q", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p), ("o", C.c_void_p), ("lse", C.c_void_p),
                ("ld_q", C.c_int64), ("ld_k", C.c_int64), ("ld_v", C.c_int64), ("ld_o", C.c_int64),
                ("dO", C.c_void_p), ("dq", C.c_void_p), ("dk", C.c_void_p), ("dv", C.c_void_p),
                ("ld_dO", C.c_int64), ("ld_dq", C.c_int64), ("ld_dk", C.c_int64), ("ld_dv", C.c_int64)]


class KvCacheDesc(C.Structure):
    """templora_kv_cache_t: a paged key/value cache in e4m3 codes with one scale per block and head."""
    _fields_ = [("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("block_tokens", C.c_int32), ("n_blocks", C.c_int32),
                ("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p),
                ("n_seqs", C.c_int32), ("max_blocks", C.c_int32), ("block_table", C.c_void_p)]


class SampleDesc(C.Structure):
    """templora_sample_t: logits, per-row settings and results of a sampling call."""
    _fields_ = [("vocab", C.c_int32), ("dtype", C.c_int32), ("logits", C.c_void_p), ("ld", C.c_int64),
                ("temperature", C.c_void_p), ("top_k", C.c_void_p), ("top_p", C.c_void_p), ("min_p", C.c_void_p),
                ("u", C.c_void_p), ("tokens", C.c_void_p), ("logprobs", C.c_void_p)]


class TemploraError(RuntimeError):
    def __init__(self, code, what):
        self.code = code
        super().__init__(f"{what}: {status_string(code)} (status {code})")


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is missing: build it with `python -m paper_2401_11504_b200.build` "
                          "(there is no fallback path)")
    lib = C.CDLL(LIB_PATH)
    vp, i32, i64, f32, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_size_t
    LP, PP = C.POINTER(LinearDesc), C.POINTER(ParamDesc)
    lib.templora_workspace_bytes.restype = sz
    lib.templora_workspace_bytes.argtypes = [LP, i32]
    lib.templora_update_block_workspace_bytes.restype = sz
    lib.templora_update_block_workspace_bytes.argtypes = [LP, i32, i32]
    lib.templora_linear_fwd.restype = i32
    lib.templora_linear_fwd.argtypes = [LP, i32, vp, vp, vp, vp, sz, vp]
    lib.templora_linear_bwd.restype = i32
    lib.templora_linear_bwd.argtypes = [LP, i32, vp, vp, vp, vp, vp, vp, i32, vp, sz, vp]
    lib.templora_adamw_step.restype = i32
    lib.templora_adamw_step.argtypes = [PP, i32, f32, f32, f32, f32, f32, i64, i32, vp]
    lib.templora_decode_fwd.restype = i32
    lib.templora_decode_fwd.argtypes = [LP, i32, vp, vp, vp, sz, vp]
    lib.templora_update_block.restype = i32
    lib.templora_update_block.argtypes = [LP, PP, PP, i32, i32, C.POINTER(vp), C.POINTER(vp), C.POINTER(vp),
                                          C.POINTER(vp), i32, f32, f32, f32, f32, f32, C.POINTER(i64), vp, sz, vp]
    lib.templora_update_block_batched.restype = i32
    lib.templora_update_block_batched.argtypes = [LP, PP, PP, i32, i32, i32, C.POINTER(vp), C.POINTER(vp), C.POINTER(vp),
                                                  C.POINTER(vp), i32, f32, f32, f32, f32, f32, C.POINTER(i64), vp, sz, vp]
    lib.templora_update_block_warmup.restype = i32
    lib.templora_update_block_warmup.argtypes = [LP, PP, PP, i32, i32, i32, C.POINTER(vp), C.POINTER(vp), C.POINTER(vp),
                                                 C.POINTER(vp), i32, f32, i64, f32, f32, f32, f32, C.POINTER(i64), vp, sz, vp]
    lib.templora_update_mlp_workspace_bytes.restype = sz
    lib.templora_update_mlp_workspace_bytes.argtypes = [LP, i32]
    lib.templora_update_mlp.restype = i32
    lib.templora_update_mlp.argtypes = [LP, PP, PP, i32, vp, vp, vp, vp, vp, vp, vp, i32, f32, f32, f32, f32, f32,
                                        C.POINTER(i64), vp, sz, vp]
    lib.templora_update_attn_in.restype = i32
    lib.templora_update_attn_in.argtypes = [LP, PP, PP, i32, i32, vp, vp, f32, C.POINTER(vp), vp, C.POINTER(vp), vp, vp,
                                            i32, f32, f32, f32, f32, f32, C.POINTER(i64), vp, sz, vp]
    lib.templora_swiglu_fwd.restype = i32
    lib.templora_swiglu_fwd.argtypes = [i64, i32, vp, vp, vp, vp]
    lib.templora_swiglu_bwd.restype = i32
    lib.templora_swiglu_bwd.argtypes = [i64, i32, vp, vp, vp, vp, vp, vp]
    lib.templora_rmsnorm_fwd.restype = i32
    lib.templora_rmsnorm_fwd.argtypes = [i32, i32, i32, vp, vp, f32, vp, vp]
    lib.templora_rmsnorm_bwd.restype = i32
    lib.templora_rmsnorm_bwd.argtypes = [i32, i32, i32, vp, vp, vp, f32, vp, vp]
    lib.templora_lr_at_step.restype = f32
    lib.templora_lr_at_step.argtypes = [f32, i64, i64]
    lib.templora_selftest_bounded_wait.restype = i32
    lib.templora_selftest_bounded_wait.argtypes = [vp, sz, i32, vp]
    lib.templora_set_stream_sm_limit.restype = i32
    lib.templora_set_stream_sm_limit.argtypes = [vp, i32]
    lib.templora_sm_partition_create.restype = i32
    lib.templora_sm_partition_create.argtypes = [i32, C.POINTER(SmPartition)]
    lib.templora_sm_partition_destroy.restype = i32
    lib.templora_sm_partition_destroy.argtypes = [C.POINTER(SmPartition)]
    lib.templora_status_string.restype = C.c_char_p
    lib.templora_status_string.argtypes = [i32]
    lib.templora_read_device_status.restype = i32
    lib.templora_read_device_status.argtypes = [vp, vp, C.POINTER(i32), C.POINTER(i32)]
    lib.templora_set_kernel_path.restype = i32
    lib.templora_set_kernel_path.argtypes = [i32]
    lib.templora_decode_block_workspace_bytes.restype = sz
    lib.templora_decode_block_workspace_bytes.argtypes = [LP, i32]
    lib.templora_decode_block_fwd.restype = i32
    lib.templora_decode_block_fwd.argtypes = [LP, i32, i32, C.POINTER(vp), C.POINTER(vp), vp, sz, vp]
    lib.templora_decode_fwd_noalloc.restype = i32
    lib.templora_decode_fwd_noalloc.argtypes = [LP, i32, vp, vp, vp]
    lib.templora_decode_fwd_noalloc_status.restype = i32
    lib.templora_decode_fwd_noalloc_status.argtypes = [vp, C.POINTER(i32), C.POINTER(i32)]
    AP, IP, KP = C.POINTER(AttentionDesc), C.POINTER(AttentionIo), C.POINTER(KvCacheDesc)
    lib.templora_attention_workspace_bytes.restype = sz
    lib.templora_attention_workspace_bytes.argtypes = [AP, i32, i32]
    for fn in (lib.templora_attention_fwd, lib.templora_attention_bwd):
        fn.restype = i32
        fn.argtypes = [AP, IP, i32, i32, i32, vp, sz, vp]
    lib.templora_kv_cache_append_workspace_bytes.restype = sz
    lib.templora_kv_cache_append_workspace_bytes.argtypes = [KP]
    lib.templora_kv_cache_append.restype = i32
    lib.templora_kv_cache_append.argtypes = [KP, vp, vp, i32, i32, vp, vp, i64, i64, vp, sz, vp]
    lib.templora_attention_decode_workspace_bytes.restype = sz
    lib.templora_attention_decode_workspace_bytes.argtypes = [AP, KP]
    lib.templora_attention_decode_fwd.restype = i32
    lib.templora_attention_decode_fwd.argtypes = [AP, KP, vp, vp, i64, vp, i64, vp, vp, sz, vp]
    lib.templora_kv_cache_weigh_workspace_bytes.restype = sz
    lib.templora_kv_cache_weigh_workspace_bytes.argtypes = [AP, KP, i32]
    lib.templora_kv_cache_weigh.restype = i32
    lib.templora_kv_cache_weigh.argtypes = [AP, KP, vp, vp, i32, vp, i64, vp, i64, i64, vp, vp, sz, vp]
    lib.templora_kv_cache_evict_workspace_bytes.restype = sz
    lib.templora_kv_cache_evict_workspace_bytes.argtypes = [KP, i32]
    lib.templora_kv_cache_evict.restype = i32
    lib.templora_kv_cache_evict.argtypes = [KP, vp, vp, KP, vp, vp, i32, i32, i32, vp, vp, sz, vp]
    lib.templora_sample.restype = i32
    lib.templora_sample.argtypes = [C.POINTER(SampleDesc), i32, vp]
    lib.templora_timing_enable.restype = None
    lib.templora_timing_enable.argtypes = [i32]
    lib.templora_timing_read.restype = i32
    lib.templora_timing_read.argtypes = [i32, C.POINTER(C.c_double), C.POINTER(i64), C.POINTER(i64), i32]
    return lib


lib = _load()


def status_string(code):
    return lib.templora_status_string(int(code)).decode()


def _check(code, what):
    if code != OK:
        raise TemploraError(code, what)


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


# the current stream's handle without a Stream object around it (0.1 us instead of 3)
_current_handle = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)


def _stream(stream):
    if stream is None:
        return C.c_void_p(_current_handle(torch.cuda.current_device()))
    return C.c_void_p(stream.cuda_stream)


def dtype_code(t):
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"unsupported storage dtype {t.dtype}")


def linear_desc(W0, A, B, s, dropout_p=0.0, dropout_seed=0, dropout_offset=0, input_group=0):
    """templora_linear_t for contiguous device tensors W0 [d_out,d_in], A [r,d_in], B [d_out,r]."""
    for t in (W0, A, B):
        if not t.is_contiguous():
            raise ValueError("W0, A and B must be contiguous")
    d_out, d_in = W0.shape
    r = A.shape[0]
    if tuple(A.shape) != (r, d_in) or tuple(B.shape) != (d_out, r) or A.dtype != W0.dtype or B.dtype != W0.dtype:
        raise ValueError("shape/dtype mismatch between W0, A and B")
    desc = LinearDesc(d_in, d_out, r, float(s), dtype_code(W0), W0.data_ptr(), A.data_ptr(), B.data_ptr(),
                      float(dropout_p), int(input_group), int(dropout_seed), int(dropout_offset))
    desc._keep = (W0, A, B)  # the descriptor holds raw pointers: keep the tensors alive with it
    return desc


def param_desc(master, m, v, grad, work=None):
    desc = ParamDesc(master.numel(), master.data_ptr(), m.data_ptr(), v.data_ptr(),
                     0 if work is None else work.data_ptr(), grad.data_ptr())
    desc._keep = (master, m, v, grad, work)
    return desc


def templora_workspace_bytes(lin, T):
    return int(lib.templora_workspace_bytes(C.byref(lin), int(T)))


def templora_update_block_workspace_bytes(lins, T):
    arr = (LinearDesc * len(lins))(*lins)
    return int(lib.templora_update_block_workspace_bytes(arr, len(lins), int(T)))


def alloc_workspace(nbytes, device="cuda"):
    """Zeroed workspace (the head holds the device status record)."""
    if nbytes <= 0:
        raise ValueError("workspace size query failed (invalid projection?)")
    return torch.zeros(int(nbytes), dtype=torch.uint8, device=device)


def templora_linear_fwd(lin, x, y, ws, U_save=None, stream=None):
    _check(lib.templora_linear_fwd(C.byref(lin), x.shape[0], _ptr(x), _ptr(y), _ptr(U_save), _ptr(ws),
                                   ws.numel(), _stream(stream)), "templora_linear_fwd")


def templora_linear_bwd(lin, x, dY, dX, dA, dB, ws, U_saved=None, accumulate=False, stream=None):
    _check(lib.templora_linear_bwd(C.byref(lin), x.shape[0], _ptr(x), _ptr(dY), _ptr(U_saved), _ptr(dX), _ptr(dA),
                                   _ptr(dB), int(bool(accumulate)), _ptr(ws), ws.numel(), _stream(stream)),
           "templora_linear_bwd")


def templora_adamw_step(params, lr, beta1, beta2, eps, weight_decay, step, work_dtype=BF16, stream=None):
    arr = (ParamDesc * len(params))(*params)
    _check(lib.templora_adamw_step(arr, len(params), lr, beta1, beta2, eps, weight_decay, int(step),
                                   int(work_dtype), _stream(stream)), "templora_adamw_step")


def templora_decode_fwd(lin, x, y, ws, stream=None):
    _check(lib.templora_decode_fwd(C.byref(lin), x.shape[0], _ptr(x), _ptr(y), _ptr(ws), ws.numel(),
                                   _stream(stream)), "templora_decode_fwd")


class UpdateBlockArgs:
    """Marshalled argument arrays of templora_update_block, built once and reusable."""

    def __init__(self, lins, A_states, B_states, xs, dYs, ys, dXs=None):
        n = len(lins)
        self.n = n
        self.T = xs[0].shape[0]
        self.lins = (LinearDesc * n)(*lins)
        self.A = (ParamDesc * n)(*A_states)
        self.B = (ParamDesc * n)(*B_states)
        vp = C.c_void_p
        self.x = (vp * n)(*[t.data_ptr() for t in xs])
        self.dY = (vp * n)(*[t.data_ptr() for t in dYs])
        self.y = (vp * n)(*[t.data_ptr() for t in ys])
        self.dX = None if dXs is None else (vp * n)(*[0 if t is None else t.data_ptr() for t in dXs])
        self._keep = (lins, A_states, B_states, xs, dYs, ys, dXs)


def templora_update_block(args, epochs, lr, beta1, beta2, eps, weight_decay, step, ws, stream=None):
    """Runs the chunk update; returns the new optimizer step count."""
    st = C.c_int64(int(step))
    _check(lib.templora_update_block(args.lins, args.A, args.B, args.n, args.T, args.x, args.dY, args.y, args.dX,
                                     int(epochs), lr, beta1, beta2, eps, weight_decay, C.byref(st), _ptr(ws),
                                     ws.numel(), _stream(stream)), "templora_update_block")
    return st.value


def templora_update_block_batched(args, batch_tokens, epochs, lr, beta1, beta2, eps, weight_decay, step, ws,
                                  stream=None):
    """Chunk update with one optimizer step per batch of batch_tokens rows; returns the new step count."""
    st = C.c_int64(int(step))
    _check(lib.templora_update_block_batched(args.lins, args.A, args.B, args.n, args.T, int(batch_tokens), args.x,
                                             args.dY, args.y, args.dX, int(epochs), lr, beta1, beta2, eps,
                                             weight_decay, C.byref(st), _ptr(ws), ws.numel(), _stream(stream)),
           "templora_update_block_batched")
    return st.value


def templora_update_block_warmup(args, batch_tokens, epochs, lr, warmup_steps, beta1, beta2, eps, weight_decay, step, ws,
                                 stream=None):
    """Batched chunk update with the linear learning-rate warm-up applied per optimizer step."""
    st = C.c_int64(int(step))
    _check(lib.templora_update_block_warmup(args.lins, args.A, args.B, args.n, args.T, int(batch_tokens), args.x,
                                            args.dY, args.y, args.dX, int(epochs), lr, int(warmup_steps), beta1, beta2,
                                            eps, weight_decay, C.byref(st), _ptr(ws), ws.numel(), _stream(stream)),
           "templora_update_block_warmup")
    return st.value


def templora_update_mlp_workspace_bytes(lins, T):
    arr = (LinearDesc * 3)(*lins)
    return int(lib.templora_update_mlp_workspace_bytes(arr, int(T)))


def templora_update_mlp(lins, A_states, B_states, x, dY, gate, up, h, y, dX, epochs, lr, beta1, beta2, eps, weight_decay,
                        step, ws, stream=None):
    """Chunk update of a block's MLP (lins, A_states, B_states: gate, up, down); returns the new step count."""
    st = C.c_int64(int(step))
    _check(lib.templora_update_mlp((LinearDesc * 3)(*lins), (ParamDesc * 3)(*A_states), (ParamDesc * 3)(*B_states),
                                   x.shape[0], _ptr(x), _ptr(dY), _ptr(gate), _ptr(up), _ptr(h), _ptr(y), _ptr(dX),
                                   int(epochs), lr, beta1, beta2, eps, weight_decay, C.byref(st), _ptr(ws), ws.numel(),
                                   _stream(stream)), "templora_update_mlp")
    return st.value


def templora_update_attn_in(lins, A_states, B_states, x, norm_weight, norm_eps, dYs, xn, ys, dXn, dX, epochs, lr, beta1,
                            beta2, eps, weight_decay, step, ws, stream=None):
    """Chunk update of the projections behind a block's input norm (q, k, v): RMSNorm, the projections on the shared
    normalised input with one summed input gradient, the norm's backward; returns the new step count."""
    n = len(lins)
    st = C.c_int64(int(step))
    vp = C.c_void_p
    dy_arr = (vp * n)(*[t.data_ptr() for t in dYs])
    y_arr = (vp * n)(*[t.data_ptr() for t in ys])
    _check(lib.templora_update_attn_in((LinearDesc * n)(*lins), (ParamDesc * n)(*A_states), (ParamDesc * n)(*B_states), n,
                                       x.shape[0], _ptr(x), _ptr(norm_weight), norm_eps, dy_arr, _ptr(xn), y_arr, _ptr(dXn),
                                       _ptr(dX), int(epochs), lr, beta1, beta2, eps, weight_decay, C.byref(st), _ptr(ws),
                                       ws.numel(), _stream(stream)), "templora_update_attn_in")
    return st.value


def templora_swiglu_fwd(gate, up, h, stream=None):
    """h = SiLU(gate) * up, element-wise over contiguous tensors of one shape and dtype."""
    _check(lib.templora_swiglu_fwd(gate.numel(), dtype_code(gate), _ptr(gate), _ptr(up), _ptr(h), _stream(stream)),
           "templora_swiglu_fwd")


def templora_swiglu_bwd(gate, up, dh, dgate, dup, stream=None):
    _check(lib.templora_swiglu_bwd(gate.numel(), dtype_code(gate), _ptr(gate), _ptr(up), _ptr(dh), _ptr(dgate), _ptr(dup),
                                   _stream(stream)), "templora_swiglu_bwd")


def templora_rmsnorm_fwd(x, w, eps, y, stream=None):
    """y = x / sqrt(mean(x^2) + eps) * w over the rows of a contiguous [T, d] tensor."""
    _check(lib.templora_rmsnorm_fwd(x.shape[0], x.shape[1], dtype_code(x), _ptr(x), _ptr(w), eps, _ptr(y),
                                    _stream(stream)), "templora_rmsnorm_fwd")


def templora_rmsnorm_bwd(x, w, dy, eps, dx, stream=None):
    _check(lib.templora_rmsnorm_bwd(x.shape[0], x.shape[1], dtype_code(x), _ptr(x), _ptr(w), _ptr(dy), eps, _ptr(dx),
                                    _stream(stream)), "templora_rmsnorm_bwd")


def _device_ints(name, t, n=None):
    if t.dtype != torch.int32 or not t.is_contiguous() or (n is not None and t.numel() != n):
        raise ValueError(f"{name} must be a contiguous int32 tensor" + ("" if n is None else f" of {n} elements"))
    return t.data_ptr()


def _rows(name, t, rows, heads, dim, dtype):
    """Row stride of a [rows, heads, dim] tensor whose heads are contiguous one after the other."""
    if tuple(t.shape) != (rows, heads, dim) or dtype_code(t) != dtype:
        raise ValueError(f"{name} must be [{rows}, {heads}, {dim}] of the descriptor's dtype")
    if (dim > 1 and t.stride(2) != 1) or (heads > 1 and t.stride(1) != dim):
        raise ValueError(f"{name}: the heads of a row must be contiguous")
    if rows > 1 and t.stride(0) < heads * dim:     # 0 (a broadcast row) would mean contiguous to the library
        raise ValueError(f"{name}: rows must not share memory")
    return t.stride(0) if rows > 1 else heads * dim


def _same_device(tensors):
    devices = {t.device for t in tensors if t is not None}
    if len(devices) != 1 or next(iter(devices)).type != "cuda":
        raise ValueError("the tensors of a call must be on one CUDA device")
    return next(iter(devices))


def _call_on(device, stream, ws, call, what):
    """Runs call(workspace, its bytes, stream) with `device` current; stream None: that device's current stream."""
    if ws.device != device:
        raise ValueError("the workspace is on another device than the tensors")
    if not ws.is_contiguous():
        raise ValueError("the workspace must be contiguous")
    if device.index == torch.cuda.current_device():
        _check(call(_ptr(ws), ws.numel(), _stream(stream)), what)
    else:
        with torch.cuda.device(device):
            _check(call(_ptr(ws), ws.numel(), _stream(stream)), what)


def _enqueue(fn, args, ws, stream, what):
    """fn(*args.call, workspace, its bytes, stream), as _call_on; ws False: a call that takes none."""
    if ws is not False and ws.device != args.device:
        raise ValueError("the workspace is on another device than the tensors")
    if ws is not False and not ws.is_contiguous():
        raise ValueError("the workspace must be contiguous")
    rest = () if ws is False else (C.c_void_p(ws.data_ptr()), ws.numel())
    if args.device.index == torch.cuda.current_device():
        _check(fn(*args.call, *rest, _stream(stream)), what)
    else:
        with torch.cuda.device(args.device):
            _check(fn(*args.call, *rest, _stream(stream)), what)


def attention_desc(n_heads, n_kv_heads, head_dim, dtype, scale=None, softcap=0.0, causal=True, window=0, slopes=None,
                   doc_offsets=None, prefix_lens=None):
    """templora_attn_t.  scale None: 1 / sqrt(head_dim).  slopes: fp32 [n_heads]; doc_offsets: int32 [n_docs + 1];
    prefix_lens: int32 [n_docs], or [1] without documents."""
    n_docs = 0
    if doc_offsets is not None:
        n_docs = doc_offsets.numel() - 1
        if n_docs < 1:
            raise ValueError("doc_offsets needs two entries at least")
    if slopes is not None and (slopes.dtype != torch.float32 or slopes.numel() != n_heads or not slopes.is_contiguous()):
        raise ValueError("slopes must be a contiguous fp32 tensor of n_heads elements")
    desc = AttentionDesc(int(n_heads), int(n_kv_heads), int(head_dim), int(dtype),
                         float(head_dim ** -0.5 if scale is None else scale), float(softcap), int(bool(causal)), int(window),
                         None if slopes is None else slopes.data_ptr(), n_docs,
                         None if doc_offsets is None else _device_ints("doc_offsets", doc_offsets),
                         None if prefix_lens is None else _device_ints("prefix_lens", prefix_lens, max(1, n_docs)))
    desc._keep = (slopes, doc_offsets, prefix_lens)
    return desc


def templora_attention_workspace_bytes(attn, Tq, Tk):
    return int(lib.templora_attention_workspace_bytes(C.byref(attn), int(Tq), int(Tk)))


class AttentionArgs:
    """Marshalled arguments of templora_attention_fwd and, with do, dq, dk, dv, of templora_attention_bwd, built once
    and reusable.  q, o [Tq, n_heads, head_dim]; k, v [Tk, n_kv_heads, head_dim]; lse fp32 [n_heads, Tq]; rows may be
    strided (slices of a wider buffer)."""

    def __init__(self, attn, q, k, v, o, lse, q_start=0, do=None, dq=None, dk=None, dv=None):
        self.attn, self.Tq, self.Tk, self.q_start = attn, q.shape[0], k.shape[0], int(q_start)
        h, g, d, dt = attn.n_heads, attn.n_kv_heads, attn.head_dim, attn.dtype
        io = AttentionIo()
        for name, t, rows, heads in (("q", q, self.Tq, h), ("k", k, self.Tk, g), ("v", v, self.Tk, g), ("o", o, self.Tq, h),
                                     ("dO", do, self.Tq, h), ("dq", dq, self.Tq, h), ("dk", dk, self.Tk, g),
                                     ("dv", dv, self.Tk, g)):
            if t is not None:
                setattr(io, "ld_" + name, _rows(name, t, rows, heads, d, dt))
                setattr(io, name, t.data_ptr())
        if lse.dtype != torch.float32 or tuple(lse.shape) != (h, self.Tq) or not lse.is_contiguous():
            raise ValueError("lse must be a contiguous fp32 tensor [n_heads, Tq]")
        io.lse = lse.data_ptr()
        self.io = io
        self.device = _same_device((q, k, v, o, lse, do, dq, dk, dv) + attn._keep)
        self._keep = (attn, q, k, v, o, lse, do, dq, dk, dv)


def templora_attention_fwd(args, ws, stream=None):
    """o and lse of one chunk's attention."""
    _call_on(args.device, stream, ws, lambda w, n, st: lib.templora_attention_fwd(
        C.byref(args.attn), C.byref(args.io), args.Tq, args.Tk, args.q_start, w, n, st), "templora_attention_fwd")


def templora_attention_bwd(args, ws, stream=None):
    """dq, dk, dv from dO and the forward's o and lse."""
    _call_on(args.device, stream, ws, lambda w, n, st: lib.templora_attention_bwd(
        C.byref(args.attn), C.byref(args.io), args.Tq, args.Tk, args.q_start, w, n, st), "templora_attention_bwd")


def kv_cache_desc(k, v, k_scale, v_scale, block_table):
    """templora_kv_cache_t for codes k, v [n_blocks, n_kv_heads, block_tokens, head_dim] (uint8 or float8_e4m3fn), fp32
    scales [n_blocks, n_kv_heads] and an int32 block table [n_seqs, max_blocks], all contiguous."""
    n_blocks, heads, block_tokens, dim = k.shape
    for t in (k, v):
        if tuple(t.shape) != tuple(k.shape) or t.dtype not in (torch.uint8, torch.float8_e4m3fn) or not t.is_contiguous():
            raise ValueError("k and v must be contiguous uint8 or float8_e4m3fn tensors of one shape")
    for t in (k_scale, v_scale):
        if tuple(t.shape) != (n_blocks, heads) or t.dtype != torch.float32 or not t.is_contiguous():
            raise ValueError("the scales must be contiguous fp32 tensors [n_blocks, n_kv_heads]")
    if block_table.dim() != 2:
        raise ValueError("block_table must be [n_seqs, max_blocks]")
    desc = KvCacheDesc(heads, dim, block_tokens, n_blocks, k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(),
                       block_table.shape[0], block_table.shape[1], _device_ints("block_table", block_table))
    desc._device = _same_device((k, v, k_scale, v_scale, block_table))
    desc._keep = (k, v, k_scale, v_scale, block_table)
    return desc


def templora_kv_cache_append_workspace_bytes(cache):
    return int(lib.templora_kv_cache_append_workspace_bytes(C.byref(cache)))


class KvCacheAppendArgs:
    """Marshalled arguments of templora_kv_cache_append: k_new, v_new [n_new, n_kv_heads, head_dim], the tokens every
    sequence holds before the call, and where its new rows begin (None: one new token per sequence)."""

    def __init__(self, cache, seq_lens, k_new, v_new, new_offsets=None):
        self.cache, self.n_new, self.dtype = cache, k_new.shape[0], dtype_code(k_new)
        self.ld = [_rows(n, t, self.n_new, cache.n_kv_heads, cache.head_dim, self.dtype)
                   for n, t in (("k_new", k_new), ("v_new", v_new))]
        self.lens = C.c_void_p(_device_ints("seq_lens", seq_lens, cache.n_seqs))
        self.offsets = None if new_offsets is None else C.c_void_p(_device_ints("new_offsets", new_offsets, cache.n_seqs + 1))
        self.k, self.v = _ptr(k_new), _ptr(v_new)
        self.device = _same_device((k_new, v_new, seq_lens, new_offsets, cache._keep[0]))
        self._keep = (cache, seq_lens, k_new, v_new, new_offsets)


def templora_kv_cache_append(args, ws, stream=None):
    """Encodes new keys and values into the cache (seq_lens is not advanced)."""
    _call_on(args.device, stream, ws, lambda w, n, st: lib.templora_kv_cache_append(
        C.byref(args.cache), args.lens, args.offsets, args.n_new, args.dtype, args.k, args.v, args.ld[0], args.ld[1], w, n, st),
        "templora_kv_cache_append")


def templora_attention_decode_workspace_bytes(attn, cache):
    return int(lib.templora_attention_decode_workspace_bytes(C.byref(attn), C.byref(cache)))


class AttentionDecodeArgs:
    """Marshalled arguments of templora_attention_decode_fwd: q, o [n_seqs, n_heads, head_dim], seq_lens the tokens of
    every sequence (the query's own included), lse fp32 [n_seqs, n_heads] or None."""

    def __init__(self, attn, cache, seq_lens, q, o, lse=None):
        self.attn, self.cache = attn, cache
        self.ld = [_rows(n, t, cache.n_seqs, attn.n_heads, attn.head_dim, attn.dtype) for n, t in (("q", q), ("o", o))]
        if lse is not None and (lse.dtype != torch.float32 or tuple(lse.shape) != (cache.n_seqs, attn.n_heads)
                                or not lse.is_contiguous()):
            raise ValueError("lse must be a contiguous fp32 tensor [n_seqs, n_heads]")
        self.lens = C.c_void_p(_device_ints("seq_lens", seq_lens, cache.n_seqs))
        self.q, self.o, self.lse = _ptr(q), _ptr(o), _ptr(lse)
        self.device = _same_device((q, o, lse, seq_lens, cache._keep[0]) + attn._keep)
        self._keep = (attn, cache, seq_lens, q, o, lse)


def templora_attention_decode_fwd(args, ws, stream=None):
    """Attention of one new token per sequence over the cache."""
    _call_on(args.device, stream, ws, lambda w, n, st: lib.templora_attention_decode_fwd(
        C.byref(args.attn), C.byref(args.cache), args.lens, args.q, args.ld[0], args.o, args.ld[1], args.lse, w, n, st),
        "templora_attention_decode_fwd")


def _cache_weights(name, t, cache):
    if t.dtype != torch.float32 or tuple(t.shape) != (cache.n_blocks, cache.n_kv_heads, cache.block_tokens) or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous fp32 tensor [n_blocks, n_kv_heads, block_tokens]")
    return C.c_void_p(t.data_ptr())


def templora_kv_cache_weigh_workspace_bytes(attn, cache, n_rows):
    return int(lib.templora_kv_cache_weigh_workspace_bytes(C.byref(attn), C.byref(cache), int(n_rows)))


class KvCacheWeighArgs:
    """Marshalled arguments of templora_kv_cache_weigh: q [n_rows, n_heads, head_dim], lse fp32 [n_rows, n_heads] in any layout
    (of a chunk, pass the transpose of templora_attention_fwd's), weights fp32 [n_blocks, n_kv_heads, block_tokens], and where
    every sequence's rows begin (None: one row per sequence)."""

    def __init__(self, attn, cache, seq_lens, q, lse, weights, row_offsets=None):
        n_rows = q.shape[0]
        ld_q = _rows("q", q, n_rows, attn.n_heads, attn.head_dim, attn.dtype)
        if lse.dtype != torch.float32 or tuple(lse.shape) != (n_rows, attn.n_heads):
            raise ValueError("lse must be an fp32 tensor [n_rows, n_heads]")
        lens = C.c_void_p(_device_ints("seq_lens", seq_lens, cache.n_seqs))
        offsets = None if row_offsets is None else C.c_void_p(_device_ints("row_offsets", row_offsets, cache.n_seqs + 1))
        self.call = (C.byref(attn), C.byref(cache), lens, offsets, n_rows, _ptr(q), ld_q, _ptr(lse), *lse.stride(),
                     _cache_weights("weights", weights, cache))
        self.device = _same_device((q, lse, weights, seq_lens, row_offsets, cache._keep[0]) + attn._keep)
        self._keep = (attn, cache, seq_lens, q, lse, weights, row_offsets)


def templora_kv_cache_weigh(args, ws, stream=None):
    """Adds what attention the new rows pay every cached token to the cache's weights."""
    _enqueue(lib.templora_kv_cache_weigh, args, ws, stream, "templora_kv_cache_weigh")


def templora_kv_cache_evict_workspace_bytes(cache, n_keep):
    return int(lib.templora_kv_cache_evict_workspace_bytes(C.byref(cache), int(n_keep)))


class KvCacheEvictArgs:
    """Marshalled arguments of templora_kv_cache_evict: the cache with its weights and lengths, the blocks its kept tokens go
    to (`to`: a descriptor of the same pool under another table, or of another pool) with their weights, the new lengths, and,
    if wanted, where the kept tokens stood (int32 [n_seqs, n_kv_heads, n_keep])."""

    def __init__(self, cache, weights, seq_lens, to, to_weights, new_lens, n_keep, n_first=0, n_recent=0, kept=None):
        w, to_w = _cache_weights("weights", weights, cache), _cache_weights("to_weights", to_weights, to)
        lens, new = (C.c_void_p(_device_ints(n, t, cache.n_seqs)) for n, t in (("seq_lens", seq_lens), ("new_lens", new_lens)))
        if kept is not None and tuple(kept.shape) != (cache.n_seqs, cache.n_kv_heads, int(n_keep)):
            raise ValueError("kept must be [n_seqs, n_kv_heads, n_keep]")
        self.call = (C.byref(cache), w, lens, C.byref(to), to_w, new, int(n_keep), int(n_first), int(n_recent),
                     None if kept is None else C.c_void_p(_device_ints("kept", kept)))
        self.device = _same_device((weights, to_weights, seq_lens, new_lens, kept, cache._keep[0], to._keep[0]))
        self._keep = (cache, weights, seq_lens, to, to_weights, new_lens, kept)


def templora_kv_cache_evict(args, ws, stream=None):
    """Moves the tokens that each sequence keeps into the blocks of args.to."""
    _enqueue(lib.templora_kv_cache_evict, args, ws, stream, "templora_kv_cache_evict")


class SampleArgs:
    """Marshalled arguments of templora_sample: logits [rows, vocab] (fp32 or bf16, rows may be strided), u fp32 [rows], tokens
    int32 [rows], and per row, or None: temperature, top_p, min_p (fp32), top_k (int32), logprobs (fp32)."""

    def __init__(self, logits, u, tokens, temperature=None, top_k=None, top_p=None, min_p=None, logprobs=None):
        if logits.dim() != 2 or (logits.shape[1] > 1 and logits.stride(1) != 1):
            raise ValueError("logits must be [rows, vocab] with contiguous rows")
        rows, vocab = logits.shape
        if rows > 1 and logits.stride(0) < vocab:      # 0 (a broadcast row) would mean contiguous to the library
            raise ValueError("logits: rows must not share memory")
        for name, t, dt in (("u", u, torch.float32), ("tokens", tokens, torch.int32), ("temperature", temperature, torch.float32),
                            ("top_k", top_k, torch.int32), ("top_p", top_p, torch.float32), ("min_p", min_p, torch.float32),
                            ("logprobs", logprobs, torch.float32)):
            if t is not None and (t.dtype != dt or tuple(t.shape) != (rows,) or not t.is_contiguous()):
                raise ValueError(f"{name} must be a contiguous {dt} tensor of one entry per row")
        at = lambda t: None if t is None else t.data_ptr()  # noqa: E731
        desc = SampleDesc(vocab, dtype_code(logits), at(logits), logits.stride(0) if rows > 1 else vocab, at(temperature),
                          at(top_k), at(top_p), at(min_p), at(u), at(tokens), at(logprobs))
        self.call = (C.byref(desc), rows)
        self.device = _same_device((logits, u, tokens, temperature, top_k, top_p, min_p, logprobs))
        self._keep = (desc, logits, u, tokens, temperature, top_k, top_p, min_p, logprobs)


def templora_sample(args, stream=None):
    """Draws the next token of every row."""
    _enqueue(lib.templora_sample, args, False, stream, "templora_sample")


def templora_lr_at_step(lr, step, warmup_steps):
    return float(lib.templora_lr_at_step(lr, int(step), int(warmup_steps)))


def templora_read_device_status(ws, stream=None):
    code, where = C.c_int32(0), C.c_int32(0)
    _check(lib.templora_read_device_status(_ptr(ws), _stream(stream), C.byref(code), C.byref(where)),
           "templora_read_device_status")
    return code.value, where.value


def templora_set_kernel_path(mode):
    return int(lib.templora_set_kernel_path(int(mode)))


def templora_timing_enable(kinds):
    """kinds: iterable of kernel classes to time, True for all, False/None for none."""
    if kinds is True:
        mask = -1
    elif not kinds:
        mask = 0
    else:
        mask = 0
        for k in kinds:
            mask |= 1 << int(k)
    lib.templora_timing_enable(mask)


def templora_timing_read(kind, reset=False):
    """-> (total_ms, timed_launches, all_launches) of one kernel class."""
    ms, timed, allc = C.c_double(0.0), C.c_int64(0), C.c_int64(0)
    _check(lib.templora_timing_read(int(kind), C.byref(ms), C.byref(timed), C.byref(allc), int(bool(reset))),
           "templora_timing_read")
    return ms.value, timed.value, allc.value


def templora_decode_fwd_noalloc(lin, x, y, stream=None):
    """Decode-time forward without a caller workspace: for hosts that may not allocate device
    memory.  Scratch is a fixed array inside the library (NOALLOC_SCRATCH_BYTES per GPU), shared by
    all calls on the device, so calls that could overlap on the GPU must be serialised."""
    _check(lib.templora_decode_fwd_noalloc(C.byref(lin), x.shape[0], _ptr(x), _ptr(y), _stream(stream)),
           "templora_decode_fwd_noalloc")


def templora_decode_fwd_noalloc_status(stream=None):
    """(code, where) of the most recent templora_decode_fwd_noalloc call on this device; synchronises the stream."""
    code, where = C.c_int32(0), C.c_int32(0)
    _check(lib.templora_decode_fwd_noalloc_status(_stream(stream), C.byref(code), C.byref(where)),
           "templora_decode_fwd_noalloc_status")
    return code.value, where.value


def templora_decode_block_workspace_bytes(lins):
    arr = (LinearDesc * len(lins))(*lins)
    return int(lib.templora_decode_block_workspace_bytes(arr, len(lins)))


class DecodeBlockArgs:
    """Marshalled argument arrays of templora_decode_block_fwd, built once and reusable."""

    def __init__(self, lins, xs, ys):
        n = len(lins)
        self.n, self.n_tokens = n, xs[0].shape[0]
        self.lins = (LinearDesc * n)(*lins)
        self.x = (C.c_void_p * n)(*[t.data_ptr() for t in xs])
        self.y = (C.c_void_p * n)(*[t.data_ptr() for t in ys])
        self._keep = (lins, xs, ys)


def templora_decode_block_fwd(args, ws, stream=None):
    _check(lib.templora_decode_block_fwd(args.lins, args.n, args.n_tokens, args.x, args.y, _ptr(ws), ws.numel(),
                                         _stream(stream)), "templora_decode_block_fwd")


def templora_set_stream_sm_limit(stream, max_sms):
    """Cap the SMs the persistent kernels use on `stream` (0 = no cap)."""
    _check(lib.templora_set_stream_sm_limit(_stream(stream), int(max_sms)), "templora_set_stream_sm_limit")


def templora_sm_partition_create(first_sms):
    """Split the current device's SMs into two groups with one stream each; returns the filled SmPartition
    (wrap its streams with torch.cuda.ExternalStream to use them from torch)."""
    part = SmPartition()
    _check(lib.templora_sm_partition_create(int(first_sms), C.byref(part)), "templora_sm_partition_create")
    return part


def templora_sm_partition_destroy(part):
    _check(lib.templora_sm_partition_destroy(C.byref(part)), "templora_sm_partition_destroy")


def templora_selftest_bounded_wait(ws, limit_ms=50, stream=None):
    """Enqueue the wait that must run out; read the outcome with templora_read_device_status."""
    _check(lib.templora_selftest_bounded_wait(_ptr(ws), ws.numel(), int(limit_ms), _stream(stream)),
           "templora_selftest_bounded_wait")
