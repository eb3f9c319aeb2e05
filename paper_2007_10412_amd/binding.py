"""ctypes binding of librad_hip.so: same names as include/rad.h, argument
marshalling only.  Tensors are torch CUDA(HIP) tensors; every computation runs
in the library's kernels.  There is no fallback: a missing library raises."""
import ctypes as C
import operator
import os

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "librad_hip.so")

RAD_OK, RAD_ERR_NULL, RAD_ERR_SHAPE, RAD_ERR_PARAM, RAD_ERR_UNSUPPORTED, RAD_ERR_CAPACITY, RAD_ERR_DEVICE = range(7)
RAD_F32, RAD_BF16 = 0, 1
(RAD_EXACT, RAD_BERNOULLI, RAD_FIXEDK_SHARED, RAD_FIXEDK_PER_EXAMPLE, RAD_REPLACE_SHARED, RAD_REPLACE_PER_EXAMPLE,
 RAD_PROJECT_SHARED, RAD_PROJECT_PER_EXAMPLE) = range(8)
RAD_LINEAR, RAD_CONV2D = 0, 1
STATUS_NAMES = ["RAD_OK", "RAD_ERR_NULL", "RAD_ERR_SHAPE", "RAD_ERR_PARAM", "RAD_ERR_UNSUPPORTED",
                "RAD_ERR_CAPACITY", "RAD_ERR_DEVICE"]


class rad_layer(C.Structure):
    _fields_ = [("kind", C.c_int32), ("dtype", C.c_int32), ("batch", C.c_int64), ("d_in", C.c_int64),
                ("d_out", C.c_int64), ("relu", C.c_int32), ("has_bias", C.c_int32),
                ("c_in", C.c_int32), ("h", C.c_int32), ("w", C.c_int32), ("c_out", C.c_int32),
                ("kh", C.c_int32), ("kw", C.c_int32), ("pad", C.c_int32)]


class rad_sampling(C.Structure):
    _fields_ = [("scheme", C.c_int32), ("p", C.c_double), ("seed", C.c_uint64),
                ("stream_id", C.c_uint32), ("step", C.c_uint32)]


class rad_store_stats(C.Structure):
    _fields_ = [("value_bytes", C.c_uint64), ("index_bytes", C.c_uint64), ("bit_bytes", C.c_uint64),
                ("nnz", C.c_uint64), ("dense_bytes", C.c_uint64)]


# every symbol include/rad.h declares: name -> (restype, argtypes)
P = C.c_void_p
RAD_SGD, RAD_ADAM = 0, 1


class rad_optimizer(C.Structure):
    _fields_ = [("kind", C.c_int32), ("lr", C.c_double), ("l2", C.c_double), ("beta1", C.c_double),
                ("beta2", C.c_double), ("eps", C.c_double)]


class rad_pde_grid(C.Structure):
    _fields_ = [("n", C.c_int32), ("steps", C.c_int64), ("D", C.c_double), ("dt", C.c_double)]


class rad_graph(C.Structure):
    _fields_ = [("n_vertices", C.c_int32), ("n_levels", C.c_int32), ("n_edges", C.c_int64), ("level_ptr", P),
                ("succ_ptr", P), ("succ", P), ("partial", P)]


class rad_teacher(C.Structure):
    _fields_ = [("k", C.c_int32), ("temperature", C.c_double), ("index", P), ("logit", P)]


class rad_logprobs(C.Structure):
    _fields_ = [("temperature", C.c_double), ("token", P), ("logprob", P), ("entropy", P), ("top_k", C.c_int32),
                ("top_index", P), ("top_logprob", P)]


_HEAD = [P, P, P, P, P, C.c_int32, P, C.c_float]     # row_weight, row_loss, loss, dX, dW, dw_dtype, dbias, beta
SIGNATURES = {
    "rad_fixed_k": (C.c_int64, [C.c_double, C.c_int64]),
    "rad_ctx_create": (C.c_int, [C.POINTER(P), P]),
    "rad_ctx_destroy": (C.c_int, [P]),
    "rad_last_error": (C.c_char_p, [P]),
    "rad_ctx_synchronize": (C.c_int, [P]),
    "rad_ctx_timing": (C.c_int, [P, C.c_char_p]),
    "rad_ctx_timing_read": (C.c_int, [P, C.c_char_p, C.POINTER(C.c_int64), C.POINTER(C.c_double)]),
    "rad_ctx_timing_read_flops": (C.c_int, [P, C.c_char_p, C.POINTER(C.c_double), C.POINTER(C.c_double)]),
    "rad_ctx_timing_reset": (C.c_int, [P]),
    "rad_debug_key_shift": (C.c_int, [P, C.c_int32]),
    "rad_debug_poll_limit": (C.c_int, [P, C.c_int32]),
    "rad_debug_absent_groups": (C.c_int, [P, C.c_uint32, C.c_int32]),
    "rad_debug_redone_launches": (C.c_int, [P, C.POINTER(C.c_int32), C.POINTER(C.c_int32)]),
    "rad_probe_ceiling": (C.c_int, [P, C.c_int32, P, P, C.c_uint64, C.c_int32, C.POINTER(C.c_double)]),
    "rad_store_create": (C.c_int, [P, C.POINTER(rad_layer), C.c_int32, C.c_double, C.c_int32, C.POINTER(P)]),
    "rad_store_destroy": (C.c_int, [P]),
    "rad_store_get_stats": (C.c_int, [P, P, C.POINTER(rad_store_stats)]),
    "rad_store_export_csr": (C.c_int, [P, P, P, P, P, C.c_int64]),
    "rad_store_export_bits": (C.c_int, [P, P, P]),
    "rad_store_import_bits": (C.c_int, [P, P, P]),
    "rad_sample_pack": (C.c_int, [P, C.POINTER(rad_sampling), P, P, C.c_int32]),
    "rad_sample_pack_static": (C.c_int, [P, C.POINTER(rad_sampling), P, P]),
    "rad_forward_sample": (C.c_int, [P, C.POINTER(rad_layer), C.POINTER(rad_sampling), P, P, P, P, P]),
    "rad_backward_dW": (C.c_int, [P, C.POINTER(rad_layer), P, P, P, P, C.c_float]),
    "rad_backward_dX": (C.c_int, [P, C.POINTER(rad_layer), P, P, P, P]),
    "rad_softmax_ce": (C.c_int, [P, P, P, C.c_int64, C.c_int64, C.c_int32, P, P]),
    "rad_distill_ce": (C.c_int, [P, P, C.POINTER(rad_teacher), P, C.c_int64, C.c_int64, C.c_int32, P, P, P]),
    "rad_linear_ce": (C.c_int, [P, C.POINTER(rad_layer), P, P, P, P] + _HEAD),
    "rad_linear_distill": (C.c_int, [P, C.POINTER(rad_layer), P, P, P, C.POINTER(rad_teacher)] + _HEAD),
    "rad_token_logprobs": (C.c_int, [P, P, C.c_int64, C.c_int64, C.c_int32, C.POINTER(rad_logprobs)]),
    "rad_token_logprobs_grad": (C.c_int, [P, P, C.c_int64, C.c_int64, C.c_int32, P, C.c_double, P, P, P]),
    "rad_linear_logprobs": (C.c_int, [P, C.POINTER(rad_layer), P, P, P, C.POINTER(rad_logprobs)]),
    "rad_linear_logprobs_grad": (C.c_int, [P, C.POINTER(rad_layer), P, P, P, P, C.c_double, P, P, P, P, C.c_int32, P, C.c_float]),
    "rad_model_create_mlp": (C.c_int, [P, C.c_int32, C.c_int64, C.c_int32, C.POINTER(C.c_int64), C.c_int32,
                                       C.c_int32, C.c_double, C.POINTER(P)]),
    "rad_model_create_rnn": (C.c_int, [P, C.c_int64, C.c_int64, C.c_int64, C.c_int64, C.c_int64, C.c_int32,
                                       C.c_double, C.POINTER(P)]),
    "rad_model_create_cnn": (C.c_int, [P, C.c_int64, C.c_int32, C.POINTER(C.c_int32), C.POINTER(C.c_int32),
                                       C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_double,
                                       C.POINTER(P)]),
    "rad_model_destroy": (C.c_int, [P]),
    "rad_model_num_stores": (C.c_int32, [P]),
    "rad_model_store": (P, [P, C.c_int32]),
    "rad_store_set_index_free": (C.c_int, [P, P, C.c_int32]),
    "rad_model_set_index_free": (C.c_int, [P, P, C.c_int32]),
    "rad_model_logits": (P, [P]),
    "rad_model_export_pool_arg": (C.c_int, [P, P, C.c_int32, P]),
    "rad_train_step": (C.c_int, [P, P, C.POINTER(rad_sampling), P, P, C.POINTER(P), C.POINTER(P),
                                 C.POINTER(C.c_float)]),
    "rad_pde_workspace_bytes": (C.c_int, [P, C.POINTER(rad_pde_grid), C.c_double, C.c_int32, C.POINTER(C.c_uint64)]),
    "rad_pde_gradient": (C.c_int, [P, C.POINTER(rad_pde_grid), C.c_int32, P, C.c_double, C.c_uint64, C.c_uint32, P,
                                   C.c_uint64, P, P, P]),
    "rad_path_sample_gradient": (C.c_int, [P, C.POINTER(rad_graph), C.c_int32, P, C.c_int32, C.c_int32, C.c_uint64,
                                           C.c_uint32, P, P]),
    "rad_optimizer_step": (C.c_int, [P, C.POINTER(rad_optimizer), C.c_int64, C.c_int32, C.c_int32,
                                     C.POINTER(C.c_int64), C.POINTER(P), C.POINTER(P), C.POINTER(P), C.POINTER(P),
                                     C.POINTER(P)]),
    "rad_optimizer_step_scaled": (C.c_int, [P, C.POINTER(rad_optimizer), C.c_int64, C.c_int32, C.c_int32] + [P] * 7),
    "rad_gradient_norm": (C.c_int, [P, C.c_int32, P, P, P, C.c_double, P, P]),
    "rad_clip_gradients": (C.c_int, [P, C.c_int32, P, P, P, C.c_double, P, P]),
}

_lib = None


def lib():
    """The loaded library; raises if it has not been built (no fallback)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError("librad_hip.so is missing: run `python -m paper_2007_10412_amd.build` "
                               "(there is no CPU fallback)")
        # torch ships its own HIP runtime under the same soname; it must be in the
        # process first so that this library binds to that one and not to a second copy
        import torch  # noqa: F401
        _lib = C.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(_lib, name)
            fn.restype, fn.argtypes = res, args
    return _lib


class RadError(RuntimeError):
    def __init__(self, status, text):
        super().__init__("%s: %s" % (STATUS_NAMES[status] if 0 <= status < 7 else status, text))
        self.status = status


def _check(ctx, status):
    if status != RAD_OK:
        raise RadError(status, lib().rad_last_error(ctx).decode() if ctx else "")


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def make_layer(batch, d_in, d_out, dtype=RAD_F32, relu=True, has_bias=False, conv=None):
    L = rad_layer(RAD_LINEAR, dtype, batch, d_in, d_out, int(relu), int(has_bias), 0, 0, 0, 0, 0, 0, 0)
    if conv is not None:
        L.kind = RAD_CONV2D
        L.c_in, L.h, L.w, L.c_out, L.kh, L.kw, L.pad = conv
    return L


def make_sampling(scheme, p, seed, stream_id=0, step=0):
    return rad_sampling(scheme, p, seed, stream_id, step)


def rad_fixed_k(p, d):
    return lib().rad_fixed_k(p, d)


def rad_ctx_create(stream=None):
    """stream: a torch.cuda.Stream (its HIP stream is borrowed) or None for the default stream."""
    ctx = P()
    handle = C.c_void_p(stream.cuda_stream) if stream is not None else None
    st = lib().rad_ctx_create(C.byref(ctx), handle)
    if st != RAD_OK:
        raise RadError(st, "rad_ctx_create failed (is a gfx950 device present?)")
    import torch
    ctx.device = torch.cuda.current_device()             # (the library takes the current device too)
    return ctx


def rad_last_error(ctx):
    return lib().rad_last_error(ctx).decode()


def rad_ctx_destroy(ctx):
    _check(None, lib().rad_ctx_destroy(ctx))


def rad_ctx_synchronize(ctx):
    _check(ctx, lib().rad_ctx_synchronize(ctx))


def rad_ctx_timing(ctx, filt):
    _check(ctx, lib().rad_ctx_timing(ctx, None if filt is None else filt.encode()))


def rad_ctx_timing_reset(ctx):
    _check(ctx, lib().rad_ctx_timing_reset(ctx))


def rad_ctx_timing_read(ctx, name):
    n, ms = C.c_int64(), C.c_double()
    _check(ctx, lib().rad_ctx_timing_read(ctx, None if name is None else name.encode(), C.byref(n), C.byref(ms)))
    return n.value, ms.value


def rad_ctx_timing_read_flops(ctx, name):
    a, x = C.c_double(), C.c_double()
    _check(ctx, lib().rad_ctx_timing_read_flops(ctx, None if name is None else name.encode(), C.byref(a), C.byref(x)))
    return a.value, x.value


def rad_probe_ceiling(ctx, kind, operands, sink, nbytes, reps=10):
    out = C.c_double(0.0)
    _check(ctx, lib().rad_probe_ceiling(ctx, kind, _ptr(operands), _ptr(sink), nbytes, reps, C.byref(out)))
    return out.value


def rad_debug_key_shift(ctx, shift):
    _check(ctx, lib().rad_debug_key_shift(ctx, shift))


def rad_debug_poll_limit(ctx, polls):
    _check(ctx, lib().rad_debug_poll_limit(ctx, polls))


def rad_debug_absent_groups(ctx, groups, launches):
    _check(ctx, lib().rad_debug_absent_groups(ctx, groups, launches))


def rad_debug_redone_launches(ctx):
    """(launches computed again, launches) of the last recurrent step of that kind."""
    redone, launches = C.c_int32(), C.c_int32()
    _check(ctx, lib().rad_debug_redone_launches(ctx, C.byref(redone), C.byref(launches)))
    return redone.value, launches.value


def rad_store_create(ctx, layer, scheme, p, steps=1):
    s = P()
    _check(ctx, lib().rad_store_create(ctx, C.byref(layer), scheme, p, steps, C.byref(s)))
    return s


def rad_store_destroy(store):
    lib().rad_store_destroy(store)


def rad_store_get_stats(ctx, store):
    st = rad_store_stats()
    _check(ctx, lib().rad_store_get_stats(ctx, store, C.byref(st)))
    return {k: getattr(st, k) for k, _ in rad_store_stats._fields_}


def rad_store_export_csr(ctx, store, rows):
    """Returns (row_ptr int64 [rows+1], col int32 [nnz], val float32 [nnz]) as numpy arrays."""
    nnz = rad_store_get_stats(ctx, store)["nnz"]
    row_ptr = np.zeros(rows + 1, dtype=np.int64)
    col = np.zeros(max(nnz, 1), dtype=np.int32)
    val = np.zeros(max(nnz, 1), dtype=np.float32)
    _check(ctx, lib().rad_store_export_csr(ctx, store, row_ptr.ctypes.data, col.ctypes.data, val.ctypes.data, nnz))
    return row_ptr, col[:nnz], val[:nnz]


def rad_store_export_bits(ctx, store, rows, d_out):
    words = np.zeros((rows, (d_out + 31) // 32), dtype=np.uint32)
    _check(ctx, lib().rad_store_export_bits(ctx, store, words.ctypes.data))
    return words


def rad_store_import_bits(ctx, store, words):
    words = np.ascontiguousarray(words, dtype=np.uint32)
    _check(ctx, lib().rad_store_import_bits(ctx, store, words.ctypes.data))


def rad_sample_pack(ctx, sampling, x, store, step_slot=0):
    _check(ctx, lib().rad_sample_pack(ctx, C.byref(sampling), _ptr(x), store, step_slot))


def rad_sample_pack_static(ctx, sampling, x, store):
    _check(ctx, lib().rad_sample_pack_static(ctx, C.byref(sampling), _ptr(x), store))


def rad_forward_sample(ctx, layer, sampling, x, W, bias, y, store):
    _check(ctx, lib().rad_forward_sample(ctx, C.byref(layer), C.byref(sampling), _ptr(x), _ptr(W), _ptr(bias),
                                         _ptr(y), store))


def rad_backward_dW(ctx, layer, store, dy, dW, dbias=None, beta=0.0):
    _check(ctx, lib().rad_backward_dW(ctx, C.byref(layer), store, _ptr(dy), _ptr(dW), _ptr(dbias), beta))


def rad_backward_dX(ctx, layer, store, dy, W, dX):
    _check(ctx, lib().rad_backward_dX(ctx, C.byref(layer), store, _ptr(dy), _ptr(W), _ptr(dX)))


def rad_softmax_ce(ctx, logits, labels, dtype, dlogits, loss_dev):
    rows, classes = logits.shape
    _check(ctx, lib().rad_softmax_ce(ctx, _ptr(logits), _ptr(labels), rows, classes, dtype, _ptr(dlogits),
                                     _ptr(loss_dev)))


def make_teacher(index, logit, temperature=1.0):
    """index (int32) and logit (fp32) [rows, k]: device tensors, which the teacher holds on to."""
    import torch
    if index.dtype != torch.int32 or logit.dtype != torch.float32 or index.dim() != 2 or index.shape != logit.shape:
        raise RadError(RAD_ERR_SHAPE, "a teacher's lists are int32 and fp32 tensors [rows, k]")
    if not index.is_contiguous() or not logit.is_contiguous():
        raise RadError(RAD_ERR_SHAPE, "a teacher's lists are not contiguous")
    teacher = rad_teacher(int(index.shape[1]), float(temperature), index.data_ptr(), logit.data_ptr())
    teacher.lists = index, logit
    return teacher


def _arg(name, t, n, dtype):
    """The address of a tensor (or None) that a call reads or writes as n elements of a type.  (An int, not a c_void_p: a call
    on a small layer takes as long on the host as on the device.)"""
    if t is None:
        return None
    if t.dtype is not dtype or t.numel() != n or not t.is_contiguous():
        raise RadError(RAD_ERR_SHAPE, "%s is not a contiguous tensor of %d elements of %s" % (name, n, dtype))
    return t.data_ptr()


def _kind(t, dtype):
    """The torch type of RAD_F32 or RAD_BF16; the tensor's own for a type that the library is to refuse."""
    import torch
    return torch.float32 if dtype == RAD_F32 else torch.bfloat16 if dtype == RAD_BF16 else t.dtype


def _on_device(ctx, *tensors):
    """Refuses tensors that lie elsewhere than on the context's GPU (on several, where the context's is not known): a kernel
    that was given their addresses would fault."""
    at = getattr(ctx, "device", None)
    for t in tensors:
        if t is None:
            continue
        where = t.get_device()                           # (-1: no GPU's)
        if where < 0 or (at is not None and where != at):
            raise RadError(RAD_ERR_PARAM, "a tensor on %s, not on the context's GPU" % t.device)
        at = where


def _check_lists(teacher, rows):
    have, k = teacher.lists[0].shape
    if have != rows or k != teacher.k:
        raise RadError(RAD_ERR_SHAPE, "the teacher has %d rows of %d entries, not %d of %d" % (have, k, rows, teacher.k))


def rad_distill_ce(ctx, logits, teacher, dtype, dlogits=None, row_weight=None, row_loss=None, loss=None):
    import torch
    rows, classes = logits.shape
    n, f32, kind = rows * classes, torch.float32, _kind(logits, dtype)
    _check_lists(teacher, rows)
    args = (_arg("logits", logits, n, kind), teacher, _arg("row_weight", row_weight, rows, f32), rows, classes, dtype,
            _arg("dlogits", dlogits, n, kind), _arg("row_loss", row_loss, rows, f32), _arg("loss", loss, 1, f32))
    _on_device(ctx, logits, *teacher.lists, row_weight, dlogits, row_loss, loss)
    _check(ctx, lib().rad_distill_ce(ctx, *args))


def _logprobs(rows, tokens, temperature, logprob, entropy, top_index, top_logprob):
    import torch
    f32, i32 = torch.float32, torch.int32
    if (top_index is None) != (top_logprob is None):
        raise RadError(RAD_ERR_NULL, "a list needs both of its arrays")
    k = 0
    if top_index is not None:
        if top_index.dim() != 2 or top_index.shape[0] != rows or top_index.shape != top_logprob.shape:
            raise RadError(RAD_ERR_SHAPE, "lists are tensors [rows, k] of one shape")
        k = int(top_index.shape[1])
    return rad_logprobs(temperature, _arg("tokens", tokens, rows, i32), _arg("logprob", logprob, rows, f32), _arg("entropy", entropy, rows, f32),
                        k, _arg("top_index", top_index, rows * k, i32), _arg("top_logprob", top_logprob, rows * k, f32))


def rad_token_logprobs(ctx, logits, dtype, tokens=None, temperature=1.0, logprob=None, entropy=None, top_index=None, top_logprob=None):
    """tokens: int32 [rows]; top_index (int32) and top_logprob: [rows, k]."""
    rows, classes = logits.shape
    out = _logprobs(rows, tokens, temperature, logprob, entropy, top_index, top_logprob)
    at = _arg("logits", logits, rows * classes, _kind(logits, dtype))
    _on_device(ctx, logits, tokens, logprob, entropy, top_index, top_logprob)
    _check(ctx, lib().rad_token_logprobs(ctx, at, rows, classes, dtype, out))


def rad_token_logprobs_grad(ctx, logits, dtype, dlogits, tokens=None, temperature=1.0, d_logprob=None, d_entropy=None):
    import torch
    rows, classes = logits.shape
    n, kind, f32 = rows * classes, _kind(logits, dtype), torch.float32
    args = (_arg("logits", logits, n, kind), rows, classes, dtype, _arg("tokens", tokens, rows, torch.int32), temperature,
            _arg("d_logprob", d_logprob, rows, f32), _arg("d_entropy", d_entropy, rows, f32), _arg("dlogits", dlogits, n, kind))
    _on_device(ctx, logits, tokens, d_logprob, d_entropy, dlogits)
    _check(ctx, lib().rad_token_logprobs_grad(ctx, *args))


def rad_linear_logprobs(ctx, layer, x, W, bias, tokens=None, temperature=1.0, logprob=None, entropy=None, top_index=None, top_logprob=None):
    import torch
    n, d, v = layer.batch, layer.d_in, layer.d_out
    out = _logprobs(n, tokens, temperature, logprob, entropy, top_index, top_logprob)
    td = torch.float32 if x is None else _kind(x, layer.dtype)
    args = (_arg("x", x, n * d, td), _arg("W", W, d * v, td), _arg("bias", bias, v, torch.float32))
    _on_device(ctx, x, W, bias, tokens, logprob, entropy, top_index, top_logprob)
    _check(ctx, lib().rad_linear_logprobs(ctx, layer, *args, out))


def rad_linear_logprobs_grad(ctx, layer, x, W, bias, tokens=None, temperature=1.0, d_logprob=None, d_entropy=None, dX=None, dW=None,
                             dbias=None, beta=0.0):
    """dW: an fp32 tensor, or one of the layer's type."""
    import torch
    n, d, v, f32 = layer.batch, layer.d_in, layer.d_out, torch.float32
    td = f32 if x is None else _kind(x, layer.dtype)
    dw_kind = RAD_F32
    if dW is not None and dW.dtype is not f32:
        dw_kind = RAD_BF16
        if dW.dtype is not torch.bfloat16:
            raise RadError(RAD_ERR_PARAM, "dW is fp32 or of the layer's type")
    args = (_arg("x", x, n * d, td), _arg("W", W, d * v, td), _arg("bias", bias, v, f32), _arg("tokens", tokens, n, torch.int32), temperature,
            _arg("d_logprob", d_logprob, n, f32), _arg("d_entropy", d_entropy, n, f32), _arg("dX", dX, n * d, td),
            None if dW is None else _arg("dW", dW, d * v, dW.dtype), dw_kind, _arg("dbias", dbias, v, f32), beta)
    _on_device(ctx, x, W, bias, tokens, d_logprob, d_entropy, dX, dW, dbias)
    _check(ctx, lib().rad_linear_logprobs_grad(ctx, layer, *args))


def _head_call(call, ctx, layer, x, W, bias, targets, lists, row_weight, row_loss, loss, dX, dW, dbias, beta):
    import torch
    n, d, v = layer.batch, layer.d_in, layer.d_out
    f32 = torch.float32
    td = f32 if x is None else _kind(x, layer.dtype)
    dw_kind = RAD_F32
    if dW is not None and dW.dtype is not f32:
        dw_kind = RAD_BF16
        if dW.dtype is not torch.bfloat16:
            raise RadError(RAD_ERR_PARAM, "dW is fp32 or of the layer's type")
    args = (_arg("x", x, n * d, td), _arg("W", W, d * v, td), _arg("bias", bias, v, f32), targets,
            _arg("row_weight", row_weight, n, f32), _arg("row_loss", row_loss, n, f32), _arg("loss", loss, 1, f32),
            _arg("dX", dX, n * d, td), None if dW is None else _arg("dW", dW, d * v, dW.dtype), dw_kind, _arg("dbias", dbias, v, f32), beta)
    _on_device(ctx, x, W, bias, *lists, row_weight, row_loss, loss, dX, dW, dbias)
    _check(ctx, call(ctx, layer, *args))


def rad_linear_ce(ctx, layer, x, W, bias, labels, row_weight=None, row_loss=None, loss=None, dX=None, dW=None, dbias=None,
                  beta=0.0):
    """dW: an fp32 tensor, or one of the layer's type."""
    import torch
    _head_call(lib().rad_linear_ce, ctx, layer, x, W, bias, _arg("labels", labels, layer.batch, torch.int32), (labels,), row_weight,
               row_loss, loss, dX, dW, dbias, beta)


def rad_linear_distill(ctx, layer, x, W, bias, teacher, row_weight=None, row_loss=None, loss=None, dX=None, dW=None,
                       dbias=None, beta=0.0):
    _check_lists(teacher, layer.batch)
    _head_call(lib().rad_linear_distill, ctx, layer, x, W, bias, teacher, teacher.lists, row_weight, row_loss, loss, dX, dW, dbias, beta)


def rad_model_create_mlp(ctx, dtype, batch, dims, has_bias, scheme, p):
    m = P()
    arr = (C.c_int64 * len(dims))(*dims)
    _check(ctx, lib().rad_model_create_mlp(ctx, dtype, batch, len(dims) - 1, arr, int(has_bias), scheme, p,
                                           C.byref(m)))
    return m


def rad_model_create_rnn(ctx, batch, T, d_input, hidden, classes, scheme, p):
    m = P()
    _check(ctx, lib().rad_model_create_rnn(ctx, batch, T, d_input, hidden, classes, scheme, p, C.byref(m)))
    return m


def rad_model_create_cnn(ctx, batch, channels, pool, ksize, height, width, classes, scheme, p):
    m = P()
    n_conv = len(channels) - 1
    ch = (C.c_int32 * len(channels))(*channels)
    pl = (C.c_int32 * n_conv)(*[int(v) for v in pool])
    _check(ctx, lib().rad_model_create_cnn(ctx, batch, n_conv, ch, pl, ksize, height, width, classes, scheme, p,
                                           C.byref(m)))
    return m


def rad_model_destroy(model):
    lib().rad_model_destroy(model)


def rad_model_num_stores(model):
    return lib().rad_model_num_stores(model)


def rad_model_store(model, l):
    return C.c_void_p(lib().rad_model_store(model, l))


def rad_model_export_pool_arg(ctx, model, l, n):
    out = np.zeros(n, dtype=np.uint8)
    _check(ctx, lib().rad_model_export_pool_arg(ctx, model, l, out.ctypes.data))
    return out


def rad_store_set_index_free(ctx, store, on=True):
    _check(ctx, lib().rad_store_set_index_free(ctx, store, 1 if on else 0))


def rad_model_set_index_free(ctx, model, on=True):
    _check(ctx, lib().rad_model_set_index_free(ctx, model, 1 if on else 0))


def rad_model_logits(model):
    return lib().rad_model_logits(model)


def rad_train_step(ctx, model, sampling, x, labels, params, grads, want_loss=True):
    """params/grads: lists of torch tensors in the model's documented order.  Returns the loss (float), or
    None with want_loss=False: the step is then only enqueued (loss_host = null)."""
    n = len(params)
    pa = (P * n)(*[p.data_ptr() for p in params])
    ga = (P * n)(*[g.data_ptr() for g in grads])
    if not want_loss:
        _check(ctx, lib().rad_train_step(ctx, model, C.byref(sampling), _ptr(x), _ptr(labels), pa, ga, None))
        return None
    loss = C.c_float()
    _check(ctx, lib().rad_train_step(ctx, model, C.byref(sampling), _ptr(x), _ptr(labels), pa, ga, C.byref(loss)))
    return loss.value


def make_optimizer(kind, lr, l2=0.0, beta1=0.9, beta2=0.999, eps=1e-8):
    return rad_optimizer(kind, lr, l2, beta1, beta2, eps)


def rad_optimizer_step(ctx, opt, t, dtype, params, grads, m=None, v=None, master=None):
    """params, grads, m, v, master: lists of torch tensors (m, v for RAD_ADAM; master for RAD_BF16)."""
    n = len(params)

    def arr(ts):
        return None if ts is None else (P * n)(*[x.data_ptr() for x in ts])
    counts = (C.c_int64 * n)(*[int(x.numel()) for x in params])
    _check(ctx, lib().rad_optimizer_step(ctx, C.byref(opt), int(t), dtype, n, counts, arr(params), arr(grads), arr(m),
                                         arr(v), arr(master)))


_DTYPE = operator.attrgetter("dtype")


# (T: torch.Tensor, whose methods go over a list faster than the list's tensors are asked one by one.)
def _addresses(T, tensors):
    return (P * len(tensors))(*map(T.data_ptr, tensors))


def _tensors(T, name, tensors, counts, kind):
    """The HOST array of addresses of tensors (None: no array) that are to be contiguous, of so many elements each and of one
    type."""
    if tensors is None:
        return None
    if list(map(T.numel, tensors)) != counts or set(map(_DTYPE, tensors)) - {kind} or not all(map(T.is_contiguous, tensors)):
        raise RadError(RAD_ERR_SHAPE, "%s are not %d contiguous tensors of %s elements of %s" % (name, len(counts), counts, kind))
    return _addresses(T, tensors)


def _lists_on_device(T, ctx, *lists):
    """_on_device for lists of tensors (None: none)"""
    at = getattr(ctx, "device", None)
    where = set()
    for ts in lists:
        if ts is not None:
            where.update(map(T.get_device, ts))
    if where - {at} and (at is not None or len(where) > 1 or min(where) < 0):
        _on_device(ctx, *[t for ts in lists if ts is not None for t in ts])


def _gradients(grads):
    """(counts, HOST arrays of counts, addresses and rad_dtypes) of a list of gradients, fp32 and bf16"""
    import torch
    T = torch.Tensor
    counts, kinds, n = list(map(T.numel, grads)), set(map(_DTYPE, grads)), len(grads)
    dtypes = None                                        # (all fp32)
    if kinds - {torch.float32}:
        if kinds - {torch.float32, torch.bfloat16}:
            raise RadError(RAD_ERR_PARAM, "gradients are fp32 or bf16")
        dtypes = (C.c_int32 * n)(*([RAD_BF16] * n if len(kinds) == 1 else [RAD_F32 if t.dtype is torch.float32 else RAD_BF16 for t in grads]))
    if not all(map(T.is_contiguous, grads)):
        raise RadError(RAD_ERR_SHAPE, "a gradient is not contiguous")
    return counts, (C.c_int64 * n)(*counts), _addresses(T, grads), dtypes


def rad_gradient_norm(ctx, grads, max_norm=float("inf"), norm=None, scale=None):
    """grads: a list of fp32 and bf16 tensors; norm and scale: fp32 tensors of one element, or None."""
    import torch
    _, counts, at, dtypes = _gradients(grads)
    args = (_arg("norm", norm, 1, torch.float32), _arg("scale", scale, 1, torch.float32))
    _lists_on_device(torch.Tensor, ctx, grads, [t for t in (norm, scale) if t is not None])
    _check(ctx, lib().rad_gradient_norm(ctx, len(grads), counts, at, dtypes, max_norm, *args))


def rad_clip_gradients(ctx, grads, max_norm, clipped=None, norm=None):
    """clipped: a list of tensors of the gradients' sizes and types; None: the gradients themselves."""
    import torch
    sizes, counts, at, dtypes = _gradients(grads)
    to = at
    if clipped is not None:
        T = torch.Tensor
        if list(map(T.numel, clipped)) != sizes or list(map(_DTYPE, clipped)) != list(map(_DTYPE, grads)) or not all(map(T.is_contiguous, clipped)):
            raise RadError(RAD_ERR_SHAPE, "clipped are not contiguous tensors of the gradients' sizes and types")
        to = _addresses(T, clipped)
    arg = _arg("norm", norm, 1, torch.float32)
    _lists_on_device(torch.Tensor, ctx, grads, clipped, None if norm is None else [norm])
    _check(ctx, lib().rad_clip_gradients(ctx, len(grads), counts, at, dtypes, max_norm, to, arg))


def rad_optimizer_step_scaled(ctx, opt, t, dtype, params, grads, scale, m=None, v=None, master=None):
    """As rad_optimizer_step; scale: an fp32 tensor of one element on the GPU."""
    import torch
    T, f32 = torch.Tensor, torch.float32
    counts = list(map(T.numel, params))
    kind = f32 if dtype == RAD_F32 else torch.bfloat16 if dtype == RAD_BF16 or not params else params[0].dtype
    args = ((C.c_int64 * len(counts))(*counts), _tensors(T, "params", params, counts, kind), _tensors(T, "grads", grads, counts, f32),
            _tensors(T, "m", m, counts, f32), _tensors(T, "v", v, counts, f32), _tensors(T, "master", master, counts, f32), _arg("scale", scale, 1, f32))
    _lists_on_device(T, ctx, params, grads, m, v, master, [scale])
    _check(ctx, lib().rad_optimizer_step_scaled(ctx, opt, int(t), dtype, len(counts), *args))


def make_pde_grid(n=32, steps=40960, D=0.25, dt=1.0 / 4096):
    return rad_pde_grid(n, steps, D, dt)


def rad_pde_workspace_bytes(ctx, grid, p, problems):
    out = C.c_uint64()
    _check(ctx, lib().rad_pde_workspace_bytes(ctx, C.byref(grid), p, problems, C.byref(out)))
    return out.value


def rad_pde_gradient(ctx, grid, theta, p, seed, stream_id, workspace, loss, grad, stored=None):
    """theta [problems, 7] fp64 device tensor; workspace a device byte tensor; loss [problems], grad [problems, 7]
    fp64, stored [problems] int64 or None."""
    problems = int(theta.shape[0])
    _check(ctx, lib().rad_pde_gradient(ctx, C.byref(grid), problems, _ptr(theta), p, seed, stream_id, _ptr(workspace),
                                       int(workspace.numel() * workspace.element_size()), _ptr(loss), _ptr(grad),
                                       _ptr(stored)))


def rad_path_sample_gradient(ctx, level_ptr, succ_ptr, succ, partial, y, inputs, k, seed, stream_id, adjoint, reached):
    """level_ptr: host sequence of ints; succ_ptr, succ (int32), partial (fp64), inputs (int32): device tensors;
    adjoint (fp64) and reached (int32 storage) device tensors of n_vertices entries."""
    lp = (C.c_int32 * len(level_ptr))(*[int(v) for v in level_ptr])
    g = rad_graph(int(succ_ptr.numel()) - 1, len(level_ptr) - 1, int(succ.numel()), C.cast(lp, P), succ_ptr.data_ptr(),
                  succ.data_ptr(), partial.data_ptr())
    _check(ctx, lib().rad_path_sample_gradient(ctx, C.byref(g), int(y), _ptr(inputs), int(inputs.numel()), int(k), seed,
                                               stream_id, _ptr(adjoint), _ptr(reached)))
