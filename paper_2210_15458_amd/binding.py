"""Thin ctypes binding of libarith_sampling.so (see include/arith_sampling.h).

Argument marshalling only: every function takes torch tensors that already live
on the GPU, checks device / dtype / contiguity, and passes raw pointers to the
C entry point of the same name.  Nothing is computed here and there is no
fallback: if the library is missing, loading it raises.
"""
import ctypes as C
import os

import torch

AS_F32, AS_BF16 = 0, 1
_STATUS = {0: "AS_OK", 1: "AS_ERR_INVALID_ARG", 2: "AS_ERR_UNSUPPORTED", 3: "AS_ERR_ALLOC", 4: "AS_ERR_DEVICE"}

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libarith_sampling.so")
_lib = None


ACTS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4, "softcap": 5}


class _Shaping(C.Structure):
    """as_shaping."""
    _fields_ = [("seen", C.c_void_p), ("seen_ld", C.c_int64), ("counts", C.c_void_p), ("counts_ld", C.c_int64),
                ("repetition", C.c_void_p), ("presence", C.c_void_p), ("frequency", C.c_void_p),
                ("bias", C.c_void_p), ("bias_ld", C.c_int64), ("bias_rows", C.c_int64), ("bias_ids", C.c_void_p),
                ("mask", C.c_void_p), ("mask_ld", C.c_int64), ("mask_rows", C.c_int64), ("mask_ids", C.c_void_p),
                ("finished", C.c_void_p)]


class _Cache(C.Structure):
    """as_cache."""
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("pages", C.c_int64), ("page_ld", C.c_int64), ("page_size", C.c_int32),
                ("kv_heads", C.c_int32), ("head_dim", C.c_int32), ("dtype", C.c_int)]


class _Sequences(C.Structure):
    """as_sequences."""
    _fields_ = [("table", C.c_void_p), ("table_ld", C.c_int64), ("lens", C.c_void_p), ("prompt_table", C.c_void_p),
                ("prompt_table_ld", C.c_int64), ("prompt_lens", C.c_void_p), ("rows_per_prompt", C.c_int32), ("finished", C.c_void_p)]


class ArithSamplingError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__(f"{_STATUS.get(code, code)}: {msg}")
        self.code = code


def lib():
    """Load the HIP library; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            f"{LIB_PATH} is missing: build it with `python -m paper_2210_15458_amd.build` "
            "(there is no CPU fallback)")
    L = C.CDLL(LIB_PATH)
    vp, i32, i64, f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_float
    L.as_ctx_create.argtypes = [C.POINTER(vp), i64, i32, C.c_int, vp]
    L.as_ctx_destroy.argtypes = [vp]
    L.as_last_error.argtypes = [vp]
    L.as_last_error.restype = C.c_char_p
    L.as_step.argtypes = [vp, vp, i64, i64, vp, f32, i32, f32, vp, vp]
    L.as_step_ex.argtypes = [vp, vp, i64, i64, vp, f32, i32, f32, vp, vp, vp, i32, vp, vp, vp, vp, i64]
    L.as_step_static.argtypes = [vp, C.c_int, i64, i64, i32, vp, f32, i32, f32, vp, vp, vp]
    L.as_lattice.argtypes = [vp, vp, i32, i32, vp]
    L.as_model_create_bigram.argtypes = [C.POINTER(vp), vp, vp, i32, i32, f32, C.c_int]
    L.as_model_destroy.argtypes = [vp]
    L.as_bigram_logits.argtypes = [vp, vp, vp, i64, vp, i64]
    L.as_decode.argtypes = [vp, vp, vp, i32, i32, i32, vp, f32, i32, f32, i32, vp, vp]
    L.as_interval_step.argtypes = [vp, vp, i64, i64, vp, f32, i32, f32, vp, vp, vp, i32, vp, vp, i64]
    L.as_encode.argtypes = [vp, vp, vp, i32, i32, i32, vp, f32, i32, f32, i32, vp, vp]
    L.as_decode_ancestral.argtypes = [vp, vp, vp, i32, i32, i32, vp, f32, i32, f32, i32, vp]
    L.as_estimate_mean.argtypes = [vp, vp, i32, i32, i32, vp, i32, vp]
    L.as_decode_fused.argtypes = [vp, vp, vp, i32, i32, i32, vp, f32, i32, vp, vp]
    L.as_bigram_group_mass.argtypes = [vp, vp, vp, i64, f32, vp, i64]
    L.as_step_fused.argtypes = [vp, vp, vp, i64, vp, i64, vp, f32, vp, vp, vp, i32, vp]
    shaping = C.POINTER(_Shaping)
    L.as_shape_logits.argtypes = [vp, vp, i64, i64, shaping, vp, i64]
    L.as_layer_create.argtypes = [C.POINTER(vp), vp, i64, vp, i32, i32, f32, C.c_int, f32, C.c_int]
    L.as_layer_destroy.argtypes = [vp]
    L.as_linear.argtypes = [vp, vp, vp, i64, i64, vp, i64, shaping, vp, i64, C.c_int]
    L.as_history_set.argtypes = [vp, vp, i64, vp, i64, i64, vp, vp, vp, i64, i32, vp, i64, i32, vp]
    L.as_history_add.argtypes = [vp, vp, i64, vp, i64, i64, vp, vp]
    cache, sequences = C.POINTER(_Cache), C.POINTER(_Sequences)
    L.as_cache_add.argtypes = [vp, cache, sequences, i64, vp, i64, vp, i64, i64, vp]
    L.as_attend.argtypes = [vp, cache, sequences, i64, vp, i64, i32, f32, i32, i32, vp, i64]
    L.as_attend_prompts.argtypes = [vp, cache, sequences, i64, vp, i64, i64, vp, i32, f32, i32, i32, vp, i64]
    L.as_ctx_set_tuning.argtypes = [vp, C.c_int, i32]
    L.as_ctx_set_tuning.restype = C.c_int
    L.as_ctx_profile.argtypes = [vp, C.c_int]
    L.as_ctx_profile_read.argtypes = [vp, C.c_int, C.POINTER(C.c_double), C.POINTER(i64), C.POINTER(i64)]
    L.as_ctx_profile_samples.argtypes = [vp, C.c_int, C.POINTER(C.c_float), i64, C.POINTER(i64)]
    L.as_ctx_profile_samples.restype = C.c_int
    L.as_ctx_profile.restype = C.c_int
    L.as_ctx_profile_read.restype = C.c_int
    for name in ("as_ctx_create", "as_ctx_destroy", "as_step", "as_step_ex", "as_step_static", "as_lattice",
                 "as_model_create_bigram", "as_model_destroy", "as_bigram_logits", "as_decode",
                 "as_interval_step", "as_encode", "as_decode_ancestral", "as_estimate_mean", "as_decode_fused",
                 "as_bigram_group_mass", "as_step_fused", "as_shape_logits", "as_layer_create", "as_layer_destroy",
                 "as_linear", "as_history_set", "as_history_add", "as_cache_add", "as_attend", "as_attend_prompts"):
        getattr(L, name).restype = C.c_int
    _lib = L
    return L


def _dtype_code(t):
    if t.dtype == torch.bfloat16:
        return AS_BF16
    if t.dtype == torch.float32:
        return AS_F32
    raise TypeError(f"unsupported storage dtype {t.dtype}")


def _dev(t, dtype, name, numel=None):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if numel is not None and t.numel() < numel:
        raise ValueError(f"{name} holds {t.numel()} elements, needs {numel}")
    return t.data_ptr()


class Ctx:
    """as_ctx: stream, vocabulary size, logits storage type and workspace."""

    def __init__(self, max_rows, V, logits_dtype=torch.bfloat16, stream=None):
        self._h = C.c_void_p()
        self.V = int(V)
        self.max_rows = int(max_rows)
        self.torch_dtype = logits_dtype
        self.dtype = AS_BF16 if logits_dtype == torch.bfloat16 else AS_F32
        if logits_dtype not in (torch.bfloat16, torch.float32):
            raise TypeError("logits dtype must be bfloat16 or float32")
        self.stream = torch.cuda.current_stream() if stream is None else stream
        rc = lib().as_ctx_create(C.byref(self._h), self.max_rows, self.V, self.dtype,
                                 C.c_void_p(self.stream.cuda_stream))
        if rc != 0:
            raise ArithSamplingError(rc, (lib().as_last_error(None) or b"").decode())

    def _check(self, rc):
        if rc != 0:
            raise ArithSamplingError(rc, (lib().as_last_error(self._h) or b"").decode())

    TUNING = {"step_shape": 0, "gemm_shape": 1, "thr_path": 2, "gemm_gm": 3, "workspace_mib": 4, "kept_rows": 5,
              "linear_shape": 6, "attend_shape": 7}

    def set_tuning(self, knob, value):
        """Pick a kernel variant (tests and measurements): knob is one of Ctx.TUNING."""
        self._check(lib().as_ctx_set_tuning(self._h, self.TUNING[knob], int(value)))

    def profile(self, enable):
        self._check(lib().as_ctx_profile(self._h, 1 if enable else 0))

    def profile_read(self, kernel):
        """(total kernel ms, timed launches, untimed launches) since the last read."""
        ms, n, dropped = C.c_double(), C.c_int64(), C.c_int64()
        self._check(lib().as_ctx_profile_read(self._h, int(kernel), C.byref(ms), C.byref(n), C.byref(dropped)))
        return ms.value, n.value, dropped.value

    def profile_samples(self, kernel, capacity=16384):
        """Milliseconds of each timed launch since the last read, in launch order (call before profile_read)."""
        import numpy as np
        buf = np.empty(capacity, dtype=np.float32)
        n = C.c_int64()
        self._check(lib().as_ctx_profile_samples(self._h, int(kernel), buf.ctypes.data_as(C.POINTER(C.c_float)),
                                                 capacity, C.byref(n)))
        return buf[:min(n.value, capacity)].copy()

    def close(self):
        if self._h:
            lib().as_ctx_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Model:
    """as_model: the synthetic low-rank bigram model (borrows E, re-lays U out as the current stream leaves it, which is waited for)."""

    def __init__(self, E, U, scale=3.0):
        V, d = E.shape
        if tuple(U.shape) != (d, V):
            raise ValueError("U must be [d, V] for E [V, d]")
        if E.dtype != U.dtype:
            raise TypeError("E and U must share a dtype")
        self.V, self.d = int(V), int(d)
        self._E = E                       # keep the borrowed tensor alive
        self._h = C.c_void_p()
        e, u, dtype = _dev(E, E.dtype, "E"), _dev(U, U.dtype, "U"), _dtype_code(E)
        torch.cuda.current_stream(E.device).synchronize()
        rc = lib().as_model_create_bigram(C.byref(self._h), e, u, self.V, self.d, float(scale), dtype)
        if rc != 0:
            raise ArithSamplingError(rc, (lib().as_last_error(None) or b"").decode())

    def close(self):
        if self._h:
            lib().as_model_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _logits_args(ctx, logits, rows_needed=None):
    if logits.dim() != 2:
        raise ValueError("logits must be [rows, ld]")
    ptr = _dev(logits, ctx.torch_dtype, "logits")
    return ptr, logits.shape[0], logits.shape[1]


def as_step(ctx, logits, codes, temp, top_k, top_p, tokens_out, codes_out):
    ptr, rows, ld = _logits_args(ctx, logits)
    ctx._check(lib().as_step(ctx._h, ptr, rows, ld, _dev(codes, torch.float32, "codes", rows), float(temp),
                             int(top_k), float(top_p), _dev(tokens_out, torch.int32, "tokens_out", rows),
                             _dev(codes_out, torch.float32, "codes_out", rows)))


def as_step_static(logits, V, codes, temp, top_k, top_p, tokens_out, codes_out, stream=None):
    """as_step without a context (the entry point that allocates nothing); V columns of logits [rows, ld]."""
    if logits.dim() != 2:
        raise ValueError("logits must be [rows, ld]")
    rows, ld = logits.shape
    stream = torch.cuda.current_stream() if stream is None else stream
    rc = lib().as_step_static(_dev(logits, logits.dtype, "logits"), _dtype_code(logits), rows, ld, int(V),
                              _dev(codes, torch.float32, "codes", rows), float(temp), int(top_k), float(top_p),
                              _dev(tokens_out, torch.int32, "tokens_out", rows),
                              _dev(codes_out, torch.float32, "codes_out", rows), C.c_void_p(stream.cuda_stream))
    if rc != 0:
        raise ArithSamplingError(rc, (lib().as_last_error(None) or b"").decode())


def as_step_ex(ctx, logits, codes, temp, top_k, top_p, tokens_out, codes_out, finished_in=None, eos_id=-1,
               finished_out=None, prob_out=None, flo_out=None, row_ids=None):
    ptr, lrows, ld = _logits_args(ctx, logits)
    rows = codes.numel() if row_ids is not None else lrows
    ctx._check(lib().as_step_ex(
        ctx._h, ptr, rows, ld, _dev(codes, torch.float32, "codes", rows), float(temp), int(top_k), float(top_p),
        _dev(tokens_out, torch.int32, "tokens_out", rows), _dev(codes_out, torch.float32, "codes_out", rows),
        _dev(finished_in, torch.uint8, "finished_in", rows), int(eos_id),
        _dev(finished_out, torch.uint8, "finished_out", rows), _dev(prob_out, torch.float32, "prob_out", rows),
        _dev(flo_out, torch.float32, "flo_out", rows), _dev(row_ids, torch.int32, "row_ids", rows), lrows))


def as_lattice(ctx, u, N, codes_out):
    B = u.numel()
    ctx._check(lib().as_lattice(ctx._h, _dev(u, torch.float32, "u"), B, int(N),
                                _dev(codes_out, torch.float32, "codes_out", B * int(N))))


def as_bigram_logits(ctx, model, prev, logits_out):
    ptr, rows, ld = _logits_args(ctx, logits_out)
    ctx._check(lib().as_bigram_logits(ctx._h, model._h, _dev(prev, torch.int32, "prev", rows), rows, ptr, ld))


def as_decode(ctx, model, prompts, N, T, u, temp, top_k, top_p, eos_id, tokens_out, codes_out=None):
    B = prompts.numel()
    ctx._check(lib().as_decode(
        ctx._h, model._h, _dev(prompts, torch.int32, "prompts"), B, int(N), int(T),
        _dev(u, torch.float32, "u", B), float(temp), int(top_k), float(top_p), int(eos_id),
        _dev(tokens_out, torch.int32, "tokens_out", B * int(N) * int(T)),
        _dev(codes_out, torch.float32, "codes_out", B * int(N))))


def as_interval_step(ctx, logits, tokens, temp, top_k, top_p, lo, width, finished_in=None, eos_id=-1,
                     finished_out=None, row_ids=None):
    ptr, lrows, ld = _logits_args(ctx, logits)
    rows = tokens.numel() if row_ids is not None else lrows
    ctx._check(lib().as_interval_step(
        ctx._h, ptr, rows, ld, _dev(tokens, torch.int32, "tokens", rows), float(temp), int(top_k), float(top_p),
        _dev(lo, torch.float64, "lo", rows), _dev(width, torch.float64, "width", rows),
        _dev(finished_in, torch.uint8, "finished_in", rows), int(eos_id),
        _dev(finished_out, torch.uint8, "finished_out", rows), _dev(row_ids, torch.int32, "row_ids", rows), lrows))


def as_encode(ctx, model, prompts, N, T, tokens, temp, top_k, top_p, eos_id, lo_out, width_out):
    B = prompts.numel()
    ctx._check(lib().as_encode(
        ctx._h, model._h, _dev(prompts, torch.int32, "prompts"), B, int(N), int(T),
        _dev(tokens, torch.int32, "tokens", B * int(N) * int(T)), float(temp), int(top_k), float(top_p),
        int(eos_id), _dev(lo_out, torch.float64, "lo_out", B * int(N)),
        _dev(width_out, torch.float64, "width_out", B * int(N))))


def as_decode_ancestral(ctx, model, prompts, N, T, uniforms, temp, top_k, top_p, eos_id, tokens_out):
    B = prompts.numel()
    ctx._check(lib().as_decode_ancestral(
        ctx._h, model._h, _dev(prompts, torch.int32, "prompts"), B, int(N), int(T),
        _dev(uniforms, torch.float32, "uniforms", B * int(N) * int(T)), float(temp), int(top_k), float(top_p),
        int(eos_id), _dev(tokens_out, torch.int32, "tokens_out", B * int(N) * int(T))))


def as_estimate_mean(ctx, tokens, score, eos_id, est_out):
    if tokens.dim() != 3:
        raise ValueError("tokens must be [B, N, T]")
    B, N, T = tokens.shape
    ctx._check(lib().as_estimate_mean(
        ctx._h, _dev(tokens, torch.int32, "tokens"), B, N, T, _dev(score, torch.float32, "score", ctx.V),
        int(eos_id), _dev(est_out, torch.float64, "est_out", B)))


def as_decode_fused(ctx, model, prompts, N, T, u, temp, eos_id, tokens_out, codes_out=None):
    B = prompts.numel()
    ctx._check(lib().as_decode_fused(
        ctx._h, model._h, _dev(prompts, torch.int32, "prompts"), B, int(N), int(T),
        _dev(u, torch.float32, "u", B), float(temp), int(eos_id),
        _dev(tokens_out, torch.int32, "tokens_out", B * int(N) * int(T)),
        _dev(codes_out, torch.float32, "codes_out", B * int(N))))


def as_bigram_group_mass(ctx, model, prev, temp, mass_out):
    if mass_out.dim() != 3 or mass_out.shape[2] != 2:
        raise ValueError("mass_out must be [rows, ldp, 2]")
    rows, ldp = mass_out.shape[0], mass_out.shape[1]
    ctx._check(lib().as_bigram_group_mass(ctx._h, model._h, _dev(prev, torch.int32, "prev", rows), rows, float(temp),
                                          _dev(mass_out, torch.float32, "mass_out"), ldp))


def as_step_fused(ctx, model, mass, prev, codes, temp, tokens_out, codes_out, finished_in=None, eos_id=-1,
                  finished_out=None):
    if mass.dim() != 3 or mass.shape[2] != 2:
        raise ValueError("mass must be [rows, ldp, 2]")
    rows, ldp = mass.shape[0], mass.shape[1]
    ctx._check(lib().as_step_fused(
        ctx._h, model._h, _dev(mass, torch.float32, "mass"), ldp, _dev(prev, torch.int32, "prev", rows), rows,
        _dev(codes, torch.float32, "codes", rows), float(temp), _dev(tokens_out, torch.int32, "tokens_out", rows),
        _dev(codes_out, torch.float32, "codes_out", rows), _dev(finished_in, torch.uint8, "finished_in", rows),
        int(eos_id), _dev(finished_out, torch.uint8, "finished_out", rows)))


# ------------------------------------------------------------------------------------------ layers and shaped logits

def _rows(t, dtype, name, rows, cols):
    """Pointer and row stride of a 2-D GPU tensor whose rows are contiguous, of `rows` rows and at least `cols` columns."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.dim() != 2:
        raise ValueError(f"{name} must have two dimensions")
    r, c = t.size(0), t.size(1)
    if r < rows or c < cols:
        raise ValueError(f"{name} is {r} x {c}, needs {rows} x {cols}")
    if c > 1 and t.stride(1) != 1:
        raise ValueError(f"{name} must have contiguous rows")
    if r < 2:
        return t.data_ptr(), c            # (one row: its stride says nothing)
    ld = t.stride(0)
    if ld < c:
        raise ValueError(f"{name} has rows that overlap")
    return t.data_ptr(), ld


class Layer:
    """as_layer: act(scale * x W^T + bias) for W [n, k].

    Made of W and bias as the current stream leaves them, which is waited for (the library reads them on another).  The bias is
    copied, and W if it is bf16 and k no multiple of 64 or its rows do not start on 16 bytes: later changes do not show.  Any
    other W is borrowed: it is kept alive, and what is written to it later shows in the calls behind that."""

    def __init__(self, W, bias=None, act="none", act_arg=0.0, scale=1.0):
        if not isinstance(W, torch.Tensor) or W.dim() != 2:
            raise ValueError("W must be [n, k]")
        if act not in ACTS:
            raise ValueError(f"unknown activation {act!r}: one of {', '.join(ACTS)}")
        self.n, self.k = W.shape
        self.torch_dtype = W.dtype
        self._W = W                       # keep the borrowed tensor alive
        self._h = C.c_void_p()
        ptr, ld = _rows(W, W.dtype, "W", self.n, self.k)
        bias, dtype = _dev(bias, W.dtype, "bias", self.n), _dtype_code(W)
        torch.cuda.current_stream(W.device).synchronize()
        rc = lib().as_layer_create(C.byref(self._h), ptr, ld, bias, self.n, self.k, float(scale), ACTS[act], float(act_arg), dtype)
        if rc != 0:
            raise ArithSamplingError(rc, (lib().as_last_error(None) or b"").decode())

    def close(self):
        if self._h:
            lib().as_layer_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Shaping:
    """as_shaping for `rows` rows of V logits: checked once, and the tensors kept alive; their contents may change from
    call to call.  Bit words (seen, mask) are int32 tensors."""

    def __init__(self, rows, V, seen=None, counts=None, repetition=None, presence=None, frequency=None, bias=None,
                 bias_ids=None, mask=None, mask_ids=None, finished=None):
        self.rows, self.V = int(rows), int(V)
        words = (self.V + 31) // 32
        self._tensors = (seen, counts, repetition, presence, frequency, bias, bias_ids, mask, mask_ids, finished)
        c = self._c = _Shaping()
        if seen is not None:
            c.seen, c.seen_ld = _rows(seen, torch.int32, "seen", self.rows, words)
        if counts is not None:
            c.counts, c.counts_ld = _rows(counts, torch.int32, "counts", self.rows, self.V)
        if bias is not None:
            c.bias, c.bias_ld = _rows(bias, torch.float32, "bias", 1, self.V)
            c.bias_rows = bias.shape[0]
        if mask is not None:
            c.mask, c.mask_ld = _rows(mask, torch.int32, "mask", 1, words)
            c.mask_rows = mask.shape[0]
        for name, t, dtype in (("repetition", repetition, torch.float32), ("presence", presence, torch.float32),
                               ("frequency", frequency, torch.float32), ("bias_ids", bias_ids, torch.int32),
                               ("mask_ids", mask_ids, torch.int32), ("finished", finished, torch.uint8)):
            if t is not None:
                setattr(c, name, _dev(t, dtype, name, self.rows))
        self._ref = C.byref(c)


def _shaping_ref(shaping, rows, V):
    if shaping.rows < rows or shaping.V != V:
        raise ValueError(f"shaping is for {shaping.rows} x {shaping.V} logits, not {rows} x {V}")
    return shaping._ref


def as_shape_logits(ctx, logits, shaping, logits_out):
    """The first V columns of logits [rows, >= V], shaped, to logits_out (which may be logits)."""
    rows, V = logits.size(0), ctx.V
    ptr, ld = _rows(logits, ctx.torch_dtype, "logits", rows, V)
    out, ldo = _rows(logits_out, ctx.torch_dtype, "logits_out", rows, V)
    rc = (_lib or lib()).as_shape_logits(ctx._h, ptr, rows, ld, _shaping_ref(shaping, rows, V), out, ldo)
    if rc:
        ctx._check(rc)


def as_linear(ctx, layer, x, out, residual=None, shaping=None):
    """out = act(scale * x W^T + bias) + residual, shaped: the layer's product with all that follows it in one pass."""
    rows, n, dtype = x.size(0), layer.n, out.dtype
    xp, ldx = _rows(x, layer.torch_dtype, "x", rows, layer.k)
    op, ldo = _rows(out, dtype, "out", rows, n)
    rp, ldr = (None, 0) if residual is None else _rows(residual, dtype, "residual", rows, n)
    rc = (_lib or lib()).as_linear(ctx._h, layer._h, xp, rows, ldx, rp, ldr, None if shaping is None else _shaping_ref(shaping, rows, n),
                                   op, ldo, _dtype_code(out))
    if rc:
        ctx._check(rc)


def as_history_set(ctx, seen, counts, prompts=None, prompt_offsets=None, rows_per_prompt=1, tokens=None, lens=None, which=None):
    """The record (seen [rows, words], counts [rows, >= V] or None) of ragged prompts and of tokens [rows, T]."""
    rows = seen.shape[0]
    sp, sld = _rows(seen, torch.int32, "seen", rows, (ctx.V + 31) // 32)
    cp, cld = (None, 0) if counts is None else _rows(counts, torch.int32, "counts", rows, ctx.V)
    pp, po, plen = None, None, 0
    if prompts is not None:
        plen, pp, per = prompts.numel(), _dev(prompts, torch.int32, "prompts"), int(rows_per_prompt)
        po = _dev(prompt_offsets, torch.int64, "prompt_offsets", (rows - 1) // per + 2 if per > 0 else None)
    tp, tld, T = None, 0, 0
    if tokens is not None:
        tp, tld = _rows(tokens, torch.int32, "tokens", rows, 0)
        T = tokens.shape[1]
    ctx._check(lib().as_history_set(ctx._h, sp, sld, cp, cld, rows, _dev(which, torch.uint8, "which", rows), pp, po, plen,
                                    int(rows_per_prompt), tp, tld, T, _dev(lens, torch.int32, "lens", rows)))


def as_history_add(ctx, seen, counts, tokens, finished=None):
    """One token more for each row of the record, but for finished rows."""
    rows = seen.size(0)
    sp, sld = _rows(seen, torch.int32, "seen", rows, (ctx.V + 31) // 32)
    cp, cld = (None, 0) if counts is None else _rows(counts, torch.int32, "counts", rows, ctx.V)
    ctx._check(lib().as_history_add(ctx._h, sp, sld, cp, cld, rows, _dev(tokens, torch.int32, "tokens", rows),
                                    _dev(finished, torch.uint8, "finished", rows)))


# ------------------------------------------------------------------------------- a cache and the attention that reads it

class Cache:
    """as_cache: keys and values [pages, kv_heads, page_size, head_dim], of one shape and dtype.  Borrowed: kept alive, and
    written to by as_cache_add.  Each page is contiguous; the pages may be further apart (one layer's part of a larger tensor)."""

    def __init__(self, k, v):
        for name, t in (("k", k), ("v", v)):
            if not isinstance(t, torch.Tensor) or not t.is_cuda:
                raise TypeError(f"{name} must be a GPU tensor")
            if t.dim() != 4:
                raise ValueError(f"{name} must be [pages, kv_heads, page_size, head_dim]")
        if v.shape != k.shape or v.dtype != k.dtype or v.device != k.device or v.stride() != k.stride():
            raise ValueError("k and v must have one shape, dtype, device and layout")
        pages, self.kv_heads, self.page_size, self.head_dim = k.shape
        page = self.kv_heads * self.page_size * self.head_dim
        if pages and (not k[0].is_contiguous() or (pages > 1 and k.stride(0) < page)):
            raise ValueError("the pages of k and v must be contiguous, one behind the other")
        self.torch_dtype, self.index, self.scale = k.dtype, k.get_device(), self.head_dim ** -0.5
        self._tensors = (k, v)
        c = self._c = _Cache(k.data_ptr(), v.data_ptr(), pages, k.stride(0) if pages > 1 else page, self.page_size, self.kv_heads, self.head_dim,
                             _dtype_code(k))
        self._ref = C.byref(c)


class Sequences:
    """as_sequences for `rows` rows: checked once, and the tensors kept alive; their contents may change from call to call."""

    def __init__(self, rows, table=None, lens=None, prompt_table=None, prompt_lens=None, rows_per_prompt=1, finished=None):
        self.rows = int(rows)
        self._tensors = (table, lens, prompt_table, prompt_lens, finished)
        devices = {t.get_device() for t in self._tensors if t is not None}
        if len(devices) > 1:
            raise ValueError("the sequences' tensors must be on one device")
        self.index = devices.pop() if devices else None
        c = self._c = _Sequences()
        if (table is None) != (lens is None) or (prompt_table is None) != (prompt_lens is None):
            raise ValueError("a table needs its lengths, and lengths a table")
        if table is not None:
            c.table, c.table_ld = self._table(table, "table", self.rows)
            c.lens = _dev(lens, torch.int32, "lens", self.rows)
        if prompt_table is not None:
            per = c.rows_per_prompt = int(rows_per_prompt)
            if per < 1:
                raise ValueError("rows_per_prompt must be at least 1")
            prompts = -(-self.rows // per)
            c.prompt_table, c.prompt_table_ld = self._table(prompt_table, "prompt_table", prompts)
            c.prompt_lens = _dev(prompt_lens, torch.int32, "prompt_lens", prompts)
        c.finished = _dev(finished, torch.uint8, "finished", self.rows)
        self._ref = C.byref(c)

    @staticmethod
    def _table(t, name, rows):
        ptr, ld = _rows(t, torch.int32, name, rows, 1)
        if t.size(1) != ld:
            raise ValueError(f"{name} must be contiguous")      # (its stride is how many pages a row may name)
        return ptr, ld


def _one_device(ctx, cache, seqs):
    if seqs.index not in (None, cache.index) or ctx.stream.device_index != cache.index:
        raise ValueError("the cache, the sequences and the context must be on one device")


def _tokens_of(cache, t, name, rows, cols):
    """Pointer and row stride of rows of heads, [tokens, heads * head_dim] or [tokens, heads, head_dim], on the cache's device."""
    if isinstance(t, torch.Tensor):
        shape, stride = t.shape, t.stride()
        if len(shape) == 3 and shape[1] * shape[2] == cols and stride[2] == 1 and (shape[1] < 2 or stride[1] == shape[2]):
            shape, stride = (shape[0], cols), (stride[0], 1)
        if (len(shape) == 2 and t.dtype is cache.torch_dtype and t.get_device() == cache.index and shape[0] >= rows and shape[1] >= cols
                and stride[1] == 1 and (stride[0] >= shape[1] or shape[0] < 2)):
            return t.data_ptr(), stride[0] if shape[0] > 1 else shape[1]
        if t.is_cuda and t.get_device() != cache.index:
            raise ValueError(f"{name} must be on the cache's device")
        if t.dim() == 3:
            raise ValueError(f"{name} must be [tokens, heads, head_dim] with a token's heads one behind the other, {rows} tokens of {cols} values")
    return _rows(t, cache.torch_dtype, name, rows, cols)        # (which says what it is)


def _offsets_of(cache, seqs, offsets):
    ptr = _dev(offsets, torch.int64, "offsets", seqs.rows + 1)
    if offsets.get_device() != cache.index:
        raise ValueError("offsets must be on the cache's device")
    return ptr


def as_cache_add(ctx, cache, seqs, k, v, offsets=None):
    """Keys and values [tokens, kv_heads * head_dim] (or [tokens, kv_heads, head_dim]) of the rows' last tokens into their pages:
    one a row, or with offsets [rows + 1] as many as they say."""
    _one_device(ctx, cache, seqs)
    cols = cache.kv_heads * cache.head_dim
    n, at = (seqs.rows, None) if offsets is None else (k.size(0), _offsets_of(cache, seqs, offsets))
    kp, ldk = _tokens_of(cache, k, "k", n, cols)
    vp, ldv = _tokens_of(cache, v, "v", n, cols)
    rc = (_lib or lib()).as_cache_add(ctx._h, cache._ref, seqs._ref, seqs.rows, kp, ldk, vp, ldv, n, at)
    if rc:
        ctx._check(rc)


def _heads_of(cache, q):
    cols = q.shape[1] if len(q.shape) == 2 else q.shape[1] * q.shape[2]
    heads = cols // cache.head_dim
    if heads * cache.head_dim != cols:
        raise ValueError(f"q has {cols} columns, no whole number of heads of {cache.head_dim}")
    return heads, cols


def _int32(x):
    """The nearest to x that an int32 holds (which ctypes would take the lowest bits for)."""
    return x if -0x80000000 <= x <= 0x7fffffff else 0x7fffffff if x > 0 else -0x80000000


def as_attend(ctx, cache, seqs, q, out, scale=None, window=0, sinks=0):
    """Attention of one query a row, q and out [rows, heads * head_dim] (or [rows, heads, head_dim]); scale: 1 / sqrt(head_dim)."""
    _one_device(ctx, cache, seqs)
    heads, cols = _heads_of(cache, q)
    rows = seqs.rows
    qp, ldq = _tokens_of(cache, q, "q", rows, cols)
    op, ldo = _tokens_of(cache, out, "out", rows, cols)
    rc = (_lib or lib()).as_attend(ctx._h, cache._ref, seqs._ref, rows, qp, ldq, heads, cache.scale if scale is None else float(scale),
                                   _int32(window), _int32(sinks), op, ldo)
    if rc:
        ctx._check(rc)


def as_attend_prompts(ctx, cache, seqs, q, offsets, out, scale=None, window=0, sinks=0):
    """The same for ragged queries: row r has q[offsets[r]:offsets[r + 1]], those of its last tokens."""
    _one_device(ctx, cache, seqs)
    heads, cols = _heads_of(cache, q)
    n, at = q.size(0), _offsets_of(cache, seqs, offsets)
    qp, ldq = _tokens_of(cache, q, "q", n, cols)
    op, ldo = _tokens_of(cache, out, "out", n, cols)
    rc = (_lib or lib()).as_attend_prompts(ctx._h, cache._ref, seqs._ref, seqs.rows, qp, ldq, n, at, heads, cache.scale if scale is None else float(scale),
                                           _int32(window), _int32(sinks), op, ldo)
    if rc:
        ctx._check(rc)
