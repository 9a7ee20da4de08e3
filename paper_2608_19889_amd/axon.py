"""Python binding of the C ABI in ``include/axon.h`` (ctypes).

Argument marshalling only: every step of the forward pass runs in the HIP
kernels of ``libaxon.so``.  torch supplies device memory and the current
stream; there is no fallback path.
"""
from __future__ import annotations

import ctypes
import functools
import os

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libaxon.so")

AXON_OK = 0
AXON_E_INVALID = -1
AXON_E_SHAPE = -2
AXON_E_MISSING = -3
AXON_E_DTYPE = -4
AXON_E_CAPACITY = -5
AXON_E_OOM = -6
AXON_E_HIP = -7
AXON_BF16 = 1
AXON_F32 = 2
AXON_ARCH_LLAMA = 0
AXON_ARCH_GPT2 = 1

STATUS_NAMES = {0: "AXON_OK", -1: "AXON_E_INVALID", -2: "AXON_E_SHAPE", -3: "AXON_E_MISSING",
                -4: "AXON_E_DTYPE", -5: "AXON_E_CAPACITY", -6: "AXON_E_OOM", -7: "AXON_E_HIP"}

EXPORTED = ["axon_init_model", "axon_prefill", "axon_decode_step", "axon_decode_step_noalloc", "axon_step", "axon_reset_slot", "axon_loss_and_grads",
            "axon_slot_lengths", "axon_timing_enable", "axon_timing_records", "axon_free", "axon_last_error",
            "axon_layernorm", "axon_layernorm_backward", "axon_layernorm_backward_workspace",
            "axon_token_loss_workspace", "axon_token_logprobs", "axon_token_logprobs_backward",
            "axon_preference_loss", "axon_policy_loss", "axon_preference_loss_and_grads",
            "axon_policy_loss_and_grads", "axon_rope_append", "axon_prefix_attention",
            "axon_prefix_attention_workspace", "axon_sample_tokens", "axon_sample_tokens_workspace"]

# kernel classes of the timing records
T_GEMV, T_GEMM, T_ATTN_DECODE, T_ATTN_PREFILL, T_GEMV_GROUPED, T_ATTN_BWD = 0, 1, 2, 3, 4, 5


class AxonConfig(ctypes.Structure):
    _fields_ = [("hidden", ctypes.c_int32), ("n_layers", ctypes.c_int32),
                ("n_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("intermediate", ctypes.c_int32),
                ("vocab", ctypes.c_int32), ("rms_eps", ctypes.c_float),
                ("rope_theta", ctypes.c_double), ("qkv_bias", ctypes.c_int32),
                ("tie_embeddings", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("max_batch", ctypes.c_int32), ("max_seq", ctypes.c_int32),
                ("max_tokens", ctypes.c_int32), ("kv_page_size", ctypes.c_int32),
                ("kv_num_pages", ctypes.c_int32), ("n_experts", ctypes.c_int32), ("top_k", ctypes.c_int32),
                ("moe_intermediate", ctypes.c_int32), ("n_shared_experts", ctypes.c_int32),
                ("first_moe_layer", ctypes.c_int32), ("norm_topk_prob", ctypes.c_int32),
                ("sliding_window", ctypes.c_int32), ("arch", ctypes.c_int32), ("max_positions", ctypes.c_int32)]


class AxonWeight(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char_p), ("dtype", ctypes.c_int32), ("ndim", ctypes.c_int32),
                ("shape", ctypes.c_int64 * 2), ("data", ctypes.c_void_p),
                ("on_device", ctypes.c_int32)]


class AxonKvPages(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("dtype", ctypes.c_int32),
                ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("page_size", ctypes.c_int32),
                ("num_pages", ctypes.c_int32)]


class AxonKvBatch(ctypes.Structure):
    _fields_ = [("seqs", ctypes.c_int32), ("table_stride", ctypes.c_int32), ("d_cu_seqlens", ctypes.c_void_p),
                ("h_cu_seqlens", ctypes.POINTER(ctypes.c_int32)), ("d_lens", ctypes.c_void_p),
                ("d_block_table", ctypes.c_void_p)]


class AxonKvPrefix(ctypes.Structure):
    _fields_ = [("groups", ctypes.c_int32), ("table_stride", ctypes.c_int32), ("d_cu_groups", ctypes.c_void_p),
                ("h_cu_groups", ctypes.POINTER(ctypes.c_int32)), ("d_prefix_lens", ctypes.c_void_p),
                ("d_prefix_table", ctypes.c_void_p)]


class AxonError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{STATUS_NAMES.get(code, code)}: {msg}")
        self.code = code


_lib = None


def lib():
    """Load ``libaxon.so``; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build()")
        L = ctypes.CDLL(LIB_PATH)
        L.axon_init_model.argtypes = [ctypes.POINTER(AxonConfig), ctypes.POINTER(AxonWeight), ctypes.c_int32,
                                      ctypes.c_void_p, ctypes.POINTER(ctypes.c_void_p)]
        L.axon_init_model.restype = ctypes.c_int
        L.axon_prefill.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p,
                                   ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int32),
                                   ctypes.c_int32, ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p,
                                   ctypes.c_void_p]
        L.axon_prefill.restype = ctypes.c_int
        L.axon_decode_step.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p,
                                       ctypes.c_void_p, ctypes.c_void_p]
        L.axon_decode_step.restype = ctypes.c_int
        L.axon_decode_step_noalloc.argtypes = L.axon_decode_step.argtypes
        L.axon_decode_step_noalloc.restype = ctypes.c_int
        L.axon_step.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.POINTER(ctypes.c_int32),
                                ctypes.POINTER(ctypes.c_int32), ctypes.c_void_p, ctypes.c_void_p,
                                ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int32), ctypes.c_int32,
                                ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
        L.axon_step.restype = ctypes.c_int
        L.axon_reset_slot.argtypes = [ctypes.c_void_p, ctypes.c_int32]
        L.axon_loss_and_grads.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_void_p, ctypes.c_void_p,
                                          ctypes.POINTER(ctypes.c_int32), ctypes.c_void_p, ctypes.c_void_p,
                                          ctypes.POINTER(AxonWeight), ctypes.c_int32, ctypes.c_void_p]
        L.axon_loss_and_grads.restype = ctypes.c_int
        L.axon_reset_slot.restype = ctypes.c_int
        L.axon_slot_lengths.argtypes = [ctypes.c_void_p, ctypes.POINTER(ctypes.c_int32), ctypes.c_int32]
        L.axon_slot_lengths.restype = ctypes.c_int
        L.axon_timing_enable.argtypes = [ctypes.c_void_p, ctypes.c_int32]
        L.axon_timing_enable.restype = ctypes.c_int
        L.axon_timing_records.argtypes = [ctypes.c_void_p, ctypes.POINTER(ctypes.c_int32),
                                          ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_float),
                                          ctypes.c_int32]
        L.axon_timing_records.restype = ctypes.c_int
        L.axon_free.argtypes = [ctypes.c_void_p]
        L.axon_free.restype = None
        L.axon_last_error.argtypes = []
        L.axon_last_error.restype = ctypes.c_char_p
        p, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
        i32p = ctypes.POINTER(ctypes.c_int32)
        logits = [i64, i32, p, i32, i64, p]                  # tokens, vocab, logits, dtype, ld, targets
        grad, work = [p, i32, i64], [p, i64, p]              # dlogits, dtype, ld; workspace, its bytes, stream
        step = [p, i32, p, p, i32p, p]                       # model, batch, tokens, cu_seqlens (both), targets
        grads = [ctypes.POINTER(AxonWeight), i32, p]
        paged = [ctypes.POINTER(AxonKvPages), ctypes.POINTER(AxonKvBatch)]
        shared = ctypes.POINTER(AxonKvPrefix)
        for name, args, res in [
                ("axon_preference_loss_and_grads", [*step, p, f32, f32, p, p, p, *grads], ctypes.c_int),
                ("axon_policy_loss_and_grads", [*step, p, p, p, f32, f32, f32, i32, p, p, p, *grads], ctypes.c_int),
                ("axon_layernorm", [i64, i32, p, i32, i64, p, p, i32, f32, p, i32, i64, p], ctypes.c_int),
                ("axon_layernorm_backward_workspace", [i64, i32], i64),
                ("axon_layernorm_backward", [i64, i32, p, i32, i64, p, i32, i64, p, i32, f32, p, i64, p, p, *work],
                 ctypes.c_int),
                ("axon_token_loss_workspace", [i64, i32, i32], i64),
                ("axon_token_logprobs", [*logits, p, *work], ctypes.c_int),
                ("axon_token_logprobs_backward", [*logits, p, *grad, p], ctypes.c_int),
                ("axon_preference_loss", [*logits, i32, p, i32p, p, f32, f32, p, p, p, *grad, *work], ctypes.c_int),
                ("axon_rope_append", [*paged, i64, i32, p, i64, p, i64, p, i64, p, i64, p, i32, i32, f32, p, p],
                 ctypes.c_int),
                ("axon_prefix_attention_workspace", [*paged, shared, i64, i32], i64),
                ("axon_prefix_attention", [*paged, shared, i64, i32, p, i64, f32, p, i64, p, *work], ctypes.c_int),
                ("axon_sample_tokens_workspace", [i64, i32], i64),
                ("axon_sample_tokens", [i64, i32, p, i32, i64, p, p, f32, p, i32, p, f32, p, f32, p, p, *work],
                 ctypes.c_int),
                ("axon_policy_loss", [*logits, i32, p, i32p, p, p, p, f32, f32, f32, i32, p, p, p, *grad, *work],
                 ctypes.c_int)]:
            getattr(L, name).argtypes = args
            getattr(L, name).restype = res
        _lib = L
    return _lib


def last_error() -> str:
    return lib().axon_last_error().decode()


def _check(rc: int):
    if rc < 0:
        raise AxonError(rc, last_error())
    return rc


def make_config(shape: dict, max_batch: int, max_seq: int, max_tokens: int = 0, page_size: int = 0,
                num_pages: int = 0) -> AxonConfig:
    """``shape`` uses HF-style keys (hidden_size, num_hidden_layers, ...);
    ``model_type == "gpt2"`` selects the GPT-2 family (layer_norm_epsilon,
    max_position_embeddings)."""
    gpt2 = shape.get("model_type") == "gpt2"
    return AxonConfig(
        hidden=shape["hidden_size"], n_layers=shape["num_hidden_layers"],
        n_heads=shape["num_attention_heads"], n_kv_heads=shape["num_key_value_heads"],
        head_dim=shape["head_dim"], intermediate=shape["intermediate_size"], vocab=shape["vocab_size"],
        rms_eps=shape["layer_norm_epsilon"] if gpt2 else shape["rms_norm_eps"],
        rope_theta=0.0 if gpt2 else shape["rope_theta"],
        qkv_bias=int(bool(shape["attention_bias"])), tie_embeddings=int(bool(shape["tie_word_embeddings"])),
        dtype=AXON_BF16 if shape["dtype"] == "bf16" else AXON_F32, max_batch=max_batch, max_seq=max_seq,
        max_tokens=max_tokens, kv_page_size=page_size, kv_num_pages=num_pages,
        n_experts=int(shape.get("n_routed_experts") or 0), top_k=int(shape.get("num_experts_per_tok") or 0),
        moe_intermediate=int(shape.get("moe_intermediate_size") or 0),
        n_shared_experts=int(shape.get("n_shared_experts") or 0),
        first_moe_layer=int(shape.get("first_k_dense_replace") or 0),
        norm_topk_prob=int(bool(shape.get("norm_topk_prob"))),
        sliding_window=int(shape.get("sliding_window") or 0), arch=AXON_ARCH_GPT2 if gpt2 else AXON_ARCH_LLAMA,
        max_positions=int(shape.get("max_position_embeddings") or 0) if gpt2 else 0)


def make_weights(weights: dict) -> tuple[ctypes.Array, list]:
    """Marshal {name: tensor} into an axon_weight array; returns it together
    with the objects that must stay alive for the call."""
    keep = []
    arr = (AxonWeight * len(weights))()
    for i, (name, t) in enumerate(weights.items()):
        if not t.is_contiguous():
            t = t.contiguous()
        keep.append(t)
        nb = name.encode()
        keep.append(nb)
        arr[i].name = nb
        arr[i].dtype = AXON_BF16 if t.dtype == torch.bfloat16 else (AXON_F32 if t.dtype == torch.float32 else 0)
        arr[i].ndim = t.dim()
        arr[i].shape[0] = t.shape[0] if t.dim() >= 1 else 0
        arr[i].shape[1] = t.shape[1] if t.dim() >= 2 else 0
        arr[i].data = t.data_ptr()
        arr[i].on_device = int(t.is_cuda)
    return arr, keep


def _stream(stream) -> int:
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


# ---------------------------------------------------------------- row operators

_CODES = {torch.bfloat16: AXON_BF16, torch.float32: AXON_F32}


def _code(t: torch.Tensor, name: str) -> int:
    code = _CODES.get(t.dtype)
    if code is None:
        raise ValueError(f"{name} must be bfloat16 or float32, got {t.dtype}")
    return code


def _tensors(values):
    for v in values:
        if isinstance(v, torch.Tensor):
            yield v
        elif isinstance(v, dict):
            yield from _tensors(v.values())


def _row_operator(f):
    """Runs f on its tensors' device and on ``stream`` (None: that device's current
    one), so that what it allocates belongs there.  Inputs made on another stream must
    be ready on this one; they are kept from reuse until its work is done."""
    @functools.wraps(f)
    def call(*args, stream=None, **kw):
        first, maps = None, []
        for t in (*args, *kw.values()):
            if isinstance(t, torch.Tensor):
                if first is None:
                    first, at = t, t.get_device()
                    if at < 0:
                        raise ValueError(f"{f.__name__} takes tensors on the GPU, got one on {t.device}")
                elif t.get_device() != at:
                    raise ValueError(f"{f.__name__}: tensors on {first.device} and {t.device} in one call")
            elif isinstance(t, dict):
                maps.append(t)
        if first is None:
            raise ValueError(f"{f.__name__} takes tensors on the GPU")
        for g in _tensors(maps):
            if g.get_device() != at:
                raise ValueError(f"{f.__name__}: a gradient buffer on {g.device}")
        if stream is None and at == torch.cuda.current_device():
            return f(*args, **kw)
        device = first.device
        with torch.cuda.device(device):
            if stream is None:
                return f(*args, **kw)
            if not hasattr(stream, "cuda_stream"):
                stream = torch.cuda.ExternalStream(int(stream))
            if stream.device != device:
                raise ValueError(f"{f.__name__}: tensors on {device}, the stream on {stream.device}")
            for t in _tensors((*args, *kw.values())):
                t.record_stream(stream)
            with torch.cuda.stream(stream):
                return f(*args, **kw)
    call.__doc__ = (f.__doc__ or "") + """

    ``stream``: the torch stream (or its raw handle) to run on; None: the current one.
    Not recorded by autograd: the results have no history, whatever the inputs require."""
    return call


def _current(t: torch.Tensor) -> int:
    """The current stream of t's device, as the C ABI takes it."""
    return torch._C._cuda_getCurrentRawStream(t.get_device())


def _rows(t: torch.Tensor, name: str, out: bool = False):
    """(the tensor, rows, columns, row stride) of a tensor whose last dimension is
    its columns.  An input of another layout is copied; an output is refused."""
    v = t
    if t.dim() != 2:
        if t.dim() == 0:
            raise ValueError(f"{name} has no columns")
        try:
            v = t.view(-1, t.shape[-1]) if t.shape[-1] else t.reshape(0, 0)
        except RuntimeError:
            v = None
    if v is not None:
        rows, cols = v.shape
        ld, one = v.stride()
        if rows < 2:
            ld = max(cols, 1)
        if (one == 1 or cols < 2) and ld >= cols:
            return v, rows, cols, ld
    if out:
        raise ValueError(f"{name} must have contiguous columns and rows that do not overlap")
    v = t.contiguous().view(-1, t.shape[-1])
    return v, v.shape[0], v.shape[1], max(v.shape[1], 1)


def _vector(t, n: int, dtype, name: str):
    """``t`` as n contiguous values of ``dtype`` (None stays None)."""
    if t is None:
        return None
    if t.dtype != dtype or t.numel() != n:
        raise ValueError(f"{name} must hold {n} {dtype} values, got {t.numel()} {t.dtype}")
    return t.contiguous()


def _ptr(t):
    return None if t is None else t.data_ptr()


def _like(out, x: torch.Tensor, dtype, name: str) -> torch.Tensor:
    """The caller's output buffer (of any dtype when dtype is None), or a new one of
    x's shape."""
    if out is None:
        return torch.empty_like(x, dtype=dtype, memory_format=torch.contiguous_format)
    if out.shape != x.shape or (dtype is not None and out.dtype != dtype):
        raise ValueError(f"{name} must be {tuple(x.shape)} {dtype or ''}, got {tuple(out.shape)} {out.dtype}")
    torch.autograd.graph.increment_version(out)  # (written through a pointer, which autograd does not see)
    return out


@_row_operator
def layernorm(x: torch.Tensor, gain: torch.Tensor, bias: torch.Tensor | None = None, eps: float = 1e-5,
              dtype: torch.dtype | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    """Layer norm over the last dimension of ``x`` (axon_layernorm), in ``dtype``
    (x's by default; ``out`` may be x)."""
    y = _like(out, x, x.dtype if dtype is None and out is None else dtype, "out")
    xv, rows, cols, ldx = _rows(x, "x")
    yv, _, _, ldy = _rows(y, "out", out=True)
    gain = _vector(gain, cols, gain.dtype, "gain")
    bias = _vector(bias, cols, gain.dtype, "bias")
    _check(lib().axon_layernorm(rows, cols, xv.data_ptr(), _code(x, "x"), ldx, gain.data_ptr(), _ptr(bias),
                                _code(gain, "gain"), eps, yv.data_ptr(), _code(y, "out"), ldy, _current(x)))
    return y


@_row_operator
def layernorm_backward(dy: torch.Tensor, x: torch.Tensor, gain: torch.Tensor, eps: float = 1e-5,
                       dx: torch.Tensor | None = None):
    """(dx, dgain, dbias) of :func:`layernorm` from the gradient ``dy`` of its
    output (axon_layernorm_backward): dx in x's dtype (``dx`` may be x or dy), dgain
    and dbias float32."""
    if dy.shape != x.shape:
        raise ValueError(f"dy has shape {tuple(dy.shape)}, x {tuple(x.shape)}")
    dx = _like(dx, x, x.dtype, "dx")
    xv, rows, cols, ldx = _rows(x, "x")
    dv, _, _, lddy = _rows(dy, "dy")
    ov, _, _, lddx = _rows(dx, "dx", out=True)
    gain = _vector(gain, cols, gain.dtype, "gain")
    dgain = torch.empty(cols, dtype=torch.float32, device=x.device)
    dbias = torch.empty_like(dgain)
    need = lib().axon_layernorm_backward_workspace(rows, cols)
    ws = torch.empty(need, dtype=torch.uint8, device=x.device)
    _check(lib().axon_layernorm_backward(rows, cols, xv.data_ptr(), _code(x, "x"), ldx, dv.data_ptr(), _code(dy, "dy"),
                                         lddy, gain.data_ptr(), _code(gain, "gain"), eps, ov.data_ptr(), lddx,
                                         dgain.data_ptr(), dbias.data_ptr(), ws.data_ptr(), need, _current(x)))
    return dx, dgain, dbias


def _logit_args(logits, targets):
    z, tokens, vocab, ld = _rows(logits, "logits")
    tg = _vector(targets, tokens, torch.int32, "targets")
    return z, tg, (tokens, vocab, z.data_ptr(), _code(logits, "logits"), ld, tg.data_ptr())


def _loss_workspace(tokens, vocab, seqs, like):
    need = lib().axon_token_loss_workspace(tokens, vocab, seqs)
    return torch.empty(need, dtype=torch.uint8, device=like.device), need


def _grad(dlogits, logits, wanted=True):
    """(the gradient's tensor, a view that keeps its rows, their C arguments)"""
    if not wanted:
        return None, None, (None, AXON_F32, 0)
    g = _like(dlogits, logits, logits.dtype if dlogits is None else None, "dlogits")
    v, _, _, ld = _rows(g, "dlogits", out=True)
    return g, v, (v.data_ptr(), _code(g, "dlogits"), ld)


def _cu_args(cu_seqlens, cu_device, like):
    n = len(cu_seqlens)
    host = (ctypes.c_int32 * max(n, 1))(*cu_seqlens)
    if cu_device is None:
        return host, torch.tensor(cu_seqlens, dtype=torch.int32, device=like.device)
    if cu_device.dtype != torch.int32 or cu_device.numel() < n or not cu_device.is_contiguous():
        raise ValueError(f"cu_device must hold the {n} int32 values of cu_seqlens")
    return host, cu_device


@_row_operator
def token_logprobs(logits: torch.Tensor, targets: torch.Tensor) -> torch.Tensor:
    """logits[t][targets[t]] - logsumexp(logits[t]) (axon_token_logprobs): logits [tokens,
    vocab] float32 or bfloat16, targets int32 [tokens] (a value outside [0, vocab)
    does not count and gives 0).  Returns float32 [tokens]."""
    z, tg, args = _logit_args(logits, targets)
    out = torch.empty(args[0], dtype=torch.float32, device=z.device)
    ws, need = _loss_workspace(args[0], args[1], 0, z)
    _check(lib().axon_token_logprobs(*args, out.data_ptr(), ws.data_ptr(), need, _current(z)))
    return out


@_row_operator
def token_logprobs_backward(logits: torch.Tensor, targets: torch.Tensor, dlogps: torch.Tensor,
                            dlogits: torch.Tensor | None = None) -> torch.Tensor:
    """The gradient at the logits of a loss whose gradient at
    :func:`token_logprobs` is ``dlogps`` (float32 [tokens]).  ``dlogits``: a buffer
    for it, of either dtype (the logits' own is allowed); by default a new one of the
    logits' dtype."""
    z, tg, args = _logit_args(logits, targets)
    dlogps = _vector(dlogps, args[0], torch.float32, "dlogps")
    g, gv, gargs = _grad(dlogits, logits)
    _check(lib().axon_token_logprobs_backward(*args, dlogps.data_ptr(), *gargs, _current(z)))
    return g


@_row_operator
def preference_loss(logits: torch.Tensor, targets: torch.Tensor, cu_seqlens: list,
                    ref_logps: torch.Tensor | None = None, beta: float = 0.1, label_smoothing: float = 0.0,
                    dlogits: torch.Tensor | None = None, want_grad: bool = True,
                    cu_device: torch.Tensor | None = None):
    """Preference loss over pairs of sequences packed back to back, chosen then
    rejected (axon_preference_loss): cu_seqlens a host list of 2 pairs + 1 prefix sums
    (cu_device: the same in a device int32 buffer, which saves its copy; a captured
    call needs it), ref_logps float32 [2 pairs], each sequence's log-probability under
    the reference model (None: zeros).  Returns (loss [1], seq_logps [2 pairs],
    margins [pairs], dlogits or None); ``dlogits`` as in :func:`token_logprobs_backward`."""
    pairs = (len(cu_seqlens) - 1) // 2
    if len(cu_seqlens) != 2 * pairs + 1 or pairs < 1:
        raise ValueError("cu_seqlens must have an odd number of entries, at least 3: sequences come in pairs")
    z, tg, args = _logit_args(logits, targets)
    ref_logps = _vector(ref_logps, 2 * pairs, torch.float32, "ref_logps")
    g, gv, gargs = _grad(dlogits, logits, want_grad)
    host, cu = _cu_args(cu_seqlens, cu_device, z)
    out = torch.empty(1 + 3 * pairs, dtype=torch.float32, device=z.device)
    at = out.data_ptr()
    ws, need = _loss_workspace(args[0], args[1], 2 * pairs, z)
    _check(lib().axon_preference_loss(*args, pairs, cu.data_ptr(), host, _ptr(ref_logps), beta, label_smoothing, at,
                                      at + 4, at + 4 + 8 * pairs, *gargs, ws.data_ptr(), need, _current(z)))
    loss, seq, margins = out.split_with_sizes((1, 2 * pairs, pairs))
    return loss, seq, margins, g


@_row_operator
def policy_loss(logits: torch.Tensor, targets: torch.Tensor, cu_seqlens: list, old_logps: torch.Tensor,
                advantages: torch.Tensor, ref_logps: torch.Tensor | None = None, clip_low: float = 0.2,
                clip_high: float = 0.2, kl_coef: float = 0.0, per_sequence: bool = False,
                dlogits: torch.Tensor | None = None, want_grad: bool = True,
                cu_device: torch.Tensor | None = None):
    """Clipped policy loss with a KL term (axon_policy_loss): old_logps, advantages
    and ref_logps (None: no KL term) float32 [tokens]; averaged over the counted
    tokens, or over each sequence's and then the sequences (per_sequence).  Returns
    (loss [1], stats [3], logps [tokens], dlogits or None)."""
    z, tg, args = _logit_args(logits, targets)
    tokens, batch = args[0], len(cu_seqlens) - 1
    old_logps = _vector(old_logps, tokens, torch.float32, "old_logps")
    advantages = _vector(advantages, tokens, torch.float32, "advantages")
    ref_logps = _vector(ref_logps, tokens, torch.float32, "ref_logps")
    g, gv, gargs = _grad(dlogits, logits, want_grad)
    host, cu = _cu_args(cu_seqlens, cu_device, z)
    out = torch.empty(4 + tokens, dtype=torch.float32, device=z.device)
    at = out.data_ptr()
    ws, need = _loss_workspace(tokens, args[1], batch, z)
    _check(lib().axon_policy_loss(*args, batch, cu.data_ptr(), host, old_logps.data_ptr(), _ptr(ref_logps),
                                  advantages.data_ptr(), clip_low, clip_high, kl_coef, int(per_sequence), at, at + 4,
                                  at + 16, *gargs, ws.data_ptr(), need, _current(z)))
    loss, stats, logps = out.split_with_sizes((1, 3, tokens))
    return loss, stats, logps, g


# ---------------------------------------------------------------- sampling answers

def _head_rows(t: torch.Tensor, heads, hd: int, dtype, name: str, out: bool = False):
    """(the tensor, its row stride) of [tokens, heads, hd] with contiguous heads.  An
    input of another layout is copied; an output is refused."""
    shape = t.shape
    if len(shape) != 3 or shape[2] != hd or (heads is not None and shape[1] != heads) or t.dtype != dtype:
        raise ValueError(f"{name} must be [tokens, {heads or 'heads'}, {hd}] {dtype}, got {tuple(shape)} {t.dtype}")
    row = shape[1] * hd
    ld, step, one = t.stride()
    if one == 1 and (step == hd or shape[1] < 2) and (ld >= row or shape[0] < 2):
        return t, max(ld, row)
    if out:
        raise ValueError(f"{name} must have contiguous heads and rows that do not overlap")
    return t.contiguous(), row


def _pages_arg(k_cache: torch.Tensor, v_cache: torch.Tensor) -> AxonKvPages:
    shape = k_cache.shape
    if len(shape) != 4 or shape != v_cache.shape or k_cache.dtype != v_cache.dtype:
        raise ValueError("k_cache and v_cache must be [pages, kv heads, page size, head dim] of one type, got "
                         f"{tuple(shape)} {k_cache.dtype} and {tuple(v_cache.shape)} {v_cache.dtype}")
    if not (k_cache.is_contiguous() and v_cache.is_contiguous()):
        raise ValueError("k_cache and v_cache must be contiguous")
    pages, kv, ps, hd = shape
    return AxonKvPages(k_cache.data_ptr(), v_cache.data_ptr(), _code(k_cache, "the cache"), kv, hd, ps, pages)


def _table(t: torch.Tensor, lens: torch.Tensor, name: str, lens_name: str):
    """(the tables, their lengths, rows, columns)"""
    shape = t.shape
    if len(shape) != 2 or t.dtype != torch.int32:
        raise ValueError(f"{name} must be int32 [sequences, pages], got {tuple(shape)} {t.dtype}")
    return t.contiguous(), _vector(lens, shape[0], torch.int32, lens_name), shape[0], shape[1]


def _sums(values, device_copy, n: int, name: str, like):
    """(host array, device tensor) of n + 1 prefix sums; (None, None) for None."""
    if values is None:
        return None, None
    if len(values) != n + 1:
        raise ValueError(f"{name} must have {n + 1} entries, got {len(values)}")
    return _cu_args(values, device_copy, like)


def _batch_arg(block_table, lens, cu_seqlens, cu_device, like):
    """The C structure and the tensors that it points at."""
    table, lens, seqs, columns = _table(block_table, lens, "block_table", "lens")
    host, cu = _sums(cu_seqlens, cu_device, seqs, "cu_seqlens", like)
    return AxonKvBatch(seqs, columns, _ptr(cu), host, lens.data_ptr(), table.data_ptr()), (table, lens, cu)


@_row_operator
def rope_append(q: torch.Tensor | None, k: torch.Tensor, v: torch.Tensor, k_cache: torch.Tensor,
                v_cache: torch.Tensor, block_table: torch.Tensor, lens: torch.Tensor,
                inv_freq: torch.Tensor | None = None, cu_seqlens: list | None = None,
                cu_device: torch.Tensor | None = None, offsets: torch.Tensor | None = None,
                interleaved: bool = False, scale: float = 1.0, out: torch.Tensor | None = None):
    """Rotates the new tokens' q [tokens, heads, head dim] and k [tokens, kv heads, head
    dim] by their positions and stores k and v in the paged cache [pages, kv heads, page
    size, head dim] (axon_rope_append); returns the rotated q (``out`` may be q; None for
    q None).  block_table int32 [sequences, pages]; lens int32 [sequences], the keys that
    each had before (negative: it takes no part); cu_seqlens a host list of prefix sums of
    the tokens (None: one each; cu_device as in :func:`preference_loss`); inv_freq float64
    [rotated dimensions / 2] (None: no rotation); offsets int32 [sequences], the position
    of each one's first key."""
    pages = _pages_arg(k_cache, v_cache)
    hd, dtype = pages.head_dim, k_cache.dtype
    kv, ldk = _head_rows(k, pages.kv_heads, hd, dtype, "k")
    vv, ldv = _head_rows(v, pages.kv_heads, hd, dtype, "v")
    tokens = k.shape[0]
    batch, keep = _batch_arg(block_table, lens, cu_seqlens, cu_device, k)
    if v.shape[0] != tokens or (q is not None and q.shape[0] != tokens):
        raise ValueError("q, k and v must have the same tokens")
    rot = 0
    if inv_freq is not None:
        rot = 2 * inv_freq.numel()
        inv_freq = _vector(inv_freq, rot // 2, torch.float64, "inv_freq")
    offsets = _vector(offsets, block_table.shape[0], torch.int32, "offsets")
    heads, qv, ldq, ov, ldo = 0, None, 0, None, 0
    if q is not None:
        qv, ldq = _head_rows(q, None, hd, dtype, "q")
        heads = q.shape[1]
        out = _like(out, q, dtype, "out")
        ov, ldo = _head_rows(out, heads, hd, dtype, "out", out=True)
    elif out is not None:
        raise ValueError("out without q")
    _check(lib().axon_rope_append(pages, batch, tokens, heads, _ptr(qv), ldq, kv.data_ptr(), ldk, vv.data_ptr(), ldv,
                                  _ptr(ov), ldo, _ptr(inv_freq), rot, int(interleaved), scale, _ptr(offsets), _current(k)))
    torch.autograd.graph.increment_version((k_cache, v_cache))
    return out


@_row_operator
def prefix_attention(q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, block_table: torch.Tensor,
                     lens: torch.Tensor, prefix_table: torch.Tensor | None = None,
                     prefix_lens: torch.Tensor | None = None, cu_groups: list | None = None,
                     groups_device: torch.Tensor | None = None, cu_seqlens: list | None = None,
                     cu_device: torch.Tensor | None = None, scale: float | None = None,
                     out: torch.Tensor | None = None, want_lse: bool = False):
    """Attention of new tokens q [tokens, heads, head dim], already in the cache, over a
    prefix that sequences share and each one's own keys up to the token itself
    (axon_prefix_attention).  Cache, block_table, lens and cu_seqlens as the
    :func:`rope_append` before it took them.  prefix_table int32 [groups, pages] and
    prefix_lens int32 [groups]; cu_groups a host list of prefix sums of the groups'
    sequences (None: one group of all; groups_device its device copy, which a captured call
    with cu_groups needs).  scale: 1 / sqrt(head dim) by default; ``out`` may be q.  Returns
    out, with want_lse (out, logarithms of the sums, float32 [tokens, heads])."""
    pages = _pages_arg(k_cache, v_cache)
    hd, dtype = pages.head_dim, k_cache.dtype
    qv, ldq = _head_rows(q, None, hd, dtype, "q")
    tokens, heads = q.shape[:2]
    batch, keep = _batch_arg(block_table, lens, cu_seqlens, cu_device, q)
    prefix = None
    if prefix_table is not None:
        if prefix_lens is None:
            raise ValueError("prefix_table without prefix_lens")
        table, plens, groups, columns = _table(prefix_table, prefix_lens, "prefix_table", "prefix_lens")
        if cu_groups is None:
            if groups != 1:
                raise ValueError("several groups need cu_groups")
            cu_groups = [0, batch.seqs]
            if groups_device is None and batch.seqs:  # (filled on the device: no capture takes a copy from the host)
                groups_device = torch.arange(0, batch.seqs + 1, batch.seqs, dtype=torch.int32, device=q.device)
        host, cu = _sums(cu_groups, groups_device, groups, "cu_groups", q)
        prefix = AxonKvPrefix(groups, columns, cu.data_ptr(), host, plens.data_ptr(), table.data_ptr())
        keep = (keep, table, plens, cu)
    elif prefix_lens is not None or cu_groups is not None:
        raise ValueError("prefix_lens and cu_groups need prefix_table")
    out = _like(out, q, dtype, "out")
    ov, ldo = _head_rows(out, heads, hd, dtype, "out", out=True)
    lse = torch.empty((tokens, heads), dtype=torch.float32, device=q.device) if want_lse else None
    need = lib().axon_prefix_attention_workspace(pages, batch, prefix, tokens, heads)
    ws = torch.empty(need, dtype=torch.uint8, device=q.device)
    _check(lib().axon_prefix_attention(pages, batch, prefix, tokens, heads, qv.data_ptr(), ldq,
                                       hd ** -0.5 if scale is None else scale, ov.data_ptr(), ldo, _ptr(lse),
                                       ws.data_ptr(), need, _current(q)))
    return (out, lse) if want_lse else out


def _setting(value, rows: int, dtype, name: str):
    """(an array over the rows or None, the number for all of them)"""
    if isinstance(value, torch.Tensor):
        return _vector(value, rows, dtype, name), 0
    if dtype == torch.int32:  # (of a longer number ctypes would hand over the low 32 bits)
        value = max(-(1 << 31), min(value, (1 << 31) - 1))
    return None, value


@_row_operator
def sample_tokens(logits: torch.Tensor, uniform: torch.Tensor, temperature: float | torch.Tensor = 1.0,
                  top_k: int | torch.Tensor = 0, top_p: float | torch.Tensor = 1.0,
                  min_p: float | torch.Tensor = 0.0, out: torch.Tensor | None = None):
    """Draws a token from each row of logits [rows, vocab] (float32 or bfloat16) by its
    number uniform (float32 [rows], in [0, 1)), after temperature, top-k, top-p and min-p,
    each a number or a tensor over the rows (int32 for top_k, else float32); temperature 0
    takes the largest, top_k 0, top_p 1 and min_p 0 keep all (axon_sample_tokens).  Returns
    (tokens int32 [rows] (``out`` if given), logprobs float32 [rows]: under the distribution
    drawn from; :func:`token_logprobs` gives the model's)."""
    z, rows, vocab, ld = _rows(logits, "logits")
    uniform = _vector(uniform, rows, torch.float32, "uniform")
    settings = [_setting(v, rows, t, n) for v, t, n in (
        (temperature, torch.float32, "temperature"), (top_k, torch.int32, "top_k"), (top_p, torch.float32, "top_p"),
        (min_p, torch.float32, "min_p"))]
    if out is None:
        out = torch.empty(rows, dtype=torch.int32, device=z.device)
    else:
        if out.shape != (rows,) or out.dtype != torch.int32 or not out.is_contiguous():
            raise ValueError(f"out must be int32 [{rows}] and contiguous")
        torch.autograd.graph.increment_version(out)
    logps = torch.empty(rows, dtype=torch.float32, device=z.device)
    need = lib().axon_sample_tokens_workspace(rows, vocab)
    ws = torch.empty(need, dtype=torch.uint8, device=z.device)
    _check(lib().axon_sample_tokens(rows, vocab, z.data_ptr(), _code(logits, "logits"), ld, uniform.data_ptr(),
                                    *(x for t, n in settings for x in (_ptr(t), n)), out.data_ptr(), logps.data_ptr(),
                                    ws.data_ptr(), need, _current(z)))
    return out, logps


class Model:
    """One decoder model resident on the current GPU."""

    def __init__(self, shape: dict, weights: dict, max_batch: int, max_seq: int, max_tokens: int = 0,
                 page_size: int = 0, num_pages: int = 0, stream=None):
        self.shape = dict(shape)
        self.vocab = shape["vocab_size"]
        self.max_batch = max_batch
        self.cfg = make_config(shape, max_batch, max_seq, max_tokens, page_size, num_pages)
        arr, keep = make_weights(weights)
        handle = ctypes.c_void_p()
        _check(lib().axon_init_model(ctypes.byref(self.cfg), arr, len(weights), ctypes.c_void_p(_stream(stream)),
                                     ctypes.byref(handle)))
        del keep
        self._h = handle
        self.device = torch.device("cuda", torch.cuda.current_device())

    # ---- calls
    def prefill(self, tokens: torch.Tensor, cu_seqlens: list, block_table: torch.Tensor | None = None,
                all_logits: bool = False, logits: torch.Tensor | None = None,
                next_tokens: torch.Tensor | None = None, want_logits: bool = True, stream=None):
        """tokens: device int32 [sum S_b]; cu_seqlens: host list of batch+1 ints;
        block_table: host int32 [batch, stride] for a paged cache.  Returns
        (logits or None, next_tokens)."""
        dev = tokens.device
        B = len(cu_seqlens) - 1
        cu_h = (ctypes.c_int32 * (B + 1))(*[int(c) for c in cu_seqlens])
        cu_d = torch.tensor([int(c) for c in cu_seqlens], dtype=torch.int32, device=dev)
        rows = int(cu_seqlens[-1]) if all_logits else B
        if logits is None and (want_logits or all_logits):
            logits = torch.empty((rows, self.vocab), dtype=torch.float32, device=dev)
        if next_tokens is None:
            next_tokens = torch.empty((B,), dtype=torch.int32, device=dev)
        bt_ptr, stride = None, 0
        if block_table is not None:
            bt = block_table.to("cpu", torch.int32).contiguous()
            stride = bt.shape[1]
            bt_ptr = ctypes.cast(bt.data_ptr(), ctypes.POINTER(ctypes.c_int32))
        _check(lib().axon_prefill(self._h, B, tokens.data_ptr(), cu_d.data_ptr(), cu_h, bt_ptr, stride,
                                  int(all_logits), logits.data_ptr() if logits is not None else None,
                                  next_tokens.data_ptr(), ctypes.c_void_p(_stream(stream))))
        self._keep = (cu_d, tokens)
        return logits, next_tokens

    def loss_and_grads(self, tokens: torch.Tensor, cu_seqlens: list, targets: torch.Tensor, grads: dict,
                       loss: torch.Tensor | None = None, stream=None):
        """Backward pass (axon_loss_and_grads): tokens / targets device int32
        [sum S_b] (targets -1 or outside [0, V) are not counted); grads: {weight
        name: device float32 tensor of that weight's shape}, overwritten with
        the gradient of the mean cross-entropy.  Returns the loss (device
        float32 [1])."""
        dev = tokens.device
        B = len(cu_seqlens) - 1
        cu_h = (ctypes.c_int32 * (B + 1))(*[int(c) for c in cu_seqlens])
        cu_d = torch.tensor([int(c) for c in cu_seqlens], dtype=torch.int32, device=dev)
        if loss is None:
            loss = torch.empty((1,), dtype=torch.float32, device=dev)
        arr, keep = make_weights(grads)
        _check(lib().axon_loss_and_grads(self._h, B, tokens.data_ptr(), cu_d.data_ptr(), cu_h, targets.data_ptr(),
                                         loss.data_ptr(), arr, len(grads), ctypes.c_void_p(_stream(stream))))
        self._keep = (cu_d, tokens, targets, keep)
        return loss

    def _check_device(self, tokens):
        if tokens.device != self.device:
            raise ValueError(f"tensors on {tokens.device}, the model on {self.device}")

    def _train_args(self, tokens, cu_seqlens, targets, grads):
        """The C arguments up to the targets, those of the gradients, and what has to
        live until the step has run."""
        B = len(cu_seqlens) - 1
        T = int(cu_seqlens[-1])
        tokens, targets = _vector(tokens, T, torch.int32, "tokens"), _vector(targets, T, torch.int32, "targets")
        for name, g in grads.items():
            if not g.is_contiguous():
                raise ValueError(f"the gradient buffer of {name} is not contiguous")
        host, cu = _cu_args([int(c) for c in cu_seqlens], None, tokens)
        arr, keep = make_weights(grads)
        return (tokens.data_ptr(), cu.data_ptr(), host, targets.data_ptr()), \
            (arr, len(grads), _current(tokens)), (cu, tokens, targets, keep)

    @_row_operator
    def preference_loss_and_grads(self, tokens: torch.Tensor, cu_seqlens: list, targets: torch.Tensor, grads: dict,
                                  ref_logps: torch.Tensor | None = None, beta: float = 0.1,
                                  label_smoothing: float = 0.0):
        """A training step with the preference loss (axon_preference_loss_and_grads):
        pairs of sequences, chosen then rejected; tokens, targets and grads as in
        :meth:`loss_and_grads`, the loss as :func:`preference_loss`.  Returns (loss [1],
        seq_logps [2 pairs], margins [pairs])."""
        B = len(cu_seqlens) - 1
        if B < 2 or B % 2:
            raise ValueError("sequences come in pairs, chosen then rejected")
        self._check_device(tokens)
        args, gargs, keep = self._train_args(tokens, cu_seqlens, targets, grads)
        ref_logps = _vector(ref_logps, B, torch.float32, "ref_logps")
        out = torch.empty((1 + B + B // 2,), dtype=torch.float32, device=tokens.device)
        at = out.data_ptr()
        _check(lib().axon_preference_loss_and_grads(self._h, B // 2, *args, _ptr(ref_logps), beta, label_smoothing, at,
                                                    at + 4, at + 4 + 4 * B, *gargs))
        self._keep = (keep, ref_logps)
        return out[:1], out[1:1 + B], out[1 + B:]

    @_row_operator
    def policy_loss_and_grads(self, tokens: torch.Tensor, cu_seqlens: list, targets: torch.Tensor, grads: dict,
                              old_logps: torch.Tensor, advantages: torch.Tensor,
                              ref_logps: torch.Tensor | None = None, clip_low: float = 0.2, clip_high: float = 0.2,
                              kl_coef: float = 0.0, per_sequence: bool = False):
        """A training step with the clipped policy loss (axon_policy_loss_and_grads):
        tokens, targets and grads as in :meth:`loss_and_grads`, the loss as
        :func:`policy_loss`.  Returns (loss [1], stats [3], logps [tokens])."""
        self._check_device(tokens)
        args, gargs, keep = self._train_args(tokens, cu_seqlens, targets, grads)
        T = int(cu_seqlens[-1])
        old_logps, advantages, ref_logps = (_vector(t, T, torch.float32, n) for t, n in (
            (old_logps, "old_logps"), (advantages, "advantages"), (ref_logps, "ref_logps")))
        out = torch.empty((4 + T,), dtype=torch.float32, device=tokens.device)
        at = out.data_ptr()
        _check(lib().axon_policy_loss_and_grads(self._h, len(cu_seqlens) - 1, *args, old_logps.data_ptr(),
                                                _ptr(ref_logps), advantages.data_ptr(), clip_low, clip_high, kl_coef,
                                                int(per_sequence), at, at + 4, at + 16, *gargs))
        self._keep = (keep, old_logps, advantages, ref_logps)
        return out[:1], out[1:4], out[4:]

    def decode_step(self, tokens: torch.Tensor, logits: torch.Tensor | None = None,
                    next_tokens: torch.Tensor | None = None, stream=None):
        """tokens: device int32 [batch].  Returns (logits or None, next_tokens)."""
        B = tokens.shape[0]
        if next_tokens is None:
            next_tokens = torch.empty((B,), dtype=torch.int32, device=tokens.device)
        _check(lib().axon_decode_step(self._h, B, tokens.data_ptr(),
                                      logits.data_ptr() if logits is not None else None,
                                      next_tokens.data_ptr(), ctypes.c_void_p(_stream(stream))))
        return logits, next_tokens

    def decode_step_noalloc(self, tokens: torch.Tensor, logits: torch.Tensor | None = None,
                            next_tokens: torch.Tensor = None, stream=None):
        """axon_decode_step_noalloc: the decode step with its work buffers in the
        library's fixed per-GPU array (nothing is allocated by the call; the
        caller provides ``next_tokens``, device int32 [batch]).  Returns
        (logits or None, next_tokens)."""
        if next_tokens is None:
            raise ValueError("decode_step_noalloc needs a caller-provided next_tokens buffer")
        _check(lib().axon_decode_step_noalloc(self._h, tokens.shape[0], tokens.data_ptr(),
                                              logits.data_ptr() if logits is not None else None,
                                              next_tokens.data_ptr(), ctypes.c_void_p(_stream(stream))))
        return logits, next_tokens

    def step(self, tokens: torch.Tensor, cu_seqlens: list, slots: list, fresh: list | None = None,
             block_rows: torch.Tensor | None = None, logits: torch.Tensor | None = None,
             next_tokens: torch.Tensor | None = None, want_logits: bool = True, stream=None,
             cu_device: torch.Tensor | None = None):
        """One continuous-batching step (axon_step).  tokens: device int32
        [sum n_i]; cu_seqlens: host list of n+1 ints; slots / fresh: host lists
        of n ints; block_rows: host int32 [n, stride] page rows (paged cache) or
        None; cu_device: optional device int32 buffer (>= n+1 entries) that
        receives cu_seqlens, so that its address stays fixed across calls.
        Returns (logits [n, V] or None, next_tokens [n])."""
        dev = tokens.device
        n = len(slots)
        cu_h = (ctypes.c_int32 * (n + 1))(*[int(c) for c in cu_seqlens])
        if cu_device is not None:
            cu_d = cu_device
            cu_d[:n + 1].copy_(torch.tensor([int(c) for c in cu_seqlens], dtype=torch.int32), non_blocking=True)
        else:
            cu_d = torch.tensor([int(c) for c in cu_seqlens], dtype=torch.int32, device=dev)
        sl_h = (ctypes.c_int32 * n)(*[int(x) for x in slots])
        fr_h = (ctypes.c_int32 * n)(*[int(x) for x in fresh]) if fresh is not None else None
        if logits is None and want_logits:
            logits = torch.empty((n, self.vocab), dtype=torch.float32, device=dev)
        if next_tokens is None:
            next_tokens = torch.empty((n,), dtype=torch.int32, device=dev)
        bt_ptr, stride = None, 0
        if block_rows is not None:
            bt = block_rows.to("cpu", torch.int32).contiguous()
            stride = bt.shape[1]
            bt_ptr = ctypes.cast(bt.data_ptr(), ctypes.POINTER(ctypes.c_int32))
        _check(lib().axon_step(self._h, n, sl_h, fr_h, tokens.data_ptr(), cu_d.data_ptr(), cu_h, bt_ptr, stride,
                               logits.data_ptr() if logits is not None else None, next_tokens.data_ptr(),
                               ctypes.c_void_p(_stream(stream))))
        self._keep = (cu_d, tokens)
        return logits, next_tokens

    def reset_slot(self, slot: int):
        """Evict the sequence of ``slot`` (axon_reset_slot)."""
        _check(lib().axon_reset_slot(self._h, int(slot)))

    def lengths(self) -> list[int]:
        buf = (ctypes.c_int32 * self.max_batch)()
        n = _check(lib().axon_slot_lengths(self._h, buf, self.max_batch))
        return list(buf)[:n]

    def timing(self, enable: bool):
        _check(lib().axon_timing_enable(self._h, int(enable)))

    def timing_records(self):
        """List of (kernel class, (d0, d1, d2), milliseconds)."""
        n = _check(lib().axon_timing_records(self._h, None, None, None, 0))
        cls = (ctypes.c_int32 * max(n, 1))()
        dims = (ctypes.c_int32 * max(3 * n, 1))()
        ms = (ctypes.c_float * max(n, 1))()
        _check(lib().axon_timing_records(self._h, cls, dims, ms, n))
        return [(cls[i], (dims[3 * i], dims[3 * i + 1], dims[3 * i + 2]), ms[i]) for i in range(n)]

    def close(self):
        if getattr(self, "_h", None):
            lib().axon_free(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def init_status(cfg: AxonConfig, weights: dict) -> tuple[int, str]:
    """Call axon_init_model and return (status, message) without raising (for
    validation tests).  A successful handle is freed immediately."""
    arr, keep = make_weights(weights)
    handle = ctypes.c_void_p()
    rc = lib().axon_init_model(ctypes.byref(cfg), arr, len(weights), None, ctypes.byref(handle))
    msg = last_error()
    if rc == AXON_OK:
        lib().axon_free(handle)
    del keep
    return rc, msg
