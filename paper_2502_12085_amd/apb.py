"""Python binding of the APB host-share C ABI (``include/apb.h``).

Argument marshalling only: every step of the path runs in the HIP kernels of
``libapb.so``.  PyTorch supplies device memory and streams.  The names match
the C entry points without the ``apb_`` prefix.  If the library is missing,
every call raises: there is no fallback.
"""
from __future__ import annotations

import ctypes
import os

PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG, "libapb.so")

APB_OK = 0
NOALLOC_SCRATCH_BYTES = 16 << 20  # APB_DECODE_NOALLOC_SCRATCH_BYTES
STATUS_NAMES = {0: "APB_OK", 1: "APB_ERR_NULL_POINTER", 2: "APB_ERR_BAD_SHAPE",
                3: "APB_ERR_UNSUPPORTED", 4: "APB_ERR_MISALIGNED", 5: "APB_ERR_HIP",
                6: "APB_ERR_ALIAS", 7: "APB_ERR_SCRATCH"}
EXPORTED = ("apb_compress_select", "apb_attention_fwd", "apb_validate_problem",
            "apb_attention_flops", "apb_status_string", "apb_last_error", "apb_abi_version",
            "apb_validate_decode", "apb_decode_workspace_size", "apb_decode_attention",
            "apb_decode_attention_noalloc",
            "apb_merge_partials", "apb_validate_scorer", "apb_scorer_workspace_size",
            "apb_retaining_scores", "apb_validate_layer", "apb_layer_workspace_size",
            "apb_layer_flops", "apb_layer_fwd", "apb_validate_cache4", "apb_cache4_write",
            "apb_cache4_read", "apb_validate_decode4", "apb_decode4_workspace_size",
            "apb_decode4_attention")


class ApbError(RuntimeError):
    def __init__(self, status: int, where: str, detail: str = ""):
        self.status = status
        msg = f"{where}: {STATUS_NAMES.get(status, status)}"
        if detail:
            msg += f" ({detail})"
        super().__init__(msg)


class Problem(ctypes.Structure):
    """``apb_problem_t``: one host's share of one attention layer."""

    _fields_ = [("n_hosts", ctypes.c_int32), ("host_idx", ctypes.c_int32),
                ("anchor_len", ctypes.c_int32), ("local_len", ctypes.c_int32),
                ("pass_len", ctypes.c_int32), ("n_q_heads", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32)]

    @classmethod
    def of(cls, p) -> "Problem":
        """From any object with the same field names (e.g. inputs.Problem)."""
        if isinstance(p, cls):
            return p
        return cls(*(int(getattr(p, f)) for f, _ in cls._fields_))


class DecodeProblem(ctypes.Structure):
    """``apb_decode_problem_t``: one host's decoding step (Alg. 3)."""

    _fields_ = [("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("cache_len", ctypes.c_int32),
                ("n_new", ctypes.c_int32), ("append_new", ctypes.c_int32)]

    @classmethod
    def of(cls, p) -> "DecodeProblem":
        if isinstance(p, cls):
            return p
        return cls(*(int(getattr(p, f)) for f, _ in cls._fields_))


class ScorerProblem(ctypes.Structure):
    """``apb_scorer_problem_t``: one host's retaining-head scoring."""

    _fields_ = [("anchor_len", ctypes.c_int32), ("local_len", ctypes.c_int32),
                ("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("hidden", ctypes.c_int32)]


class LayerProblem(ctypes.Structure):
    """``apb_layer_problem_t``: one host's whole layer (Alg. 2)."""

    _fields_ = [("attn", Problem), ("hidden", ctypes.c_int32), ("intermediate", ctypes.c_int32),
                ("scorer_hidden", ctypes.c_int32), ("rms_eps", ctypes.c_float),
                ("rope_theta", ctypes.c_float)]

    @classmethod
    def of(cls, lw) -> "LayerProblem":
        """From an object with ``problem``, ``hidden``, ``intermediate``,
        ``scorer_hidden``, ``eps`` and ``theta`` (e.g. inputs.LayerWorkload)."""
        if isinstance(lw, cls):
            return lw
        return cls(Problem.of(lw.problem), int(lw.hidden), int(lw.intermediate),
                   int(lw.scorer_hidden), float(lw.eps), float(lw.theta))


class LayerWeights(ctypes.Structure):
    """``apb_layer_weights_t``: device pointers of one layer's weights."""

    _fields_ = [(n, ctypes.c_void_p) for n in ("ln1", "w_qkv", "w_o", "ln2", "w_gate", "w_up",
                                               "w_down", "r_w1", "r_b1", "r_w2", "r_b2")]


class Cache4(ctypes.Structure):
    """``apb_cache4_t``: device pointers of a KV cache in 4 bits."""

    _fields_ = [(n, ctypes.c_void_p) for n in ("k_codes", "k_scales", "v_codes", "v_scales")]


class Cache4Problem(ctypes.Structure):
    """``apb_cache4_problem_t``: the rows that a write to, or a read of, a KV
    cache in 4 bits moves."""

    _fields_ = [("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("capacity", ctypes.c_int32), ("first_row", ctypes.c_int32),
                ("n_rows", ctypes.c_int32), ("bf16_rows", ctypes.c_int32),
                ("bf16_first", ctypes.c_int32)]


class Decode4Problem(ctypes.Structure):
    """``apb_decode4_problem_t``: one host's decoding step over a KV cache in
    4 bits."""

    _fields_ = [("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("capacity", ctypes.c_int32),
                ("cache_len", ctypes.c_int32), ("n_new", ctypes.c_int32),
                ("causal", ctypes.c_int32)]


_lib = None


def lib() -> ctypes.CDLL:
    """Load ``libapb.so`` (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2502_12085_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        vp, i32p = ctypes.c_void_p, ctypes.POINTER(Problem)
        L.apb_compress_select.argtypes = [i32p, vp, vp, vp, vp, vp, vp, vp]
        L.apb_compress_select.restype = ctypes.c_int
        L.apb_attention_fwd.argtypes = [i32p, vp, vp, vp, vp, vp, vp, vp, ctypes.c_float, vp]
        L.apb_attention_fwd.restype = ctypes.c_int
        L.apb_validate_problem.argtypes = [i32p]
        L.apb_validate_problem.restype = ctypes.c_int
        L.apb_attention_flops.argtypes = [i32p]
        L.apb_attention_flops.restype = ctypes.c_double
        L.apb_status_string.argtypes = [ctypes.c_int]
        L.apb_status_string.restype = ctypes.c_char_p
        L.apb_last_error.argtypes = []
        L.apb_last_error.restype = ctypes.c_char_p
        L.apb_abi_version.argtypes = []
        L.apb_abi_version.restype = ctypes.c_int
        dp = ctypes.POINTER(DecodeProblem)
        L.apb_validate_decode.argtypes = [dp]
        L.apb_validate_decode.restype = ctypes.c_int
        L.apb_decode_workspace_size.argtypes = [dp, ctypes.POINTER(ctypes.c_uint64)]
        L.apb_decode_workspace_size.restype = ctypes.c_int
        L.apb_decode_attention.argtypes = [dp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_float, vp,
                                           ctypes.c_uint64, vp]
        L.apb_decode_attention.restype = ctypes.c_int
        L.apb_decode_attention_noalloc.argtypes = [dp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_float,
                                                   vp]
        L.apb_decode_attention_noalloc.restype = ctypes.c_int
        L.apb_merge_partials.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32, vp, vp,
                                         vp, vp, vp]
        L.apb_merge_partials.restype = ctypes.c_int
        sp = ctypes.POINTER(ScorerProblem)
        L.apb_validate_scorer.argtypes = [sp]
        L.apb_validate_scorer.restype = ctypes.c_int
        L.apb_scorer_workspace_size.argtypes = [sp, ctypes.POINTER(ctypes.c_uint64)]
        L.apb_scorer_workspace_size.restype = ctypes.c_int
        L.apb_retaining_scores.argtypes = [sp, vp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_uint64,
                                           vp]
        L.apb_retaining_scores.restype = ctypes.c_int
        lp_ = ctypes.POINTER(LayerProblem)
        L.apb_validate_layer.argtypes = [lp_]
        L.apb_validate_layer.restype = ctypes.c_int
        L.apb_layer_workspace_size.argtypes = [lp_, ctypes.POINTER(ctypes.c_uint64)]
        L.apb_layer_workspace_size.restype = ctypes.c_int
        L.apb_layer_flops.argtypes = [lp_]
        L.apb_layer_flops.restype = ctypes.c_double
        L.apb_layer_fwd.argtypes = [lp_, ctypes.POINTER(LayerWeights), vp, vp, vp, vp, vp, vp, vp,
                                    vp, ctypes.c_uint64, vp]
        L.apb_layer_fwd.restype = ctypes.c_int
        cp, c4 = ctypes.POINTER(Cache4Problem), ctypes.POINTER(Cache4)
        L.apb_validate_cache4.argtypes = [cp]
        L.apb_validate_cache4.restype = ctypes.c_int
        L.apb_cache4_write.argtypes = [cp, vp, vp, c4, vp]
        L.apb_cache4_write.restype = ctypes.c_int
        L.apb_cache4_read.argtypes = [cp, c4, vp, vp, vp]
        L.apb_cache4_read.restype = ctypes.c_int
        d4 = ctypes.POINTER(Decode4Problem)
        L.apb_validate_decode4.argtypes = [d4]
        L.apb_validate_decode4.restype = ctypes.c_int
        L.apb_decode4_workspace_size.argtypes = [d4, ctypes.POINTER(ctypes.c_uint64)]
        L.apb_decode4_workspace_size.restype = ctypes.c_int
        L.apb_decode4_attention.argtypes = [d4, vp, c4, vp, vp, ctypes.c_float, vp,
                                            ctypes.c_uint64, vp]
        L.apb_decode4_attention.restype = ctypes.c_int
        _lib = L
    return _lib


# What a call costs the host counts: a small decoding step's kernel takes about
# 6 us.  The current stream's handle comes from the raw lookup
# (0.5 us with the device's index; a torch.cuda.Stream object took 3), and a
# tensor's checks are one expression: 11.7 -> 9.4 us per decode_attention call,
# 7.9 -> 5.6 per merge_partials call.
def _ptr(t, name, dtypes):
    """Device pointer of a contiguous CUDA/HIP tensor, or None."""
    if t is None:
        return None
    if t.is_cuda and t.dtype in dtypes and t.is_contiguous():
        return t.data_ptr()
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype not in dtypes:
        raise ValueError(f"{name} has dtype {t.dtype}, expected one of {dtypes}")
    raise ValueError(f"{name} must be contiguous")


def _stream(stream):
    if stream is None:
        import torch
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if raw is None:
            return torch.cuda.current_stream().cuda_stream
        return raw(torch.cuda.current_device())
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _check(status, where):
    if status != APB_OK:
        detail = lib().apb_status_string(status).decode()
        if status == 5:
            detail += ": " + lib().apb_last_error().decode()
        raise ApbError(status, where, detail)


def _bf16_types():
    import torch
    return (torch.bfloat16, torch.int16, torch.uint16)


def compress_select(problem, scores, k, v, out_idx, out_k, out_v, stream=None):
    """``apb_compress_select``: top-l_p of ``scores`` [n_kv, Lb] (fp32) per KV
    head and gather of K/V rows La+idx into ``out_k``/``out_v`` [n_kv, l_p, d]."""
    import torch
    b = _bf16_types()
    st = lib().apb_compress_select(
        ctypes.byref(Problem.of(problem)), _ptr(scores, "scores", (torch.float32,)),
        _ptr(k, "k", b), _ptr(v, "v", b), _ptr(out_idx, "out_idx", (torch.int32,)),
        _ptr(out_k, "out_k", b), _ptr(out_v, "out_v", b), _stream(stream))
    _check(st, "apb_compress_select")


def attention_fwd(problem, q, k, v, k_pass, v_pass, o, lse=None, softmax_scale=0.0,
                  stream=None):
    """``apb_attention_fwd``: modified-mask attention of one host share."""
    import torch
    b = _bf16_types()
    st = lib().apb_attention_fwd(
        ctypes.byref(Problem.of(problem)), _ptr(q, "q", b), _ptr(k, "k", b), _ptr(v, "v", b),
        _ptr(k_pass, "k_pass", b), _ptr(v_pass, "v_pass", b), _ptr(o, "o", b),
        _ptr(lse, "lse", (torch.float32,)), float(softmax_scale), _stream(stream))
    _check(st, "apb_attention_fwd")


def validate_problem(problem) -> int:
    return lib().apb_validate_problem(ctypes.byref(Problem.of(problem)))


def attention_flops(problem) -> float:
    return lib().apb_attention_flops(ctypes.byref(Problem.of(problem)))


def abi_version() -> int:
    return lib().apb_abi_version()


def validate_decode(problem) -> int:
    return lib().apb_validate_decode(ctypes.byref(DecodeProblem.of(problem)))


def decode_workspace_size(problem) -> int:
    """``apb_decode_workspace_size``: device scratch bytes a decode call needs."""
    n = ctypes.c_uint64(0)
    _check(lib().apb_decode_workspace_size(ctypes.byref(DecodeProblem.of(problem)),
                                           ctypes.byref(n)), "apb_decode_workspace_size")
    return int(n.value)


def decode_attention(problem, q, k_cache, v_cache, k_new, v_new, o_part, lse_part, workspace,
                     softmax_scale=0.0, stream=None):
    """``apb_decode_attention``: one host's stage-2 partial attention (Alg. 3).
    ``workspace`` is a device tensor of at least ``decode_workspace_size``
    bytes (any dtype)."""
    import torch
    b = _bf16_types()
    f = (torch.float32,)
    if workspace is None or not workspace.is_cuda or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous device tensor")
    st = lib().apb_decode_attention(
        ctypes.byref(DecodeProblem.of(problem)), _ptr(q, "q", b), _ptr(k_cache, "k_cache", b),
        _ptr(v_cache, "v_cache", b), _ptr(k_new, "k_new", b), _ptr(v_new, "v_new", b),
        _ptr(o_part, "o_part", f), _ptr(lse_part, "lse_part", f), float(softmax_scale),
        workspace.data_ptr(), workspace.numel() * workspace.element_size(), _stream(stream))
    _check(st, "apb_decode_attention")


def decode_attention_noalloc(problem, q, k_cache, v_cache, k_new, v_new, o_part, lse_part,
                             softmax_scale=0.0, stream=None):
    """``apb_decode_attention_noalloc``: ``decode_attention`` without a
    workspace; the library's own per-GPU scratch holds the split partials
    (``NOALLOC_SCRATCH_BYTES``).  Calls that overlap on one GPU race."""
    import torch
    b = _bf16_types()
    f = (torch.float32,)
    st = lib().apb_decode_attention_noalloc(
        ctypes.byref(DecodeProblem.of(problem)), _ptr(q, "q", b), _ptr(k_cache, "k_cache", b),
        _ptr(v_cache, "v_cache", b), _ptr(k_new, "k_new", b), _ptr(v_new, "v_new", b),
        _ptr(o_part, "o_part", f), _ptr(lse_part, "lse_part", f), float(softmax_scale),
        _stream(stream))
    _check(st, "apb_decode_attention_noalloc")


def merge_partials(o_parts, lse_parts, o, lse=None, stream=None):
    """``apb_merge_partials``: MergeScore (Alg. 3) of ``o_parts`` [P, rows, d]
    (fp32) with ``lse_parts`` [P, rows] into ``o`` [rows, d] (bf16)."""
    import torch
    f = (torch.float32,)
    n_parts, rows, d = o_parts.shape
    st = lib().apb_merge_partials(
        int(n_parts), int(rows), int(d), _ptr(o_parts, "o_parts", f),
        _ptr(lse_parts, "lse_parts", f), _ptr(o, "o", _bf16_types()), _ptr(lse, "lse", f),
        _stream(stream))
    _check(st, "apb_merge_partials")


def validate_scorer(problem) -> int:
    return lib().apb_validate_scorer(ctypes.byref(problem))


def scorer_workspace_size(problem) -> int:
    """``apb_scorer_workspace_size``: device scratch bytes a scorer call needs."""
    n = ctypes.c_uint64(0)
    _check(lib().apb_scorer_workspace_size(ctypes.byref(problem), ctypes.byref(n)),
           "apb_scorer_workspace_size")
    return int(n.value)


def retaining_scores(problem, q, k, v, w1, b1, w2, b2, scores, workspace, stream=None):
    """``apb_retaining_scores``: retaining-head scores [n_kv, Lb] (fp32) of the
    local rows of ``q``/``k``/``v`` with weights ``w1`` (bf16 [hidden, F]),
    ``b1``, ``w2`` [n_kv, hidden], ``b2`` (fp32)."""
    import torch
    b = _bf16_types()
    f = (torch.float32,)
    if workspace is None or not workspace.is_cuda or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous device tensor")
    st = lib().apb_retaining_scores(
        ctypes.byref(problem), _ptr(q, "q", b), _ptr(k, "k", b), _ptr(v, "v", b),
        _ptr(w1, "w1", b), _ptr(b1, "b1", f), _ptr(w2, "w2", f), _ptr(b2, "b2", f),
        _ptr(scores, "scores", f), workspace.data_ptr(),
        workspace.numel() * workspace.element_size(), _stream(stream))
    _check(st, "apb_retaining_scores")


def validate_layer(problem) -> int:
    return lib().apb_validate_layer(ctypes.byref(LayerProblem.of(problem)))


def layer_workspace_size(problem) -> int:
    """``apb_layer_workspace_size``: device scratch bytes a layer call needs."""
    n = ctypes.c_uint64(0)
    _check(lib().apb_layer_workspace_size(ctypes.byref(LayerProblem.of(problem)), ctypes.byref(n)),
           "apb_layer_workspace_size")
    return int(n.value)


def layer_flops(problem) -> float:
    return lib().apb_layer_flops(ctypes.byref(LayerProblem.of(problem)))


def layer_fwd(problem, weights: dict, hidden_in, positions, k_cache, v_cache, pass_k, pass_v,
              hidden_out, workspace, stream=None):
    """``apb_layer_fwd``: one host's whole layer (Alg. 2).  ``weights`` maps the
    ``apb_layer_weights_t`` field names to device tensors (bf16, the
    retaining head's r_b1/r_w2/r_b2 fp32); ``pass_k``/``pass_v`` are the
    rank-major [H, n_kv, l_p, d] passing buffers (slots < host_idx read, slot
    host_idx written)."""
    import torch
    b = _bf16_types()
    f = (torch.float32,)
    w = LayerWeights()
    for name, _ in LayerWeights._fields_:
        setattr(w, name, _ptr(weights[name], name, f if name in ("r_b1", "r_w2", "r_b2") else b))
    if workspace is None or not workspace.is_cuda or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous device tensor")
    st = lib().apb_layer_fwd(
        ctypes.byref(LayerProblem.of(problem)), ctypes.byref(w), _ptr(hidden_in, "hidden_in", b),
        _ptr(positions, "positions", (torch.int32,)), _ptr(k_cache, "k_cache", b),
        _ptr(v_cache, "v_cache", b), _ptr(pass_k, "pass_k", b), _ptr(pass_v, "pass_v", b),
        _ptr(hidden_out, "hidden_out", b), workspace.data_ptr(),
        workspace.numel() * workspace.element_size(), _stream(stream))
    _check(st, "apb_layer_fwd")


# The elements that a call's sizes ask of each tensor are counted here (its shape is
# its own: a flat buffer in the documented order will do): a cache is sized by its
# capacity, not by the rows in use, so a tensor of another size is an easy mistake,
# and one that the C call cannot see.  Nor can it see a tensor
# of another device than the current one, whose stream the call would use.  A call
# on a few rows takes 2 us of the GPU, so what the host does is what it costs: a
# tensor that is as it should be is one expression, and what is wrong is found after.
class _Cuda:
    """Types and lookups, filled in by ``_device``."""

    bf16 = f32 = raw_stream = raw_device = u8 = None


def _device():
    """The current device's index; -2 where there is none (no tensor's device)."""
    if _Cuda.raw_device is not None:
        return _Cuda.raw_device()
    import torch
    _Cuda.bf16, _Cuda.f32, _Cuda.u8 = _bf16_types(), torch.float32, torch.uint8
    if not torch.cuda.is_available():
        return -2
    dev = torch.cuda.current_device()  # initialises the runtime
    _Cuda.raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    _Cuda.raw_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)
    return dev


def _wrong(t, name, types, n, dev, status, where):
    """Raises what is wrong with a tensor of a call, whose sizes have `status`."""
    _check(status, where)  # sizes that are wrong in themselves
    _ptr(t, name, types)
    if t.get_device() != dev:
        raise ValueError(f"{name} is on {t.device}, not on the current device")
    raise ValueError(f"{name} has {t.numel()} elements, expected {n}")


def _rows4(t, name, n, dev, validate, problem, where):
    """Device pointer of a bf16 tensor of n elements, or None."""
    if t is None:
        return None
    if (t.dtype in _Cuda.bf16 and t.numel() == n and t.get_device() == dev
            and t.is_contiguous()):
        return t.data_ptr()
    return _wrong(t, name, _Cuda.bf16, n, dev, validate(problem), where)


def _cache4(cache, dev, validate, problem, where):
    """``apb_cache4_t`` of a mapping of the four tensors (uint8); None for None."""
    if cache is None:
        return None
    rows, d, u8 = problem.n_kv_heads * problem.capacity, problem.head_dim, _Cuda.u8
    codes, scales = rows * (d // 2), rows * (d // 32)
    kc, ks, vc, vs = (cache["k_codes"], cache["k_scales"], cache["v_codes"], cache["v_scales"])
    if (kc is not None and ks is not None and vc is not None and vs is not None
            and kc.dtype is u8 and ks.dtype is u8 and vc.dtype is u8 and vs.dtype is u8
            and kc.numel() == codes and vc.numel() == codes
            and ks.numel() == scales and vs.numel() == scales
            and kc.get_device() == dev and vc.get_device() == dev
            and ks.get_device() == dev and vs.get_device() == dev
            and kc.is_contiguous() and vc.is_contiguous()
            and ks.is_contiguous() and vs.is_contiguous()):
        return Cache4(kc.data_ptr(), ks.data_ptr(), vc.data_ptr(), vs.data_ptr())
    # a call that moves or sees no rows takes None in place of any of them
    idle = 0 == (problem.n_rows if validate is validate_cache4 else problem.cache_len)
    for name, n in (("k_codes", codes), ("k_scales", scales), ("v_codes", codes),
                    ("v_scales", scales)):
        t = cache[name]
        if t is None:
            _check(validate(problem) or (0 if idle else 1), where)
        elif not (t.dtype is u8 and t.numel() == n and t.get_device() == dev
                and t.is_contiguous()):
            _wrong(t, name, (u8,), n, dev, validate(problem), where)
    return Cache4(*(None if t is None else t.data_ptr() for t in (kc, ks, vc, vs)))


def _stream4(stream, dev):
    if stream is None and _Cuda.raw_stream is not None:
        return _Cuda.raw_stream(dev)
    return _stream(stream)


def validate_cache4(problem) -> int:
    return lib().apb_validate_cache4(ctypes.byref(problem))


def cache4_write(problem, k, v, cache: dict, stream=None):
    """``apb_cache4_write``: quantise rows of ``k``/``v`` [n_kv, bf16_rows, d]
    (bf16) into ``cache``, a mapping of ``k_codes``/``v_codes`` [n_kv, capacity,
    d / 2] and ``k_scales``/``v_scales`` [n_kv, capacity, d / 32] (uint8).  Every
    tensor may be None when n_rows is 0, the mapping too."""
    dev, where = _device(), "apb_cache4_write"
    n = problem.n_kv_heads * problem.bf16_rows * problem.head_dim
    st = lib().apb_cache4_write(problem, _rows4(k, "k", n, dev, validate_cache4, problem, where),
                                _rows4(v, "v", n, dev, validate_cache4, problem, where),
                                _cache4(cache, dev, validate_cache4, problem, where),
                                _stream4(stream, dev))
    if st:
        _check(st, where)


def cache4_read(problem, cache: dict, k, v, stream=None):
    """``apb_cache4_read``: the values of cache rows into ``k``/``v`` [n_kv,
    bf16_rows, d] (bf16); ``cache`` as in ``cache4_write``."""
    dev, where = _device(), "apb_cache4_read"
    n = problem.n_kv_heads * problem.bf16_rows * problem.head_dim
    st = lib().apb_cache4_read(problem, _cache4(cache, dev, validate_cache4, problem, where),
                               _rows4(k, "k", n, dev, validate_cache4, problem, where),
                               _rows4(v, "v", n, dev, validate_cache4, problem, where),
                               _stream4(stream, dev))
    if st:
        _check(st, where)


def validate_decode4(problem) -> int:
    return lib().apb_validate_decode4(ctypes.byref(problem))


def decode4_workspace_size(problem) -> int:
    """``apb_decode4_workspace_size``: device scratch bytes a call needs."""
    n = ctypes.c_uint64(0)
    _check(lib().apb_decode4_workspace_size(ctypes.byref(problem), ctypes.byref(n)),
           "apb_decode4_workspace_size")
    return int(n.value)


def decode4_attention(problem, q, cache: dict, o_part, lse_part, workspace, softmax_scale=0.0,
                      stream=None):
    """``apb_decode4_attention``: one host's stage-2 partial attention over a KV
    cache in 4 bits (``cache`` as in ``cache4_write``; it and its tensors may be
    None when cache_len is 0).  ``workspace`` is a device tensor of at least
    ``decode4_workspace_size`` bytes (any dtype)."""
    dev, where = _device(), "apb_decode4_attention"
    if workspace is None or workspace.get_device() != dev or not workspace.is_contiguous():
        _check(validate_decode4(problem), where)
        raise ValueError("workspace must be a contiguous device tensor, on the current device")
    rows, f32 = problem.n_q_heads * problem.n_new, _Cuda.f32
    n = rows * problem.head_dim
    if not (o_part is not None and lse_part is not None
            and o_part.dtype is f32 and lse_part.dtype is f32
            and o_part.numel() == n and lse_part.numel() == rows
            and o_part.get_device() == dev and lse_part.get_device() == dev
            and o_part.is_contiguous() and lse_part.is_contiguous()):
        status = validate_decode4(problem)
        for t, name, size in ((o_part, "o_part", n), (lse_part, "lse_part", rows)):
            if t is None:
                _check(status or 1, where)
            if not (t.dtype is f32 and t.numel() == size and t.get_device() == dev
                    and t.is_contiguous()):
                _wrong(t, name, (f32,), size, dev, status, where)
    st = lib().apb_decode4_attention(
        problem, _rows4(q, "q", n, dev, validate_decode4, problem, where),
        _cache4(cache, dev, validate_decode4, problem, where),
        o_part.data_ptr(), lse_part.data_ptr(), softmax_scale, workspace.data_ptr(),
        workspace.numel() * workspace.element_size(), _stream4(stream, dev))
    if st:
        _check(st, where)
