"""Python binding of libgraft (include/graft.h): argument marshalling only.

Every step of GRAFT's per-round draft-tree construction runs in the HIP
kernels of libgraft.so; this module passes torch tensors' device pointers and
the current HIP stream through ctypes.  If the library is not built, importing
works but creating a Context raises: there is no fallback path.
"""
from __future__ import annotations

import ctypes as C
import os
import struct

import torch

__all__ = ["Context", "QuantRows", "paged_cache", "TreeBuffers", "TdesTrainer", "TdesHyper", "saba_fit", "read_stream", "lib",
           "library_path", "GraftError", "EXPORTED_SYMBOLS"]

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libgraft.so")
_lib = None

EXPORTED_SYMBOLS = (
    "graft_create", "graft_destroy", "graft_set_scorer", "graft_set_saba", "graft_set_history",
    "graft_get_history", "graft_set_fusion",
    "graft_build_tree", "graft_build_tree_static", "graft_accept", "graft_get_device_status",
    "graft_synth_node_targets", "graft_profile_begin", "graft_profile_end", "graft_status_string", "graft_last_error",
    "graft_mask_to_bias", "graft_commit_accepted", "graft_tdes_create", "graft_tdes_destroy",
    "graft_tdes_param_count", "graft_tdes_step", "graft_tdes_device_status", "graft_saba_fit",
    "graft_read_stream", "graft_tree_attention", "graft_tree_attention_workspace",
    "graft_accept_sampled", "graft_accept_sampled_workspace", "graft_cache_write",
    "graft_cache_read", "graft_paged_write", "graft_paged_attention", "graft_paged_attention_workspace",
    "graft_paged_commit",
)

READ_STREAM_SINK_WORDS = 4096
_BF16_BITS = (torch.bfloat16, torch.int16, torch.uint16)   # dtypes that hold bf16 bit patterns


class GraftError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        L = lib()
        super().__init__("%s: %s (%s)" % (where, L.graft_status_string(status).decode(),
                                          L.graft_last_error().decode()))


class Dims(C.Structure):
    _fields_ = [("max_batch", C.c_int32), ("num_pos", C.c_int32), ("vocab", C.c_int32),
                ("top_k", C.c_int32), ("max_nodes", C.c_int32), ("hist_window", C.c_int32)]


class ScorerDesc(C.Structure):
    _fields_ = [("emb", C.c_void_p), ("g_parent", C.c_void_p), ("g_child", C.c_void_p),
                ("depth_emb", C.c_void_p), ("emb_dim", C.c_int32), ("score_dim", C.c_int32),
                ("scale", C.c_float), ("beta", C.c_float), ("center", C.c_int32)]


class SabaDesc(C.Structure):
    _fields_ = [("budgets", C.c_void_p), ("n_budgets", C.c_int32), ("phi", C.c_float * 4),
                ("tau_min", C.c_float), ("c0", C.c_float), ("c1", C.c_float), ("c2", C.c_float)]


class RoundIn(C.Structure):
    _fields_ = [("batch", C.c_int32), ("logits", C.c_void_p), ("root_token", C.c_void_p),
                ("base_pos", C.c_void_p), ("prefix_len", C.c_void_p), ("hist", C.c_void_p),
                ("fixed_budget", C.c_void_p), ("hidden", C.c_void_p), ("hidden_dim", C.c_int32)]


class TreeOut(C.Structure):
    _fields_ = [("budget", C.c_void_p), ("n_nodes", C.c_void_p), ("tokens", C.c_void_p),
                ("parents", C.c_void_p), ("pos_ids", C.c_void_p), ("mask", C.c_void_p),
                ("topk_ids", C.c_void_p), ("topk_logq", C.c_void_p), ("row_lse", C.c_void_p),
                ("row_maxprob", C.c_void_p), ("row_entropy", C.c_void_p),
                ("edge_scores", C.c_void_p), ("node_scores", C.c_void_p),
                ("saba_state", C.c_void_p), ("adj_cos", C.c_void_p)]


class TdesDims(C.Structure):
    _fields_ = [("vocab", C.c_int32), ("emb_dim", C.c_int32), ("score_dim", C.c_int32),
                ("num_pos", C.c_int32), ("top_k", C.c_int32), ("max_groups", C.c_int32),
                ("max_pairs", C.c_int32)]


class TdesBatch(C.Structure):
    _fields_ = [("n_groups", C.c_int32), ("parent", C.c_void_p), ("depth", C.c_void_p),
                ("child", C.c_void_p), ("logq", C.c_void_p), ("z_target", C.c_void_p),
                ("target", C.c_void_p), ("n_pairs", C.c_int32), ("pairs", C.c_void_p)]


class TdesHyper(C.Structure):
    """Loss weights, margin, positive weight and AdamW settings; the defaults
    are the paper's training setup (lambda 1 / 1 / 0.25, lr 2e-3, weight decay
    1e-4) with the usual AdamW betas and eps, margin 1 and w1 = 1."""
    _fields_ = [(n, C.c_float) for n in ("lambda_kl", "lambda_pair", "lambda_bce", "gamma", "w1",
                                         "lr", "weight_decay", "beta1", "beta2", "eps")]

    def __init__(self, lambda_kl=1.0, lambda_pair=1.0, lambda_bce=0.25, gamma=1.0, w1=1.0,
                 lr=2e-3, weight_decay=1e-4, beta1=0.9, beta2=0.999, eps=1e-8):
        super().__init__(lambda_kl, lambda_pair, lambda_bce, gamma, w1, lr, weight_decay, beta1,
                         beta2, eps)


class SabaReplay(C.Structure):
    _fields_ = [("n_rounds", C.c_int32), ("n_budgets", C.c_int32), ("budgets", C.c_void_p),
                ("state", C.c_void_p), ("prefix", C.c_void_p), ("accepted", C.c_void_p),
                ("latency", C.c_void_p), ("tau_min", C.c_float)]


class Targets(C.Structure):
    _fields_ = [("target_root", C.c_void_p), ("target_node", C.c_void_p),
                ("target_depth", C.c_void_p)]


class Rows(C.Structure):
    _fields_ = ([("data", C.c_void_p)]
                + [(n + "_stride", C.c_int64) for n in ("plane", "batch", "row", "head")]
                + [("scale", C.c_void_p)]
                + [("scale_%s_stride" % n, C.c_int64) for n in ("plane", "batch", "row", "head")])


class Attention(C.Structure):
    _fields_ = [("batch", C.c_int32), ("slots", C.c_int32), ("with_root", C.c_int32),
                ("q_heads", C.c_int32), ("kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("dtype", C.c_int32), ("cache_dtype", C.c_int32), ("scale", C.c_float),
                ("q", Rows), ("k", Rows), ("v", Rows), ("n_nodes", C.c_void_p),
                ("mask", C.c_void_p), ("cache_k", Rows), ("cache_v", Rows),
                ("cache_rows", C.c_int32), ("cache_len", C.c_void_p), ("shared_k", Rows),
                ("shared_v", Rows), ("shared_len", C.c_int32), ("out", Rows), ("lse", C.c_void_p),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_int64)]


class TargetLogits(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("root", C.c_void_p), ("root_stride", C.c_int64),
                ("node", C.c_void_p), ("node_batch_stride", C.c_int64),
                ("node_row_stride", C.c_int64), ("node_rows", C.c_int32),
                ("temperature", C.c_void_p), ("uniform", C.c_void_p)]


class CacheMove(C.Structure):
    _fields_ = [("batch", C.c_int32), ("n_planes", C.c_int32), ("heads", C.c_int32),
                ("head_dim", C.c_int32), ("src_dtype", C.c_int32), ("dst_dtype", C.c_int32),
                ("src", Rows), ("dst", Rows), ("src_rows", C.c_int32), ("dst_rows", C.c_int32),
                ("n_rows", C.c_void_p), ("start", C.c_void_p), ("list", C.c_void_p),
                ("list_len", C.c_int32), ("with_root", C.c_int32)]


class PageTable(C.Structure):
    _fields_ = [("table", C.c_void_p), ("table_stride", C.c_int64), ("table_len", C.c_int32),
                ("pages", C.c_int32), ("page_rows", C.c_int32)]


class PagedRows(C.Structure):
    _fields_ = ([(n, C.c_int32) for n in ("batch", "slots", "q_heads", "kv_heads", "head_dim", "rot_dim",
                                          "interleaved", "dtype", "cache_dtype")]
                + [(n, Rows) for n in ("q", "q_out", "k", "v", "cache_k", "cache_v")]
                + [("pages", PageTable), ("n_rows", C.c_void_p), ("start", C.c_void_p),
                   ("positions", C.c_void_p), ("axes", C.c_int32), ("axis", C.c_void_p),
                   ("freq", C.c_void_p)])


class PagedAttention(C.Structure):
    _fields_ = ([(n, C.c_int32) for n in ("batch", "slots", "with_root", "q_heads", "kv_heads", "head_dim",
                                          "dtype", "cache_dtype")]
                + [("scale", C.c_float), ("window", C.c_int32), ("sinks", C.c_int32), ("q", Rows),
                   ("n_nodes", C.c_void_p), ("mask", C.c_void_p), ("cache_k", Rows), ("cache_v", Rows),
                   ("pages", PageTable), ("cache_len", C.c_void_p), ("out", Rows), ("lse", C.c_void_p),
                   ("workspace", C.c_void_p), ("workspace_bytes", C.c_int64)])


class PagedPath(C.Structure):
    _fields_ = [("batch", C.c_int32), ("n_planes", C.c_int32), ("heads", C.c_int32), ("head_dim", C.c_int32),
                ("dtype", C.c_int32), ("rows", Rows), ("pages", PageTable), ("start", C.c_void_p),
                ("acc_len", C.c_void_p), ("acc_nodes", C.c_void_p), ("with_root", C.c_int32)]


# The descriptors that a layer's step passes, packed in one go: at small batches the step waits for the
# host, and structures of structures take 2 to 3 us of a call (of a commit's 10.4 us, an attention's 18.5).
# A graft_rows without scales is its address and three strides, one with them twice that; pads are zeros.
def _packing(form, size):
    """[of 16-bit caches, of quantised ones]; R: a graft_rows without scales, C: the cache's."""
    plain, quant = "q8x3q40x", "q8x4q8x3q"
    packings = [struct.Struct("@" + form.replace("R", plain).replace("C", c)) for c in (plain, quant)]
    assert all(p.size == C.sizeof(size) for p in packings)
    return packings


_PACK_ROWS = _packing("9iRRRRCCqqiii4xqqqiqq", PagedRows)
_PACK_ATTENTION = _packing("8ifiiRqqCCqqiii4xqRqqq", PagedAttention)
_PACK_PATH = [struct.Struct("@5i%sqqiii4xqqqi4x" % c) for c in ("5q40x", "10q")]   # with planes
_NO_ROWS = (0,) * 8


def library_path() -> str:
    return _LIB_PATH


def lib():
    """The loaded libgraft.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError("libgraft.so is not built (python -m paper_2608_20375_amd.build); "
                               "this package has no non-HIP path")
        L = C.CDLL(_LIB_PATH)
        vp, i32 = C.c_void_p, C.c_int32
        L.graft_create.argtypes = [C.POINTER(Dims), C.POINTER(vp)]
        L.graft_destroy.argtypes = [vp]
        L.graft_destroy.restype = None
        L.graft_set_scorer.argtypes = [vp, C.POINTER(ScorerDesc), vp]
        L.graft_set_saba.argtypes = [vp, C.POINTER(SabaDesc)]
        L.graft_set_history.argtypes = [vp, i32, vp, vp]
        L.graft_get_history.argtypes = [vp, i32, vp, vp, vp]
        L.graft_set_fusion.argtypes = [vp, i32, C.POINTER(C.c_int32)]
        L.graft_build_tree.argtypes = [vp, C.POINTER(RoundIn), C.POINTER(TreeOut), vp]
        L.graft_build_tree_static.argtypes = [vp, C.POINTER(RoundIn), C.POINTER(TreeOut), vp]
        L.graft_accept.argtypes = [vp, i32, vp, vp, vp, C.POINTER(Targets), vp, vp, vp, i32, vp]
        L.graft_get_device_status.argtypes = [vp, vp]
        L.graft_synth_node_targets.argtypes = [vp, i32, C.c_uint64, vp, vp, vp, vp, vp, vp, vp, vp]
        i64 = C.c_int64
        L.graft_mask_to_bias.argtypes = [vp, i32, vp, vp, vp, i32, i64, i64, vp]
        L.graft_commit_accepted.argtypes = [vp, i32, vp, vp, vp, vp, i64, i32, i64, i64, i64,
                                            i64, i64, i64, vp]
        L.graft_profile_begin.argtypes = [vp, i32]
        L.graft_profile_end.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(C.c_int32)]
        L.graft_tdes_create.argtypes = [C.POINTER(TdesDims), C.POINTER(vp)]
        L.graft_tdes_destroy.argtypes = [vp]
        L.graft_tdes_destroy.restype = None
        L.graft_tdes_param_count.argtypes = [C.POINTER(TdesDims)]
        L.graft_tdes_param_count.restype = C.c_int64
        L.graft_tdes_step.argtypes = [vp, vp, C.POINTER(TdesBatch), C.POINTER(TdesHyper), i32, vp,
                                      vp, vp, vp, vp, vp]
        L.graft_tdes_device_status.argtypes = [vp, vp]
        L.graft_saba_fit.argtypes = [C.POINTER(SabaReplay), C.POINTER(C.c_float), i32,
                                     C.POINTER(C.c_float), C.POINTER(C.c_float),
                                     C.POINTER(C.c_double), vp]
        L.graft_read_stream.argtypes = [vp, C.c_int64, vp, vp]
        L.graft_tree_attention_workspace.argtypes = [vp, C.POINTER(Attention), C.POINTER(i64)]
        L.graft_tree_attention.argtypes = [vp, C.POINTER(Attention), vp]
        L.graft_accept_sampled_workspace.argtypes = [vp, i32, C.POINTER(i64)]
        L.graft_accept_sampled.argtypes = [vp, i32, vp, vp, vp, C.POINTER(TargetLogits), vp, vp,
                                           vp, vp, i32, vp, i64, vp]
        L.graft_cache_write.argtypes = [vp, C.POINTER(CacheMove), vp]
        L.graft_cache_read.argtypes = [vp, C.POINTER(CacheMove), vp]
        L.graft_paged_write.argtypes = [vp, vp, vp]                 # packed descriptors
        L.graft_paged_attention_workspace.argtypes = [vp, vp, C.POINTER(i64)]
        L.graft_paged_attention.argtypes = [vp, vp, vp]
        L.graft_paged_commit.argtypes = [vp, vp, vp]
        L.graft_status_string.argtypes = [C.c_int]
        L.graft_status_string.restype = C.c_char_p
        L.graft_last_error.argtypes = []
        L.graft_last_error.restype = C.c_char_p
        for n in ("graft_create", "graft_set_scorer", "graft_set_saba", "graft_set_history",
                  "graft_get_history", "graft_set_fusion",
                  "graft_build_tree", "graft_build_tree_static", "graft_accept",
                  "graft_get_device_status",
                  "graft_synth_node_targets", "graft_profile_begin", "graft_profile_end",
                  "graft_mask_to_bias", "graft_commit_accepted", "graft_tdes_create",
                  "graft_tdes_step", "graft_tdes_device_status", "graft_saba_fit",
                  "graft_read_stream", "graft_tree_attention", "graft_tree_attention_workspace",
                  "graft_accept_sampled", "graft_accept_sampled_workspace", "graft_cache_write",
                  "graft_cache_read", "graft_paged_write", "graft_paged_attention",
                  "graft_paged_attention_workspace", "graft_paged_commit"):
            getattr(L, n).restype = C.c_int
        _lib = L
    return _lib


def _ptr(t, dtype=None, name="tensor"):
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.device.type != "cuda":
        raise TypeError("%s must be a CUDA (HIP) tensor" % name)
    if dtype is not None and t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    return t.data_ptr()


def _need(t, name, *dims):
    """Raises ValueError unless tensor t (when given) has one extent per entry of
    dims: an int is the exact extent, a 1-tuple (n,) the least one.  Every
    kernel indexes its buffers by the context's sizes and the call's batch, so
    a buffer that is too small would be read or written out of bounds."""
    if t is None:
        return
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch tensor" % name)
    ok = t.dim() == len(dims) and all(
        (s >= d[0]) if isinstance(d, tuple) else (s == d) for s, d in zip(t.shape, dims))
    if not ok:
        want = ", ".join((">=%d" % d[0]) if isinstance(d, tuple) else str(d) for d in dims)
        raise ValueError("%s must be [%s], got %s" % (name, want, list(t.shape)))


def _plain(t, dtype, shape):
    """Device pointer of a tensor that is exactly what a call takes: on the GPU,
    contiguous, of this dtype and shape; None for None.  Anything else gives -1,
    and the caller goes through _need and _ptr, which accept what else the call
    allows or raise.  A call passes a dozen tensors, and at small batches the
    round waits for the host: this check takes a third of their time."""
    if t is None:
        return None
    if (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is dtype and t.shape == shape
            and t.is_contiguous()):
        return t.data_ptr()
    return -1


_INT32_MAX = 2 ** 31 - 1


def _fits(n, name):
    """n, which the library takes as a 32-bit number: ctypes would drop the bits above."""
    if n > _INT32_MAX:
        raise ValueError("%s has an extent of %d, past 2^31 - 1" % (name, n))
    return n


def _batch_of(t, name):
    if not isinstance(t, torch.Tensor) or t.dim() < 1:
        raise ValueError("%s must be a tensor whose first extent is the batch" % name)
    n = t.shape[0]
    return n if n <= _INT32_MAX else _fits(n, name)


def _stream():
    return torch.cuda.current_stream().cuda_stream


# The current stream's handle without the Stream object around it, where this
# torch offers it (1.3 us a call less).
if hasattr(torch._C, "_cuda_getCurrentRawStream"):
    def _stream():  # noqa: F811
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _check(status: int, where: str):
    if status != 0:
        raise GraftError(status, where)


_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


class QuantRows:
    """Quantised key/value rows: codes [..., rows, heads, head_dim] (e4m3: uint8 or
    float8_e4m3fn) and scales [..., rows, heads] (uint8, s stands for 2^(s - 127)),
    the numbers being code * 2^(s - 127); s from 9 to 247 as cache_write makes it.
    Indexing takes views of both."""

    __slots__ = ("codes", "scales")

    def __init__(self, codes, scales):
        for name, t in (("codes", codes), ("scales", scales)):
            if not isinstance(t, torch.Tensor):
                raise TypeError("%s must be a torch tensor" % name)
        if codes.dtype not in (torch.uint8, torch.float8_e4m3fn) or scales.dtype != torch.uint8:
            raise TypeError("codes must be uint8 or float8_e4m3fn and scales uint8")
        if codes.dim() < 3 or codes.shape[:-1] != scales.shape:
            raise ValueError("scales must be codes' shape without its last extent, got %s and %s"
                             % (list(codes.shape), list(scales.shape)))
        if codes.device != scales.device:
            raise ValueError("codes and scales must be on one device")
        self.codes, self.scales = codes, scales

    @classmethod
    def empty(cls, *shape, device=None):
        """Unwritten rows of shape [..., rows, heads, head_dim]."""
        dev = device or torch.device("cuda", torch.cuda.current_device())
        return cls(torch.empty(shape, dtype=torch.uint8, device=dev),
                   torch.empty(shape[:-1], dtype=torch.uint8, device=dev))

    @property
    def shape(self):
        return self.codes.shape

    @property
    def device(self):
        return self.codes.device

    def __getitem__(self, index):
        """A view by leading indices: codes[index], scales[index]."""
        return QuantRows(self.codes[index], self.scales[index])


def paged_cache(pages, page_rows, heads, dim, dtype=torch.bfloat16, planes=None, device=None):
    """An unwritten pool of pages [pages, page_rows, heads, dim] (planes given: [planes, ...], layers x
    {key, value}, say) whose memory holds a head's rows of a page side by side, the order
    that the attention reads fastest.  dtype: bfloat16, float16, or float8_e4m3fn for
    QuantRows."""
    dev = device or torch.device("cuda", torch.cuda.current_device())
    lead = () if planes is None else (planes,)
    if dtype == torch.float8_e4m3fn:
        codes = torch.empty(*lead, pages, heads, page_rows, dim, dtype=torch.uint8, device=dev)
        scales = torch.empty(*lead, pages, heads, page_rows, dtype=torch.uint8, device=dev)
        return QuantRows(codes.transpose(-2, -3), scales.transpose(-1, -2))
    if dtype not in (torch.bfloat16, torch.float16):
        raise TypeError("dtype must be bfloat16, float16 or float8_e4m3fn")
    return torch.empty(*lead, pages, heads, page_rows, dim, dtype=dtype, device=dev).transpose(-2, -3)


def _rows(t, n, name):
    """graft_rows of a tensor or QuantRows: n extents, the last of (plane, batch, row, head),
    and head_dim.  Strides of extents with one entry are 0."""
    quant = isinstance(t, QuantRows)
    data = t.codes if quant else t
    e, s = data.shape, data.stride()
    if s[n] != 1 and e[n] > 1:
        raise ValueError("%s must have unit stride along its last dimension" % name)
    if n == 3 and not quant:
        return Rows(data.data_ptr(), 0, s[0] if e[0] > 1 else 0, s[1] if e[1] > 1 else 0,
                    s[2] if e[2] > 1 else 0)
    lead = (0,) * (4 - n)
    at = (data.data_ptr(), *lead, *[s[i] if e[i] > 1 else 0 for i in range(n)])
    if not quant:
        return Rows(*at)
    s = t.scales.stride()
    return Rows(*at, t.scales.data_ptr(), *lead, *[s[i] if e[i] > 1 else 0 for i in range(n)])


def _row_at(t, batch, slots, heads, dim, name):
    """Address and strides of a block's rows; strides of extents with one entry are 0."""
    a, b, c, d = t.stride()
    if d != 1 and dim > 1:
        raise ValueError("%s must have unit stride along its last dimension" % name)
    return t.data_ptr(), a if batch > 1 else 0, b if slots > 1 else 0, c if heads > 1 else 0


def _at(t, dtype, shape, dev):
    """Address of a tensor that is exactly what a call takes, 0 for None, -1 for anything else."""
    if t is None:
        return 0
    if (isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape and t.get_device() == dev
            and t.is_contiguous()):
        return t.data_ptr()
    return -1


def _apart(t, name):
    """Raises unless every number of a tensor or QuantRows that is written has a place of its own:
    in the order of their size, each stride passes what the smaller ones span."""
    for x in (t.codes, t.scales) if isinstance(t, QuantRows) else (t,):
        span = 1
        for stride, n in sorted((a, b) for a, b in zip(x.stride(), x.shape) if b > 1):
            if stride < span:
                raise ValueError("%s is written and must not overlap itself (strides %s of %s)"
                                 % (name, list(x.stride()), list(x.shape)))
            span += stride * (n - 1)


class TreeBuffers:
    """Preallocated outputs of one build_tree call (torch tensors on the device)."""

    def __init__(self, ctx: "Context", batch: int, mask=True, topk=True, stats=True, edges=False,
                 node_scores=True, saba_state=True, adj_cos=False, device=None):
        d = ctx.dims
        dev = device or torch.device("cuda", torch.cuda.current_device())
        L, K, N = d.num_pos, d.top_k, d.max_nodes
        W = (N + 63) // 64
        i32 = dict(dtype=torch.int32, device=dev)
        f32 = dict(dtype=torch.float32, device=dev)
        self.batch = batch
        self.sizes = (L, K, N)
        self.budget = torch.empty(batch, **i32)
        self.n_nodes = torch.empty(batch, **i32)
        self.tokens = torch.empty(batch, N, **i32)
        self.parents = torch.empty(batch, N, **i32)
        self.pos_ids = torch.empty(batch, N, **i32)
        # uint64 words of the ancestor bitset, held as int64 (same bits)
        self.mask = torch.empty(batch, N, W, dtype=torch.int64, device=dev) if mask else None
        self.topk_ids = torch.empty(batch, L, K, **i32) if topk else None
        self.topk_logq = torch.empty(batch, L, K, **f32) if topk else None
        self.row_lse = torch.empty(batch, L, **f32) if stats else None
        self.row_maxprob = torch.empty(batch, L, **f32) if stats else None
        self.row_entropy = torch.empty(batch, L, **f32) if stats else None
        self.edge_scores = torch.empty(batch, L, K, K, **f32) if edges else None
        self.node_scores = (torch.empty(batch, N, dtype=torch.float64, device=dev)
                            if node_scores else None)
        self.saba_state = torch.empty(batch, 4, **f32) if saba_state else None
        # cosines of adjacent hidden states (written only when build_tree gets them)
        self.adj_cos = torch.zeros(batch, max(L - 1, 1), **f32) if adj_cos else None
        t = TreeOut()
        for name, _ in TreeOut._fields_:
            setattr(t, name, _ptr(getattr(self, name), name=name))
        self._struct = t

    def as_dict(self) -> dict:
        return {n: getattr(self, n) for n, _ in TreeOut._fields_ if getattr(self, n) is not None}


class Context:
    """A graft_ctx: sizes fixed at creation, workspace owned by the library."""

    def __init__(self, max_batch: int, num_pos: int, vocab: int, top_k: int, max_nodes: int,
                 hist_window: int = 4):
        L = lib()
        self.dims = Dims(max_batch, num_pos, vocab, top_k, max_nodes, hist_window)
        h = C.c_void_p()
        _check(L.graft_create(C.byref(self.dims), C.byref(h)), "graft_create")
        self._h = h
        self._keep = []
        self._device = torch.cuda.current_device()

    def close(self):
        if getattr(self, "_h", None):
            lib().graft_destroy(self._h)
            self._h = None

    def __del__(self):  # pragma: no cover
        try:
            self.close()
        except Exception:
            pass

    def set_scorer(self, emb, g_parent, g_child, depth_emb=None, scale=1.0, beta=1.0, center=0):
        dm = self.dims
        _need(emb, "emb", dm.vocab, (1,))
        E = int(emb.shape[1])
        _need(g_parent, "g_parent", E, (1,))
        m = int(g_parent.shape[1])
        _need(g_child, "g_child", E, m)
        _need(depth_emb, "depth_emb", dm.num_pos, m)
        d = ScorerDesc(_ptr(emb, torch.float32, "emb"), _ptr(g_parent, torch.float32, "g_parent"),
                       _ptr(g_child, torch.float32, "g_child"),
                       _ptr(depth_emb, torch.float32, "depth_emb"), emb.shape[1],
                       g_parent.shape[1], float(scale), float(beta), int(center))
        self._keep = [emb, g_parent, g_child, depth_emb]
        _check(lib().graft_set_scorer(self._h, C.byref(d), _stream()), "graft_set_scorer")

    def set_saba(self, budgets, phi, tau_min=1.0, c0=1.0, c1=0.0, c2=0.0):
        arr = (C.c_int32 * len(budgets))(*[int(b) for b in budgets])
        d = SabaDesc(C.cast(arr, C.c_void_p), len(budgets), (C.c_float * 4)(*map(float, phi)),
                     float(tau_min), float(c0), float(c1), float(c2))
        _check(lib().graft_set_saba(self._h, C.byref(d)), "graft_set_saba")

    def set_fusion(self, enable=True):
        """Lets the selection kernel compute the edge scores and the budget
        itself when the rows fit its stage (graft_set_fusion); returns True
        when that path is taken for this context."""
        active = C.c_int32(0)
        _check(lib().graft_set_fusion(self._h, 1 if enable else 0, C.byref(active)),
               "graft_set_fusion")
        return bool(active.value)

    def set_history(self, init):
        _need(init, "init", (1,), self.dims.hist_window)
        _check(lib().graft_set_history(self._h, init.shape[0], _ptr(init, torch.int32, "init"),
                                       _stream()), "graft_set_history")

    def get_history(self, batch: int):
        """(ring [batch, hist_window], pos [batch]) int32 copies of the device
        acceptance-history ring."""
        dev = torch.device("cuda", torch.cuda.current_device())
        ring = torch.empty(batch, self.dims.hist_window, dtype=torch.int32, device=dev)
        pos = torch.empty(batch, dtype=torch.int32, device=dev)
        _check(lib().graft_get_history(self._h, int(batch), _ptr(ring, torch.int32, "ring"),
                                       _ptr(pos, torch.int32, "pos"), _stream()),
               "graft_get_history")
        return ring, pos

    def build_tree(self, logits, root_token, base_pos, prefix_len=None, hist=None,
                   fixed_budget=None, hidden=None, out: TreeBuffers | None = None,
                   static_scratch=False, **want) -> TreeBuffers:
        """hidden: optional [batch, L, H] bf16 bit patterns of the drafter's hidden
        states; with them the SABA state uses the degeneration signal.
        static_scratch: call graft_build_tree_static (no device allocation in the
        library; pass preallocated `out` to allocate nothing here either)."""
        r = self._round_plain(logits, root_token, base_pos, prefix_len, hist, fixed_budget, hidden,
                              out)
        if r is None:
            r, out = self._round_checked(logits, root_token, base_pos, prefix_len, hist,
                                         fixed_budget, hidden, out, want)
        L = lib()
        if static_scratch:
            _check(L.graft_build_tree_static(self._h, C.byref(r), C.byref(out._struct), _stream()),
                   "graft_build_tree_static")
        else:
            _check(L.graft_build_tree(self._h, C.byref(r), C.byref(out._struct), _stream()),
                   "graft_build_tree")
        return out

    def _round_plain(self, logits, root_token, base_pos, prefix_len, hist, fixed_budget, hidden,
                     out):
        """The round's inputs when every tensor is plain and out fits; else None."""
        dm = self.dims
        L, V = dm.num_pos, dm.vocab
        if (out is None or out.sizes != (L, dm.top_k, dm.max_nodes) or not isinstance(logits, torch.Tensor)
                or logits.dim() != 3 or root_token is None or base_pos is None):
            return None
        shape = logits.shape
        batch = shape[0]
        if out.batch < batch or shape[1] != L or shape[2] != V:
            return None
        one = (batch,)
        i32 = torch.int32
        H = 0
        p_hid = None
        if hidden is not None:
            if not isinstance(hidden, torch.Tensor) or hidden.dim() != 3 or hidden.shape[2] < 1:
                return None
            H = hidden.shape[2]
            p_hid = _plain(hidden, hidden.dtype if hidden.dtype in _BF16_BITS else None,
                           (batch, L, H))
        p = (_plain(logits, logits.dtype if logits.dtype in _BF16_BITS else None, shape),
             _plain(root_token, i32, one), _plain(base_pos, i32, one), _plain(prefix_len, i32, one),
             _plain(hist, torch.float32, one), _plain(fixed_budget, i32, one), p_hid)
        if -1 in p:
            return None
        return RoundIn(batch, *p, H)

    def _round_checked(self, logits, root_token, base_pos, prefix_len, hist, fixed_budget, hidden,
                       out, want):
        dm = self.dims
        batch = _batch_of(logits, "logits")
        _need(logits, "logits", batch, dm.num_pos, dm.vocab)
        for name, t in (("root_token", root_token), ("base_pos", base_pos),
                        ("prefix_len", prefix_len), ("hist", hist), ("fixed_budget", fixed_budget)):
            _need(t, name, batch)
        if root_token is None or base_pos is None:
            raise ValueError("root_token and base_pos are required")
        _need(hidden, "hidden", batch, dm.num_pos, (1,))
        if out is None:
            out = TreeBuffers(self, batch, **want)
        elif out.batch < batch or out.sizes != (dm.num_pos, dm.top_k, dm.max_nodes):
            raise ValueError("out holds %d sequences of sizes (L, K, max_nodes) = %s; this call "
                             "needs %d of %s" % (out.batch, out.sizes, batch,
                                                 (dm.num_pos, dm.top_k, dm.max_nodes)))
        if logits.dtype not in (torch.bfloat16, torch.int16, torch.uint16):
            raise TypeError("logits must hold bf16 bit patterns")
        if hidden is not None and hidden.dtype not in (torch.bfloat16, torch.int16, torch.uint16):
            raise TypeError("hidden must hold bf16 bit patterns")
        r = RoundIn(batch, _ptr(logits, None, "logits"), _ptr(root_token, torch.int32, "root_token"),
                    _ptr(base_pos, torch.int32, "base_pos"),
                    _ptr(prefix_len, torch.int32, "prefix_len"), _ptr(hist, torch.float32, "hist"),
                    _ptr(fixed_budget, torch.int32, "fixed_budget"), _ptr(hidden, None, "hidden"),
                    0 if hidden is None else int(hidden.shape[-1]))
        return r, out

    def accept(self, n_nodes, tokens, parents, target_root=None, target_node=None,
               target_depth=None, update_history=False, acc_len=None, acc_nodes=None, bonus=None):
        p = None
        if (acc_len is not None and acc_nodes is not None and bonus is not None
                and isinstance(n_nodes, torch.Tensor) and n_nodes.dim() == 1
                and tokens is not None and parents is not None):
            L, N = self.dims.num_pos, self.dims.max_nodes
            batch = n_nodes.shape[0]
            i32 = torch.int32
            one, row = (batch,), (batch, N)
            p = (_plain(target_root, i32, one), _plain(target_node, i32, row),
                 _plain(target_depth, i32, (batch, L + 1)), _plain(n_nodes, i32, one),
                 _plain(tokens, i32, row), _plain(parents, i32, row), _plain(acc_len, i32, one),
                 _plain(acc_nodes, i32, (batch, L)), _plain(bonus, i32, one))
        if p is None or -1 in p:
            batch, p, acc_len, acc_nodes, bonus = self._accept_checked(
                n_nodes, tokens, parents, target_root, target_node, target_depth, acc_len,
                acc_nodes, bonus)
        t = Targets(p[0], p[1], p[2])
        _check(lib().graft_accept(self._h, batch, p[3], p[4], p[5], C.byref(t), p[6], p[7], p[8],
                                  1 if update_history else 0, _stream()), "graft_accept")
        return acc_len, acc_nodes, bonus

    def _accept_checked(self, n_nodes, tokens, parents, target_root, target_node, target_depth,
                        acc_len, acc_nodes, bonus):
        dm = self.dims
        batch = _batch_of(n_nodes, "n_nodes")
        _need(n_nodes, "n_nodes", batch)
        _need(tokens, "tokens", (batch,), dm.max_nodes)
        _need(parents, "parents", (batch,), dm.max_nodes)
        _need(target_root, "target_root", (batch,))
        _need(target_node, "target_node", (batch,), dm.max_nodes)
        _need(target_depth, "target_depth", (batch,), dm.num_pos + 1)
        _need(acc_len, "acc_len", (batch,))
        _need(acc_nodes, "acc_nodes", (batch,), dm.num_pos)
        _need(bonus, "bonus", (batch,))
        dev = n_nodes.device
        acc_len = torch.empty(batch, dtype=torch.int32, device=dev) if acc_len is None else acc_len
        acc_nodes = (torch.empty(batch, self.dims.num_pos, dtype=torch.int32, device=dev)
                     if acc_nodes is None else acc_nodes)
        bonus = torch.empty(batch, dtype=torch.int32, device=dev) if bonus is None else bonus
        p = (_ptr(target_root, torch.int32, "target_root"),
             _ptr(target_node, torch.int32, "target_node"),
             _ptr(target_depth, torch.int32, "target_depth"),
             _ptr(n_nodes, torch.int32, "n_nodes"), _ptr(tokens, torch.int32, "tokens"),
             _ptr(parents, torch.int32, "parents"), _ptr(acc_len, torch.int32, "acc_len"),
             _ptr(acc_nodes, torch.int32, "acc_nodes"), _ptr(bonus, torch.int32, "bonus"))
        return batch, p, acc_len, acc_nodes, bonus

    def synth_node_targets(self, seed, root_token, n_nodes, tokens, parents, topk_ids,
                           target_root=None, target_node=None):
        dm = self.dims
        batch = _batch_of(n_nodes, "n_nodes")
        _need(n_nodes, "n_nodes", batch)
        _need(root_token, "root_token", (batch,))
        _need(tokens, "tokens", (batch,), dm.max_nodes)
        _need(parents, "parents", (batch,), dm.max_nodes)
        _need(topk_ids, "topk_ids", (batch,), dm.num_pos, dm.top_k)
        _need(target_root, "target_root", (batch,))
        _need(target_node, "target_node", (batch,), dm.max_nodes)
        dev = n_nodes.device
        if target_root is None:
            target_root = torch.empty(batch, dtype=torch.int32, device=dev)
        if target_node is None:
            target_node = torch.empty(batch, self.dims.max_nodes, dtype=torch.int32, device=dev)
        _check(lib().graft_synth_node_targets(
            self._h, batch, C.c_uint64(int(seed) & ((1 << 64) - 1)),
            _ptr(root_token, torch.int32, "root_token"), _ptr(n_nodes, torch.int32, "n_nodes"),
            _ptr(tokens, torch.int32, "tokens"), _ptr(parents, torch.int32, "parents"),
            _ptr(topk_ids, torch.int32, "topk_ids"), _ptr(target_root, torch.int32, "target_root"),
            _ptr(target_node, torch.int32, "target_node"), _stream()), "graft_synth_node_targets")
        return target_root, target_node

    def mask_to_bias(self, n_nodes, mask, bias=None, dtype=torch.bfloat16):
        """Additive attention bias of the draft block (0 / -inf) from the ancestor
        masks.  bias: [batch, max_nodes, >= max_nodes] tensor or strided view with
        unit stride along the last dimension (e.g. the tree columns of a wider
        bias); allocated as [batch, max_nodes, max_nodes] when None."""
        batch = _batch_of(n_nodes, "n_nodes")
        N = self.dims.max_nodes
        p_n = _plain(n_nodes, torch.int32, (batch,))
        p_mask = _plain(mask, torch.int64, (batch, N, (N + 63) // 64))
        if p_n in (None, -1) or p_mask in (None, -1):
            _need(n_nodes, "n_nodes", batch)
            _need(mask, "mask", (batch,), N, (N + 63) // 64)
        if bias is None:
            bias = torch.empty(batch, N, N, dtype=dtype, device=n_nodes.device)
        if bias.dtype not in (torch.float32, torch.bfloat16):
            raise TypeError("bias must be float32 or bfloat16")
        shape = bias.shape
        if len(shape) != 3 or shape[0] < batch or shape[1] < N or shape[2] < N:
            raise ValueError("bias must be at least [batch, max_nodes, max_nodes]")
        step = bias.stride()
        if step[2] != 1:
            raise ValueError("bias must have unit stride along its last dimension")
        if p_n in (None, -1) or p_mask in (None, -1):
            p_n = _ptr(n_nodes, torch.int32, "n_nodes")
            p_mask = _ptr(mask, torch.int64, "mask")
        _check(lib().graft_mask_to_bias(self._h, batch, p_n, p_mask, bias.data_ptr(),
                                        1 if bias.dtype == torch.bfloat16 else 0, step[1], step[0],
                                        _stream()), "graft_mask_to_bias")
        return bias

    def commit_accepted(self, acc_len, acc_nodes, src, dst=None):
        """Moves the accepted nodes' rows to rows 0..acc_len-1: src and dst are
        [planes, batch, rows, width] tensors (any dtype, unit stride along width);
        dst defaults to src (compaction in place)."""
        dst = src if dst is None else dst
        batch = _batch_of(acc_len, "acc_len")
        dm = self.dims
        L, N = dm.num_pos, dm.max_nodes
        p_len = _plain(acc_len, torch.int32, (batch,))
        p_nodes = _plain(acc_nodes, torch.int32, (batch, L))
        if p_len in (None, -1) or p_nodes in (None, -1):
            _need(acc_len, "acc_len", batch)
            _need(acc_nodes, "acc_nodes", (batch,), L)
        # node indices reach max_nodes - 1 in src; at most L rows are written in dst
        for name, t, rows in (("src", src, N), ("dst", dst, L)):
            if not (isinstance(t, torch.Tensor) and t.dim() == 4 and min(t.shape) >= 1
                    and t.shape[1] >= batch and t.shape[2] >= rows):
                _need(t, name, (1,), (batch,), (rows,), (1,))
        for name, t in (("src", src), ("dst", dst)):
            if not t.is_cuda:
                raise TypeError("%s must be a CUDA (HIP) tensor [planes, batch, rows, width]" % name)
            if t.stride(3) != 1:
                raise ValueError("%s must have unit stride along its last dimension" % name)
        planes, _, _, width = src.shape
        ss, ds = src.stride(), dst.stride()
        if src.dtype != dst.dtype or planes != dst.shape[0] or width != dst.shape[3]:
            raise ValueError("src and dst must agree in dtype, planes and width")
        if p_len in (None, -1) or p_nodes in (None, -1):
            p_len = _ptr(acc_len, torch.int32, "acc_len")
            p_nodes = _ptr(acc_nodes, torch.int32, "acc_nodes")
        es = src.element_size()
        _check(lib().graft_commit_accepted(
            self._h, batch, p_len, p_nodes, src.data_ptr(), dst.data_ptr(), width * es, planes,
            ss[0] * es, ss[1] * es, ss[2] * es, ds[0] * es, ds[1] * es, ds[2] * es, _stream()),
            "graft_commit_accepted")
        return dst

    def _here(self, **tensors):
        """Raises unless every tensor given is on the context's device and that is the
        current one."""
        for name, t in tensors.items():
            if t is None:
                continue
            if not isinstance(t, (torch.Tensor, QuantRows)) or t.device.type != "cuda":
                raise TypeError("%s must be a CUDA (HIP) tensor" % name)
            if t.device.index != self._device:
                raise ValueError("%s is on device %s, the context on device %d"
                                 % (name, t.device.index, self._device))
        if torch.cuda.current_device() != self._device:
            raise ValueError("the context's device %d is not the current one" % self._device)

    def _args(self, others, *args):
        """Device pointers of contiguous tensors, after all extents, devices and types have
        been checked: args are (name, tensor, type, extents as _need's, shape), a tensor of
        that very shape being right without a second look; others: (name, tensor or
        QuantRows) for which only the device is checked.  None stays None."""
        dev = self._device
        out = []
        for name, t, dtype, dims, shape in args:
            if t is None:
                out.append(None)
            elif (isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape
                  and t.get_device() == dev and t.is_contiguous()):
                out.append(t.data_ptr())
            else:
                break
        else:
            for _, t in others:
                if t is not None and (t.codes if isinstance(t, QuantRows) else t).get_device() != dev:
                    break
            else:
                self._here()
                return out
        for name, t, dtype, dims, shape in args:
            _need(t, name, *dims)
        self._here(**dict(others), **{a[0]: a[1] for a in args})
        return [_ptr(t, dtype, name) for name, t, dtype, dims, shape in args]

    def _kv_pair(self, pair, name, lead, heads, dim, dtype):
        """(rows, type) of a key and a value tensor or QuantRows; lead: the extents in
        front of heads, None for any."""
        if not isinstance(pair, (tuple, list)) or len(pair) != 2:
            raise ValueError("%s must be a pair of keys and values" % name)
        x, y = pair
        n = len(lead)
        if type(x) is type(y) and isinstance(x, (torch.Tensor, QuantRows)) and x.shape == y.shape:
            quant, s = isinstance(x, QuantRows), x.shape
            if (len(s) == n + 2 and s[-1] == dim and s[-2] == heads and (n == 1 or s[0] >= lead[0])
                    and (quant or (x.dtype is dtype and y.dtype is dtype))):
                if s[n - 1] <= _INT32_MAX:
                    return s[n - 1], quant
        kinds = set()
        for t in pair:
            if not isinstance(t, (torch.Tensor, QuantRows)):
                raise TypeError("%s must hold tensors or QuantRows" % name)
            s = list(t.shape)
            if (len(s) != len(lead) + 2 or s[-2:] != [heads, dim]
                    or any(w is not None and a < w for a, w in zip(s, lead))):
                raise ValueError("%s must be [%s, %d, %d], got %s" % (
                    name, ", ".join("rows" if w is None else ">=%d" % w for w in lead), heads, dim, s))
            quant = isinstance(t, QuantRows)
            if not quant and t.dtype != dtype:
                raise TypeError("%s must be %s or QuantRows, got %s" % (name, dtype, t.dtype))
            kinds.add(quant)
        if len(kinds) != 1 or pair[0].shape[len(lead) - 1] != pair[1].shape[len(lead) - 1]:
            raise ValueError("%s: keys and values must agree in type and rows" % name)
        return _fits(pair[0].shape[len(lead) - 1], name), kinds.pop()

    def tree_attention(self, q, k, v, n_nodes, mask=None, cache=None, cache_len=None, shared=None,
                       scale=None, with_root=False, out=None, lse=None, workspace=None):
        """Attention of a draft block (graft_tree_attention): q [batch, slots, q_heads, dim],
        k and v [batch, slots, kv_heads, dim], bfloat16 or float16; slot 0 is the root with
        with_root, the tree's nodes follow.  mask [batch, max_nodes, words] int64 as
        build_tree writes it, or None for a chain.  cache: a pair of [batch, rows,
        kv_heads, dim] keys and values, tensors of q's type or QuantRows (bfloat16 only),
        of which sequence b has cache_len[b] rows; shared: a pair of [rows, kv_heads, dim]
        of the cache's type that every sequence sees.  scale defaults to dim ** -0.5.
        Writes out (allocated as zeros when None) up to each sequence's slots and, when
        given, lse [batch, slots, q_heads] float32; returns out.  workspace: uint8, at
        least tree_attention_workspace bytes; allocated when None."""
        a, out = self._attention(q, k, v, n_nodes, mask, cache, cache_len, shared, scale,
                                       with_root, out, lse)
        L = lib()
        need = C.c_int64()
        _check(L.graft_tree_attention_workspace(self._h, C.byref(a), C.byref(need)),
               "graft_tree_attention_workspace")
        workspace = self._workspace(workspace, need.value, q.device)
        if workspace is not None:
            a.workspace, a.workspace_bytes = workspace.data_ptr(), workspace.numel()
        _check(L.graft_tree_attention(self._h, C.byref(a), _stream()), "graft_tree_attention")
        return out

    def tree_attention_workspace(self, q, k, v, n_nodes, mask=None, cache=None, cache_len=None,
                                 shared=None, scale=None, with_root=False, out=None, lse=None):
        """Bytes of workspace that tree_attention needs for these arguments."""
        a, _ = self._attention(q, k, v, n_nodes, mask, cache, cache_len, shared, scale,
                                  with_root, out, lse)
        need = C.c_int64()
        _check(lib().graft_tree_attention_workspace(self._h, C.byref(a), C.byref(need)),
               "graft_tree_attention_workspace")
        return need.value

    def _workspace(self, workspace, need, device):
        if workspace is None:
            return torch.empty(need, dtype=torch.uint8, device=device) if need else None
        if (not isinstance(workspace, torch.Tensor) or workspace.dtype != torch.uint8
                or workspace.dim() != 1 or not workspace.is_contiguous() or workspace.numel() < need):
            raise ValueError("workspace must be a contiguous uint8 vector of at least %d bytes" % need)
        self._here(workspace=workspace)
        return workspace

    def _attention(self, q, k, v, n_nodes, mask, cache, cache_len, shared, scale, with_root, out,
                   lse):
        for name, t in (("q", q), ("k", k), ("v", v)):
            if not isinstance(t, torch.Tensor) or t.dim() != 4 or min(t.shape) < 1:
                raise ValueError("%s must be [batch, slots, heads, dim]" % name)
        shape = q.shape
        B, S, Hq, D = shape
        H, N = k.shape[2], self.dims.max_nodes
        if B | S | Hq | D | H > _INT32_MAX:      # the largest's bits are in it
            _fits(max(B, S, Hq, D, H), "q or k")
        W = (N + 63) // 64
        if k.shape != (B, S, H, D) or v.shape != (B, S, H, D):
            _need(k, "k", B, S, H, D)
            _need(v, "v", B, S, H, D)
        if out is not None and not (isinstance(out, torch.Tensor) and out.shape == shape):
            _need(out, "out", B, S, Hq, D)
        if out is not None and not out.is_contiguous():
            _apart(out, "out")
        if n_nodes is None:
            raise ValueError("n_nodes is required")
        if q.dtype not in (torch.bfloat16, torch.float16):
            raise TypeError("q must be bfloat16 or float16")
        for name, t in (("k", k), ("v", v), ("out", out)):
            if t is not None and t.dtype != q.dtype:
                raise TypeError("%s must be %s" % (name, q.dtype))
        dtype = _DTYPES[q.dtype]
        a = Attention(B, S, 1 if with_root else 0, Hq, H, D, dtype, dtype,
                      float(D ** -0.5 if scale is None else scale))
        quant = None
        if cache is not None:
            if cache_len is None:
                raise ValueError("a cache needs cache_len")
            a.cache_rows, quant = self._kv_pair(cache, "cache", (B, None), H, D, q.dtype)
        if shared is not None:
            a.shared_len, other = self._kv_pair(shared, "shared", (None,), H, D, q.dtype)
            if quant is not None and other != quant:
                raise ValueError("cache and shared must be of one type")
            quant = other
        if quant:
            a.cache_dtype = 3
        ck, cv = cache or (None, None)
        sk, sv = shared or (None, None)
        one, i32 = (B,), torch.int32
        a.n_nodes, a.mask, a.cache_len, a.lse = self._args(
            (("q", q), ("k", k), ("v", v), ("out", out), ("cache keys", ck), ("cache values", cv),
             ("shared keys", sk), ("shared values", sv)),
            ("n_nodes", n_nodes, i32, one, one),
            ("mask", mask, torch.int64, (one, N, W), (B, N, W)),
            ("cache_len", cache_len, i32, one, one),
            ("lse", lse, torch.float32, (B, S, Hq), (B, S, Hq)))
        if out is None:
            out = torch.zeros_like(q, memory_format=torch.contiguous_format)
        a.q, a.k, a.v, a.out = _rows(q, 3, "q"), _rows(k, 3, "k"), _rows(v, 3, "v"), _rows(out, 3, "out")
        if a.cache_rows:
            a.cache_k, a.cache_v = _rows(ck, 3, "cache"), _rows(cv, 3, "cache")
        if a.shared_len:
            a.shared_k, a.shared_v = _rows(sk, 2, "shared"), _rows(sv, 2, "shared")
        return a, out

    def accept_sampled(self, n_nodes, tokens, parents, root_logits, node_logits, uniform,
                       temperature=None, update_history=False, acc_len=None, acc_nodes=None,
                       bonus=None, logp=None, workspace=None):
        """The sampled acceptance walk (graft_accept_sampled).  root_logits [batch, V] and
        node_logits [batch, rows, V] of the target model: float32, bfloat16 or float16,
        unit stride along V (row 0 and rows 1.. of a block's logits, say); nodes from
        `rows` on are not part of the tree.  uniform [batch, L + 1] float64 in [0, 1);
        temperature [batch] float32, 0 for the largest logit, or None for 1.  Returns
        (acc_len, acc_nodes, bonus, logp [batch, L + 1] of the tokens taken)."""
        dm = self.dims
        batch = _batch_of(n_nodes, "n_nodes")
        L, N, V = dm.num_pos, dm.max_nodes, dm.vocab
        if root_logits is None or node_logits is None or uniform is None:
            raise ValueError("root_logits, node_logits and uniform are required")
        _need(root_logits, "root_logits", (batch,), V)
        _need(node_logits, "node_logits", (batch,), (0,), V)
        if root_logits.dtype not in _DTYPES or node_logits.dtype != root_logits.dtype:
            raise TypeError("logits must both be float32, bfloat16 or float16")
        root, node = root_logits.stride(), node_logits.stride()
        if V > 1 and (root[1] != 1 or node[2] != 1):
            raise ValueError("%s must have unit stride along V"
                             % ("root_logits" if root[1] != 1 else "node_logits"))
        i32, f32, one = torch.int32, torch.float32, (batch,)
        if tokens is None or parents is None:
            raise ValueError("tokens and parents are required")
        p_n, p_tok, p_par, p_u, p_t, p_acc, p_path, p_bonus, p_lp = self._args(
            (("root_logits", root_logits), ("node_logits", node_logits)),
            ("n_nodes", n_nodes, i32, one, one),
            ("tokens", tokens, i32, (one, N), (batch, N)),
            ("parents", parents, i32, (one, N), (batch, N)),
            ("uniform", uniform, torch.float64, (one, L + 1), (batch, L + 1)),
            ("temperature", temperature, f32, (one,), one),
            ("acc_len", acc_len, i32, (one,), one),
            ("acc_nodes", acc_nodes, i32, (one, L), (batch, L)),
            ("bonus", bonus, i32, (one,), one),
            ("logp", logp, f32, (one, L + 1), (batch, L + 1)))
        dev = n_nodes.device
        if acc_len is None:
            acc_len = torch.empty(batch, dtype=i32, device=dev)
            p_acc = acc_len.data_ptr()
        if acc_nodes is None:
            acc_nodes = torch.empty(batch, L, dtype=i32, device=dev)
            p_path = acc_nodes.data_ptr()
        if bonus is None:
            bonus = torch.empty(batch, dtype=i32, device=dev)
            p_bonus = bonus.data_ptr()
        if logp is None:
            logp = torch.empty(batch, L + 1, dtype=f32, device=dev)
            p_lp = logp.data_ptr()
        rows = min(node_logits.shape[1], N)
        t = TargetLogits(_DTYPES[root_logits.dtype], root_logits.data_ptr(), root[0],
                         node_logits.data_ptr() if rows else None, node[0],
                         node[1] if rows > 1 else 0, rows, p_t, p_u)
        lib_ = lib()
        need = C.c_int64()
        _check(lib_.graft_accept_sampled_workspace(self._h, batch, C.byref(need)),
               "graft_accept_sampled_workspace")
        workspace = self._workspace(workspace, need.value, dev)
        _check(lib_.graft_accept_sampled(
            self._h, batch, p_n, p_tok, p_par, C.byref(t), p_acc, p_path, p_bonus, p_lp,
            1 if update_history else 0, workspace.data_ptr(), workspace.numel(), _stream()),
            "graft_accept_sampled")
        return acc_len, acc_nodes, bonus, logp

    def _move(self, src, dst, n_rows, start, rows, with_root):
        for name, t in (("src", src), ("dst", dst)):
            if not isinstance(t, (torch.Tensor, QuantRows)):
                raise TypeError("%s must be a tensor or QuantRows" % name)
            if len(t.shape) != 5 or min(t.shape) < 1:
                raise ValueError("%s must be [planes, batch, rows, heads, dim], got %s"
                                 % (name, list(t.shape)))
        batch = _batch_of(n_rows, "n_rows")
        P, _, _, H, D = src.shape
        for name, t in (("src", src), ("dst", dst)):
            s = t.shape
            if s[0] != P or s[1] < batch or s[3] != H or s[4] != D:
                raise ValueError("%s must be [%d, >=%d, rows, %d, %d], got %s"
                                 % (name, P, batch, H, D, list(s)))
        src_rows, dst_rows = src.shape[2], dst.shape[2]
        entries = rows.shape[1] if isinstance(rows, torch.Tensor) and rows.dim() == 2 else 0
        if P | H | D | src_rows | dst_rows | entries > _INT32_MAX:      # the largest's bits are in it
            _fits(max(P, H, D, src_rows, dst_rows, entries), "src, dst or rows")
        to = dst.codes if isinstance(dst, QuantRows) else dst
        if not to.is_contiguous() or to is not dst and not dst.scales.is_contiguous():
            _apart(dst, "dst")
        i32, one = torch.int32, (batch,)
        p_n, p_start, p_list = self._args(
            (("src", src), ("dst", dst)),
            ("n_rows", n_rows, i32, one, one),
            ("start", start, i32, (one,), one),
            ("rows", rows, i32, (one, (1,)), (batch, entries) if entries else None))
        kind = lambda t: 3 if isinstance(t, QuantRows) else _DTYPES.get(t.dtype, -1)
        return CacheMove(batch, P, H, D, kind(src), kind(dst), _rows(src, 4, "src"),
                         _rows(dst, 4, "dst"), src_rows, dst_rows, p_n, p_start, p_list,
                         entries, 1 if with_root else 0)

    def cache_write(self, dst, src, n_rows, rows=None, start=None, with_root=False):
        """Appends rows of src [planes, batch, rows, heads, dim] to the cache dst of the same
        form (graft_cache_write): a tensor of src's type (a copy), or QuantRows (src
        bfloat16).  rows [batch, entries] lists source rows (None: 0 .. n_rows - 1); with
        with_root its entries are tree nodes, at source rows entry + 1, and source row 0 is
        written first.  The first row written is cache row start[b] (None: 0)."""
        m = self._move(src, dst, n_rows, start, rows, with_root)
        _check(lib().graft_cache_write(self._h, C.byref(m), _stream()), "graft_cache_write")
        return dst

    def cache_read(self, src, n_rows, start=None, out=None, dtype=torch.bfloat16):
        """Rows start[b] .. start[b] + n_rows[b] - 1 of the QuantRows src [planes, batch, rows,
        heads, dim] as bfloat16 or float32 numbers in rows 0 .. n_rows[b] - 1 of out, which
        is allocated as zeros of src's shape when None."""
        if not isinstance(src, QuantRows):
            raise TypeError("src must be QuantRows")
        if out is None:
            out = torch.zeros(src.shape, dtype=dtype, device=src.device)
        m = self._move(src, out, n_rows, start, None, False)
        _check(lib().graft_cache_read(self._h, C.byref(m), _stream()), "graft_cache_read")
        return out

    def _pages(self, cache, name, heads, dim, dtype, written=False):
        """(keys, values, quantised, addresses and strides) of a layer's pages [pages, page_rows, heads, dim]."""
        if not isinstance(cache, (tuple, list)) or len(cache) != 2:
            raise ValueError("%s must be a pair of keys and values" % name)
        k, v = cache
        for t in cache:
            if not isinstance(t, (torch.Tensor, QuantRows)):
                raise TypeError("%s must hold tensors or QuantRows" % name)
        quant, s = isinstance(k, QuantRows), k.shape
        if isinstance(v, QuantRows) != quant or v.shape != s:
            raise ValueError("%s: keys and values must agree in type and shape" % name)
        if len(s) != 4 or s[2] != heads or s[3] != dim or s[0] < 1 or s[1] < 1:
            raise ValueError("%s must be [pages, page_rows, %d, %d], got %s" % (name, heads, dim, list(s)))
        if not quant and (k.dtype is not dtype or v.dtype is not dtype):
            raise TypeError("%s must be %s or QuantRows, got %s and %s" % (name, dtype, k.dtype, v.dtype))
        pages, rows = s[0], s[1]
        if pages | rows > _INT32_MAX:
            _fits(max(pages, rows), name)
        at = ()
        for t in cache:
            x = t.codes if quant else t
            st = x.stride()
            if st[3] != 1 and dim > 1:
                raise ValueError("%s must have unit stride along its last dimension" % name)
            # paged_cache's layout, a place for every number, is seen at a glance
            if written and (st != (rows * heads * dim, dim, rows * dim, 1) or (
                    quant and t.scales.stride() != (rows * heads, 1, rows))):
                _apart(t, name)
            at += (x.data_ptr(), st[0] if pages > 1 else 0, st[1] if rows > 1 else 0, st[2] if heads > 1 else 0)
            if quant:
                st = t.scales.stride()
                at += (t.scales.data_ptr(), st[0] if pages > 1 else 0, st[1] if rows > 1 else 0,
                       st[2] if heads > 1 else 0)
        return k, v, quant, at

    def _table(self, page_table, batch):
        """(address, distance of its rows, pages of a sequence) of a page table [batch or more, n]."""
        if not isinstance(page_table, torch.Tensor) or page_table.dim() != 2:
            raise ValueError("page_table must be [batch, pages of a sequence]")
        if page_table.dtype is not torch.int32:
            raise TypeError("page_table must be torch.int32, got %s" % page_table.dtype)
        rows, n = page_table.shape
        if rows < batch or n < 1:
            _need(page_table, "page_table", (batch,), (1,))
        if n > _INT32_MAX:
            _fits(n, "page_table")
        stride, unit = page_table.stride()
        if unit != 1 and n > 1:
            raise ValueError("page_table must have unit stride along its last dimension")
        return page_table.data_ptr(), stride if batch > 1 else 0, n

    def paged_write(self, cache, page_table, k, v, n_rows=None, start=None, q=None, q_out=None, freq=None,
                    positions=None, axis=None, interleaved=False):
        """Rotates a block's queries and keys and appends keys and values to pages
        (graft_paged_write).  cache: a pair of [pages, page_rows, kv_heads, dim] keys and
        values of one layer, tensors of k's type or QuantRows (bfloat16 rows), paged_cache's
        for one; page_table [batch, n] int32 (columns of a wider table, too): row r of sequence
        b is row r % page_rows of page page_table[b, r // page_rows].  k, v [batch, slots, kv_heads, dim] and q
        [batch, slots, q_heads, dim], bfloat16 or float16: slot i < n_rows[b] (None: all)
        goes to row start[b] + i (None: 0).  freq [rot / 2] float64, radians a position,
        rotates the first rot numbers of every head of q and k, in pairs (f, f + rot / 2)
        or, interleaved, (2f, 2f + 1); None rotates nothing.  positions [axes, batch,
        slots] or [batch, slots] int32 (None: start + i), axis [rot / 2] int32 the axis of
        each pair (None: the first).  Returns q_out (None without q; allocated as
        zeros when None; q itself rotates in place)."""
        shape = k.shape if isinstance(k, torch.Tensor) else ()
        if len(shape) != 4 or min(shape) < 1:
            raise ValueError("k must be [batch, slots, heads, dim]")
        B, S, H, D = shape
        kind = k.dtype
        if not isinstance(v, torch.Tensor) or v.shape != shape:
            _need(v, "v", B, S, H, D)
        Hq = 0
        if q is not None:
            if not isinstance(q, torch.Tensor) or q.dim() != 4 or q.shape[2] < 1:
                raise ValueError("q must be [batch, slots, heads, dim]")
            Hq = q.shape[2]
            if q.shape != (B, S, Hq, D):
                _need(q, "q", B, S, Hq, D)
        elif q_out is not None:
            raise ValueError("q_out needs q")
        if B | S | H | Hq | D > _INT32_MAX:
            _fits(max(B, S, H, Hq, D), "q or k")
        if kind is not torch.bfloat16 and kind is not torch.float16:
            raise TypeError("k must be bfloat16 or float16")
        if v.dtype is not kind or (q is not None and q.dtype is not kind):
            raise TypeError("v and q must be %s" % kind)
        if q_out is not None:
            if not isinstance(q_out, torch.Tensor) or q_out.dtype is not kind:
                raise TypeError("q_out must be a tensor of %s" % kind)
            if q_out.shape != q.shape:
                _need(q_out, "q_out", B, S, Hq, D)
            if not q_out.is_contiguous():
                _apart(q_out, "q_out")
        ck, cv, quant, pools = self._pages(cache, "cache", H, D, kind, True)
        F, axes = 0, 1
        if freq is not None:
            if not isinstance(freq, torch.Tensor) or freq.dim() != 1:
                raise ValueError("freq must be [rot / 2]")
            F = freq.shape[0]
            if F < 1 or 2 * F > D:
                raise ValueError("freq must have 1..%d entries, got %d" % (D // 2, F))
        elif positions is not None or axis is not None:
            raise ValueError("positions and axis need freq")
        if positions is not None:
            if not isinstance(positions, torch.Tensor) or positions.dim() not in (2, 3):
                raise ValueError("positions must be [axes, batch, slots] or [batch, slots]")
            if positions.dim() == 2:
                positions = positions[None]
            axes = positions.shape[0]
        elif axis is not None:
            raise ValueError("axis needs positions")
        dtype, one, i32, dev = _DTYPES[kind], (B,), torch.int32, self._device
        table, table_stride, n = self._table(page_table, B)
        p_n, p_start = _at(n_rows, i32, one, dev), _at(start, i32, one, dev)
        p_pos, p_axis, p_freq = 0, 0, 0
        if F:
            p_pos, p_axis = _at(positions, i32, (axes, B, S), dev), _at(axis, i32, (F,), dev)
            p_freq = _at(freq, torch.float64, (F,), dev)
        if (p_n < 0 or p_start < 0 or p_pos < 0 or p_axis < 0 or p_freq < 0
                or not self._all_here((k, v, q, q_out, ck, cv, page_table))):
            p_n, p_start, p_pos, p_axis, p_freq = [p or 0 for p in self._args(
                (("k", k), ("v", v), ("q", q), ("q_out", q_out), ("cache keys", ck), ("cache values", cv),
                 ("page_table", page_table)),
                ("n_rows", n_rows, i32, one, one),
                ("start", start, i32, one, one),
                ("positions", positions, i32, ((1,), B, S), (axes, B, S)),
                ("axis", axis, i32, (F,), (F,)),
                ("freq", freq, torch.float64, (F,), (F,)))]
        queries = _NO_ROWS
        if Hq:
            if q_out is None:
                q_out = torch.zeros_like(q, memory_format=torch.contiguous_format)
            queries = _row_at(q, B, S, Hq, D, "q") + _row_at(q_out, B, S, Hq, D, "q_out")
        pool = ck.shape
        desc = _PACK_ROWS[quant].pack(
            B, S, Hq, H, D, 2 * F, 1 if interleaved else 0, dtype, 3 if quant else dtype, *queries,
            *_row_at(k, B, S, H, D, "k"), *_row_at(v, B, S, H, D, "v"), *pools, table, table_stride, n,
            pool[0], pool[1], p_n, p_start, p_pos, axes, p_axis, p_freq)
        _check(lib().graft_paged_write(self._h, desc, _stream()), "graft_paged_write")
        return q_out

    def _all_here(self, tensors):
        """Whether all that are given are on the context's device, and that is the current one."""
        dev = self._device
        for t in tensors:
            if t is not None and (t.codes if isinstance(t, QuantRows) else t).get_device() != dev:
                return False
        return torch.cuda.current_device() == dev

    def paged_attention(self, q, cache, page_table, cache_len, n_nodes=None, mask=None, scale=None,
                        window=None, sinks=0, with_root=False, out=None, lse=None, workspace=None):
        """Attention of a block over pages (graft_paged_attention): q [batch, slots, q_heads,
        dim], bfloat16 or float16; cache and page_table as in paged_write, the block's own
        rows being rows cache_len[b] + slot (as paged_write leaves them with
        start=cache_len).  n_nodes[b] (+ 1 with_root) slots are used, None: all.  mask
        [batch, max_nodes, words] int64 as build_tree writes it, or None for a chain.
        window: a slot at position p sees rows past p - window, and the first `sinks`
        ones; None: all.  scale defaults to dim ** -0.5.  Writes out (allocated as zeros
        when None) up to each sequence's slots and, when given, lse [batch, slots, q_heads]
        float32; returns out.  workspace: uint8, at least paged_attention_workspace
        bytes; allocated when None."""
        desc, out = self._paged(q, cache, page_table, cache_len, n_nodes, mask, scale, window, sinks, with_root,
                                out, lse)
        L = lib()
        need = C.c_int64()
        _check(L.graft_paged_attention_workspace(self._h, desc, C.byref(need)), "graft_paged_attention_workspace")
        workspace = self._workspace(workspace, need.value, q.device)
        if workspace is not None:
            desc = desc[:-16] + struct.pack("qq", workspace.data_ptr(), workspace.numel())
        _check(L.graft_paged_attention(self._h, desc, _stream()), "graft_paged_attention")
        return out

    def paged_attention_workspace(self, q, cache, page_table, cache_len, n_nodes=None, mask=None, scale=None,
                                  window=None, sinks=0, with_root=False, out=None, lse=None):
        """Bytes of workspace that paged_attention needs for these arguments."""
        desc, _ = self._paged(q, cache, page_table, cache_len, n_nodes, mask, scale, window, sinks, with_root,
                              out, lse)
        need = C.c_int64()
        _check(lib().graft_paged_attention_workspace(self._h, desc, C.byref(need)),
               "graft_paged_attention_workspace")
        return need.value

    def _paged(self, q, cache, page_table, cache_len, n_nodes, mask, scale, window, sinks, with_root, out,
               lse):
        """(its descriptor without a workspace, out)"""
        shape = q.shape if isinstance(q, torch.Tensor) else ()
        if len(shape) != 4 or min(shape) < 1:
            raise ValueError("q must be [batch, slots, heads, dim]")
        kind = q.dtype
        if kind is not torch.bfloat16 and kind is not torch.float16:
            raise TypeError("q must be bfloat16 or float16")
        if cache_len is None:
            raise ValueError("cache_len is required")
        B, S, Hq, D = shape
        if B | S | Hq | D > _INT32_MAX:
            _fits(max(B, S, Hq, D), "q")
        if out is not None:
            if not (isinstance(out, torch.Tensor) and out.shape == shape):
                _need(out, "out", B, S, Hq, D)
            if out.dtype is not kind:
                raise TypeError("out must be %s" % kind)
            if not out.is_contiguous():
                _apart(out, "out")
        if window is None:
            window = 0
        elif not 1 <= window <= _INT32_MAX:
            raise ValueError("window must be 1..2^31 - 1 or None")
        if not 0 <= sinks <= _INT32_MAX:
            raise ValueError("sinks must be 0..2^31 - 1")
        first = cache[0] if isinstance(cache, (tuple, list)) and len(cache) == 2 else None
        H = first.shape[2] if isinstance(first, (torch.Tensor, QuantRows)) and len(first.shape) == 4 else 1
        ck, cv, quant, pools = self._pages(cache, "cache", H, D, kind)
        N = self.dims.max_nodes
        W = (N + 63) // 64
        one, i32, dev = (B,), torch.int32, self._device
        table, table_stride, n = self._table(page_table, B)
        p_len, p_n = _at(cache_len, i32, one, dev), _at(n_nodes, i32, one, dev)
        p_mask, p_lse = _at(mask, torch.int64, (B, N, W), dev), _at(lse, torch.float32, (B, S, Hq), dev)
        if (p_len < 0 or p_n < 0 or p_mask < 0 or p_lse < 0
                or not self._all_here((q, out, ck, cv, page_table))):
            p_len, p_n, p_mask, p_lse = [p or 0 for p in self._args(
                (("q", q), ("out", out), ("cache keys", ck), ("cache values", cv), ("page_table", page_table)),
                ("cache_len", cache_len, i32, one, one),
                ("n_nodes", n_nodes, i32, one, one),
                ("mask", mask, torch.int64, (one, N, W), (B, N, W)),
                ("lse", lse, torch.float32, (B, S, Hq), (B, S, Hq)))]
        if out is None:
            out = torch.zeros_like(q, memory_format=torch.contiguous_format)
        dtype, pool = _DTYPES[kind], ck.shape
        desc = _PACK_ATTENTION[quant].pack(
            B, S, 1 if with_root else 0, Hq, H, D, dtype, 3 if quant else dtype,
            float(D ** -0.5 if scale is None else scale), window, sinks, *_row_at(q, B, S, Hq, D, "q"), p_n, p_mask,
            *pools, table, table_stride, n, pool[0], pool[1], p_len, *_row_at(out, B, S, Hq, D, "out"), p_lse, 0, 0)
        return desc, out

    def paged_commit(self, cache, page_table, start, acc_len, acc_nodes, with_root=False):
        """Moves the accepted path's rows up to the front of the block in the pages
        (graft_paged_commit): cache [planes, pages, page_rows, heads, dim], a tensor or
        QuantRows; row start[b] + r + acc_nodes[b, i] goes to start[b] + r + i for i <
        acc_len[b], r = 1 with_root.  start None: 0.  Returns cache."""
        if not isinstance(cache, (torch.Tensor, QuantRows)):
            raise TypeError("cache must be a tensor or QuantRows")
        if len(cache.shape) != 5 or min(cache.shape) < 1:
            raise ValueError("cache must be [planes, pages, page_rows, heads, dim], got %s" % list(cache.shape))
        batch = _batch_of(acc_len, "acc_len")
        P, pages, rows, H, D = cache.shape
        if P | pages | rows | H | D > _INT32_MAX:
            _fits(max(P, pages, rows, H, D), "cache")
        quant = isinstance(cache, QuantRows)
        x = cache.codes if quant else cache
        st = x.stride()
        if st[4] != 1 and D > 1:
            raise ValueError("cache must have unit stride along its last dimension")
        # paged_cache's layout, a place for every number, is seen at a glance
        if st != (pages * rows * H * D, rows * H * D, D, rows * D, 1) or (
                quant and cache.scales.stride() != (pages * rows * H, rows * H, 1, rows)):
            _apart(cache, "cache")
        if acc_nodes is None:
            raise ValueError("acc_nodes is required")
        L, one, i32, dev = self.dims.num_pos, (batch,), torch.int32, self._device
        table, table_stride, n = self._table(page_table, batch)
        p_start = _at(start, i32, one, dev)
        p_acc, p_nodes = _at(acc_len, i32, one, dev), _at(acc_nodes, i32, (batch, L), dev)
        if p_start < 0 or p_acc < 0 or p_nodes < 0 or not self._all_here((cache, page_table)):
            p_start, p_acc, p_nodes = [p or 0 for p in self._args(
                (("cache", cache), ("page_table", page_table)),
                ("start", start, i32, (one,), one),
                ("acc_len", acc_len, i32, (one,), one),
                ("acc_nodes", acc_nodes, i32, (one, L), (batch, L)))]
        at = (x.data_ptr(), st[1] if pages > 1 else 0, st[2] if rows > 1 else 0, st[3] if H > 1 else 0)
        if quant:
            sc = cache.scales.stride()
            at += (cache.scales.data_ptr(), sc[0] if P > 1 else 0, sc[1] if pages > 1 else 0,
                   sc[2] if rows > 1 else 0, sc[3] if H > 1 else 0)
        desc = _PACK_PATH[quant].pack(
            batch, P, H, D, 3 if quant else _DTYPES.get(cache.dtype, -1), at[0], st[0] if P > 1 else 0, *at[1:],
            table, table_stride, n, pages, rows, p_start, p_acc, p_nodes, 1 if with_root else 0)
        _check(lib().graft_paged_commit(self._h, desc, _stream()), "graft_paged_commit")
        return cache

    def profile_begin(self, max_calls: int):
        _check(lib().graft_profile_begin(self._h, int(max_calls)), "graft_profile_begin")

    def profile_end(self):
        """(summed ms, timed launches) per stage: logits, edges + budget, select, accept."""
        ms = (C.c_double * 4)()
        n = (C.c_int32 * 4)()
        _check(lib().graft_profile_end(self._h, ms, n), "graft_profile_end")
        return list(ms), list(n)

    def device_status(self) -> int:
        return lib().graft_get_device_status(self._h, _stream())


class TdesTrainer:
    """A graft_tdes: one TDES training step per call (objectives of eq.
    tdes-training and AdamW), on tensors the caller owns.  theta, adam_m and
    adam_v are fp32 [param_count] vectors laid out as g_parent [E, m] |
    g_child [E, m] | depth_emb [L, m] | scale."""

    def __init__(self, vocab: int, emb_dim: int, score_dim: int, num_pos: int, top_k: int,
                 max_groups: int, max_pairs: int):
        L = lib()
        self.dims = TdesDims(vocab, emb_dim, score_dim, num_pos, top_k, max_groups, max_pairs)
        h = C.c_void_p()
        _check(L.graft_tdes_create(C.byref(self.dims), C.byref(h)), "graft_tdes_create")
        self._h = h
        self.param_count = int(L.graft_tdes_param_count(C.byref(self.dims)))

    def close(self):
        if getattr(self, "_h", None):
            lib().graft_tdes_destroy(self._h)
            self._h = None

    def __del__(self):  # pragma: no cover
        try:
            self.close()
        except Exception:
            pass

    def split(self, theta):
        """Views (g_parent, g_child, depth_emb, scale) of a parameter vector."""
        d = self.dims
        n = d.emb_dim * d.score_dim
        return (theta[:n].view(d.emb_dim, d.score_dim), theta[n:2 * n].view(d.emb_dim, d.score_dim),
                theta[2 * n:2 * n + d.num_pos * d.score_dim].view(d.num_pos, d.score_dim),
                theta[-1:])

    def step(self, emb, batch: dict, theta, adam_m, adam_v, step: int, hyper: TdesHyper = None,
             loss=None, grad=None):
        """One step on `batch` (CUDA tensors: parent, depth, target int32 [G]; child
        int32 [G, K]; logq, z float32 [G, K]; pairs int32 [P, 6]).  Updates theta,
        adam_m, adam_v in place; writes loss (float64 [4]) and grad when given."""
        p = self._step_plain(emb, batch, theta, adam_m, adam_v, loss, grad)
        if p is None:
            p = self._step_checked(emb, batch, theta, adam_m, adam_v, loss, grad)
        b, p_emb, p_theta, p_m, p_v, p_loss, p_grad = p
        h = hyper if hyper is not None else TdesHyper()
        _check(lib().graft_tdes_step(self._h, p_emb, C.byref(b), C.byref(h), int(step), p_theta, p_m,
                                     p_v, p_loss, p_grad, _stream()), "graft_tdes_step")

    def _step_plain(self, emb, batch, theta, adam_m, adam_v, loss, grad):
        """The step's arguments when every tensor is plain; else None."""
        if type(batch) is not dict:
            return None
        d = self.dims
        i32, f32, f64 = torch.int32, torch.float32, torch.float64
        child, pairs = batch.get("child"), batch.get("pairs")
        if (not isinstance(child, torch.Tensor) or child.dim() != 2
                or not isinstance(pairs, torch.Tensor) or pairs.dim() != 2):
            return None
        G, P = child.shape[0], pairs.shape[0]
        if G < 1 or P < 1:
            return None
        K, n = d.top_k, (self.param_count,)
        per, one = (G, K), (G,)
        g = (_plain(batch.get("parent"), i32, one), _plain(batch.get("depth"), i32, one),
             _plain(child, i32, per), _plain(batch.get("logq"), f32, per),
             _plain(batch.get("z"), f32, per), _plain(batch.get("target"), i32, one))
        p = (_plain(emb, f32, (d.vocab, d.emb_dim)), _plain(theta, f32, n), _plain(adam_m, f32, n),
             _plain(adam_v, f32, n))
        q = (_plain(pairs, i32, (P, 6)), _plain(loss, f64, (4,)), _plain(grad, f32, n))
        if -1 in g or None in g or -1 in p or None in p or -1 in q:
            return None
        return (TdesBatch(G, *g, P, q[0]), *p, q[1], q[2])

    def _step_checked(self, emb, batch, theta, adam_m, adam_v, loss, grad):
        d = self.dims
        G = int(batch["child"].shape[0]) if "child" in batch else 0
        P = int(batch["pairs"].shape[0]) if "pairs" in batch else 0
        if G and tuple(batch["child"].shape) != (G, d.top_k):
            raise ValueError("child must be [G, %d]" % d.top_k)
        i32, f32 = torch.int32, torch.float32
        b = TdesBatch(G, _ptr(batch["parent"], i32, "parent") if G else None,
                      _ptr(batch["depth"], i32, "depth") if G else None,
                      _ptr(batch["child"], i32, "child") if G else None,
                      _ptr(batch["logq"], f32, "logq") if G else None,
                      _ptr(batch["z"], f32, "z") if G else None,
                      _ptr(batch["target"], i32, "target") if G else None,
                      P, _ptr(batch["pairs"], i32, "pairs") if P else None)
        if G:
            for k in ("parent", "depth", "target"):
                if batch[k].numel() != G:
                    raise ValueError("%s must have %d entries" % (k, G))
            for k in ("logq", "z"):
                if tuple(batch[k].shape) != (G, d.top_k):
                    raise ValueError("%s must be [G, K]" % k)
        if P and tuple(batch["pairs"].shape) != (P, 6):
            raise ValueError("pairs must be [P, 6]")
        for name, t in (("theta", theta), ("adam_m", adam_m), ("adam_v", adam_v), ("grad", grad)):
            if t is not None and t.numel() != self.param_count:
                raise ValueError("%s must have %d entries" % (name, self.param_count))
        if tuple(emb.shape) != (d.vocab, d.emb_dim):
            raise ValueError("emb must be [%d, %d]" % (d.vocab, d.emb_dim))
        if loss is not None and (loss.dtype != torch.float64 or loss.numel() < 4):
            raise ValueError("loss must be float64 with 4 entries")
        return (b, _ptr(emb, f32, "emb"), _ptr(theta, f32, "theta"), _ptr(adam_m, f32, "adam_m"),
                _ptr(adam_v, f32, "adam_v"), _ptr(loss, torch.float64, "loss"),
                _ptr(grad, f32, "grad"))

    def device_status(self) -> int:
        return lib().graft_tdes_device_status(self._h, _stream())


def saba_fit(budgets, state, prefix, accepted, latency, tau_min, phi_init, max_iter=200):
    """SABA's gain weights phi and cost c0..c2 fitted on a same-prefix replay
    log (graft_saba_fit): budgets a host sequence of ints; state [T, 3],
    prefix [T] int32, accepted and latency [T, n_budgets] float32 as CUDA
    tensors.  Returns a dict with phi (4), c (3), gain_sse, cost_sse,
    iterations and converged."""
    import numpy as np
    T = int(state.shape[0])
    nb = len(budgets)
    b = np.ascontiguousarray(np.asarray(budgets, np.int32))
    for name, t, shape in (("state", state, (T, 3)), ("accepted", accepted, (T, nb)),
                           ("latency", latency, (T, nb))):
        if tuple(t.shape) != shape:
            raise ValueError("%s must be %s" % (name, shape))
    if tuple(prefix.shape) != (T,):
        raise ValueError("prefix must be [T]")
    log = SabaReplay(T, nb, b.ctypes.data, _ptr(state, torch.float32, "state"),
                     _ptr(prefix, torch.int32, "prefix"), _ptr(accepted, torch.float32, "accepted"),
                     _ptr(latency, torch.float32, "latency"), float(tau_min))
    phi0 = (C.c_float * 4)(*[float(v) for v in phi_init])
    phi = (C.c_float * 4)()
    c = (C.c_float * 3)()
    st = (C.c_double * 4)()
    _check(lib().graft_saba_fit(C.byref(log), phi0, int(max_iter), phi, c, st, _stream()),
           "graft_saba_fit")
    return dict(phi=list(phi), c=list(c), gain_sse=st[0], cost_sse=st[1], iterations=int(st[2]),
                converged=bool(st[3]))


def read_stream(src, sink=None):
    """A plain read of every byte of the contiguous CUDA tensor src
    (graft_read_stream): the streaming read rate to compare the logits pass
    with.  Returns the sink, READ_STREAM_SINK_WORDS int32 words whose xor is the
    xor of src's 32-bit words."""
    if not isinstance(src, torch.Tensor) or src.device.type != "cuda" or not src.is_contiguous():
        raise TypeError("src must be a contiguous CUDA (HIP) tensor")
    if sink is None:
        sink = torch.empty(READ_STREAM_SINK_WORDS, dtype=torch.int32, device=src.device)
    if sink.numel() < READ_STREAM_SINK_WORDS:
        raise ValueError("sink must hold %d words" % READ_STREAM_SINK_WORDS)
    _check(lib().graft_read_stream(src.data_ptr(), src.numel() * src.element_size(),
                                   _ptr(sink, torch.int32, "sink"), _stream()), "graft_read_stream")
    return sink
