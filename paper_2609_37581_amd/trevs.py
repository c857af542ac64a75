"""ctypes binding of libtrevs.so (include/trevs.h).

Argument marshalling only: every step of both pruning stages runs in the HIP
kernels of the library.  PyTorch supplies device memory (outputs, workspace)
and the current stream.  If the library is missing the import of any entry
point raises; there is no fallback path.

A handle (a class here) owns its outputs and workspace, made on the stream that
is current then: a call on another stream has to be ordered after that, and the
handle kept until the stream is past its calls.  The one-off functions see to
both themselves for the stream that they are given.
"""

import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtrevs.so")

TREVS_F32, TREVS_BF16 = 0, 1
PRELLM_NUM_KERNELS = 5
INLLM_NUM_KERNELS = 5
SENSITIVITY_NUM_KERNELS = 7
MAX_SELECT_N = 65536
MAX_FPS_N = 32768
PRELLM_KERNELS = ("prep", "relevance", "norm_stats", "fuse_topk", "gather")
INLLM_KERNELS = ("t2v_stats", "head_var", "token_score", "topk", "compaction")
# both questions run in one launch each; slots without a launch have no name
SENSITIVITY_KERNELS = ("t2v_stats", "head_var", "profile", "", "", "", "sensitivity")

SOFTMAX = {"visual": 0, "causal": 1}  # trevs_softmax
ROPE_SCALING = {"none": 0, "linear": 1, "parts": 2}  # trevs_rope_scaling
MAX_POS_PLANES = 4
MAX_PAGE_REQUESTS = 1024
MAX_BEAMS = 64
MAX_BEAM_OUT = 64

_STATUS = {0: "ok", 1: "invalid argument", 2: "unsupported", 3: "workspace", 4: "hip error"}


class TrevsError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__(f"{where}: {_STATUS.get(status, status)} (status {status})")


c_int32, c_uint32, c_float, c_void_p, c_size_t = (ctypes.c_int32, ctypes.c_uint32, ctypes.c_float,
                                                   ctypes.c_void_p, ctypes.c_size_t)
c_int64, c_double = ctypes.c_int64, ctypes.c_double


class PrellmArgs(ctypes.Structure):
    _fields_ = [("struct_size", c_uint32), ("B", c_int32), ("N", c_int32), ("n_seg", c_int32),
                ("H_v", c_int32), ("d", c_int32), ("M_max", c_int32), ("k_keep", c_int32),
                ("k_div", c_int32), ("textual_ratio", c_float), ("tau_v", c_float),
                ("tau_t", c_float), ("lambda_", c_float), ("eps", c_float), ("dtype", c_int32),
                ("cls_logits", c_void_p), ("vis_feats", c_void_p), ("text_emb", c_void_p),
                ("text_len", c_void_p), ("kept_idx", c_void_p), ("kept_feats", c_void_p),
                ("score_out", c_void_p), ("sal_out", c_void_p), ("rel_out", c_void_p),
                ("norm_stats", c_void_p), ("events", c_void_p), ("ratio_mode", c_int32),
                ("div_idx", c_void_p)]


RATIO_MODES = {"weights": 0, "budget": 1}


class InllmArgs(ctypes.Structure):
    _fields_ = [("struct_size", c_uint32), ("B", c_int32), ("S", c_int32), ("P", c_int32),
                ("K_in", c_int32), ("T_max", c_int32), ("H_q", c_int32), ("H_kv", c_int32),
                ("d_head", c_int32), ("D", c_int32), ("n_pos", c_int32),
                ("n_keep_heads", c_int32), ("k_keep", c_int32), ("scale", c_float),
                ("dtype", c_int32), ("q", c_void_p), ("k", c_void_p), ("v", c_void_p),
                ("hidden", c_void_p), ("pos", c_void_p), ("text_len", c_void_p),
                ("lse_rest", c_void_p), ("kept_idx", c_void_p), ("hidden_out", c_void_p),
                ("k_out", c_void_p), ("v_out", c_void_p), ("pos_out", c_void_p),
                ("head_sel", c_void_p), ("head_var", c_void_p), ("score_out", c_void_p),
                ("events", c_void_p), ("softmax", c_int32), ("row_stats", c_void_p)]


class SensitivityArgs(ctypes.Structure):
    _fields_ = [("struct_size", c_uint32), ("B", c_int32), ("S", c_int32), ("P", c_int32),
                ("K_in", c_int32), ("T_max", c_int32), ("H_q", c_int32), ("H_kv", c_int32),
                ("d_head", c_int32), ("scale", c_float), ("dtype", c_int32),
                ("q", c_void_p * 2), ("k", c_void_p * 2), ("text_len", c_void_p * 2),
                ("lse_rest", c_void_p * 2), ("ts", c_void_p), ("profile", c_void_p * 2),
                ("head_var", c_void_p * 2), ("events", c_void_p), ("softmax", c_int32)]


class RopeArgs(ctypes.Structure):
    _fields_ = [("struct_size", c_uint32), ("B", c_int32), ("S", c_int32), ("H_q", c_int32),
                ("H_k", c_int32), ("d_head", c_int32), ("rot_dim", c_int32), ("n_pos", c_int32),
                ("section", c_int32 * MAX_POS_PLANES), ("interleaved", c_int32),
                ("inverse", c_int32), ("dtype", c_int32), ("attn_factor", c_float),
                ("freqs", c_void_p), ("pos", c_void_p), ("q", c_void_p), ("k", c_void_p),
                ("q_out", c_void_p), ("k_out", c_void_p), ("q_ld", c_int64), ("k_ld", c_int64),
                ("q_out_ld", c_int64), ("k_out_ld", c_int64)]


class Kv8CacheArgs(ctypes.Structure):
    _fields_ = [("struct_size", c_uint32), ("n_layers", c_int32), ("n_pages", c_int32),
                ("page_tokens", c_int32), ("H_kv", c_int32), ("d_head", c_int32),
                ("n_slots", c_int32), ("max_pages", c_int32), ("k", c_void_p), ("v", c_void_p),
                ("k_scale", c_void_p), ("v_scale", c_void_p), ("table", c_void_p),
                ("len", c_void_p), ("ref", c_void_p)]


class Kv8WriteArgs(ctypes.Structure):
    _fields_ = [("struct_size", c_uint32), ("B", c_int32), ("T_max", c_int32), ("layer", c_int32),
                ("dtype", c_int32), ("k", c_void_p), ("v", c_void_p), ("k_ld", c_int64),
                ("v_ld", c_int64), ("n_new", c_void_p), ("slots", c_void_p)]


class Kv8AttentionArgs(ctypes.Structure):
    _fields_ = [("struct_size", c_uint32), ("B", c_int32), ("T_max", c_int32), ("H_q", c_int32),
                ("layer", c_int32), ("dtype", c_int32), ("causal", c_int32), ("kv_max", c_int32),
                ("scale", c_float), ("q", c_void_p), ("q_ld", c_int64), ("q_len", c_void_p),
                ("slots", c_void_p), ("out", c_void_p), ("lse", c_void_p)]


class Kv8CompactArgs(ctypes.Structure):
    _fields_ = [("struct_size", c_uint32), ("B", c_int32), ("P", c_int32), ("K_in", c_int32),
                ("n_kept", c_int32), ("kept_idx", c_void_p), ("src_slots", c_void_p),
                ("dst_slots", c_void_p)]


class NormRopeArgs(ctypes.Structure):
    _fields_ = [("struct_size", c_uint32), ("eps", c_float), ("weight_offset", c_float),
                ("weight_dtype", c_int32), ("per_head", c_int32), ("q_weight", c_void_p),
                ("k_weight", c_void_p), ("rope", RopeArgs)]


class Kv8WeightsArgs(ctypes.Structure):
    _fields_ = [("struct_size", c_uint32), ("B", c_int32), ("T_max", c_int32), ("H_q", c_int32),
                ("layer", c_int32), ("dtype", c_int32), ("causal", c_int32), ("kv_max", c_int32),
                ("scale", c_float), ("decay", c_float), ("q", c_void_p), ("q_ld", c_int64),
                ("q_len", c_void_p), ("slots", c_void_p), ("lse", c_void_p), ("score", c_void_p)]


class Kv8EvictArgs(ctypes.Structure):
    _fields_ = [("struct_size", c_uint32), ("B", c_int32), ("n_keep", c_int32), ("n_first", c_int32),
                ("n_last", c_int32), ("keep", c_void_p), ("slots", c_void_p), ("score", c_void_p),
                ("n_evicted", c_void_p), ("kept_idx", c_void_p)]


class BeamSelectArgs(ctypes.Structure):
    _fields_ = [("struct_size", c_uint32), ("B", c_int32), ("W", c_int32), ("V", c_int32),
                ("n_out", c_int32), ("dtype", c_int32), ("eos", c_int32), ("logits", c_void_p),
                ("logits_ld", c_int64), ("score", c_void_p), ("done", c_void_p),
                ("score_out", c_void_p), ("parent", c_void_p), ("token", c_void_p)]


def _torch_empty(shape, dtype, device):
    return torch.empty(shape, dtype=dtype, device=device)


_alloc = _torch_empty


def set_allocator(fn=None):
    """Route every output and workspace allocation of this binding through
    fn(shape, dtype, device) -> contiguous tensor (None: torch.empty).
    Returns the previous allocator.  The tests use it to surround each
    buffer with guard bands."""
    global _alloc
    prev = _alloc
    _alloc = fn or _torch_empty
    return prev


def _empty(shape, dtype, device):
    t = _alloc(tuple(shape), dtype, device)
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype or not t.is_contiguous():
        raise RuntimeError("allocator returned a tensor of the wrong shape, dtype or layout")
    return t


_lib = None


def lib():
    """The loaded library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2609_37581_amd.build`")
        L = ctypes.CDLL(LIB_PATH)
        L.trevs_prellm_workspace_size.argtypes = [ctypes.POINTER(PrellmArgs)]
        L.trevs_prellm_workspace_size.restype = c_size_t
        L.trevs_inllm_workspace_size.argtypes = [ctypes.POINTER(InllmArgs)]
        L.trevs_inllm_workspace_size.restype = c_size_t
        L.trevs_topk_workspace_size.argtypes = [c_int32, c_int32, c_int32]
        L.trevs_topk_workspace_size.restype = c_size_t
        L.trevs_prellm_prune.argtypes = [ctypes.POINTER(PrellmArgs), c_void_p, c_size_t, c_void_p]
        L.trevs_prellm_prune.restype = ctypes.c_int
        L.trevs_inllm_prune.argtypes = [ctypes.POINTER(InllmArgs), c_void_p, c_size_t, c_void_p]
        L.trevs_inllm_prune.restype = ctypes.c_int
        L.trevs_inllm_prune_noalloc.argtypes = [ctypes.POINTER(InllmArgs), c_void_p]
        L.trevs_inllm_prune_noalloc.restype = ctypes.c_int
        L.trevs_topk_select.argtypes = [c_void_p, c_int32, c_int32, c_int32, c_void_p, c_void_p,
                                        c_size_t, c_void_p]
        L.trevs_topk_select.restype = ctypes.c_int
        L.trevs_status_string.argtypes = [ctypes.c_int]
        L.trevs_status_string.restype = ctypes.c_char_p
        L.trevs_keep_count.argtypes = [c_float, c_int32]
        L.trevs_keep_count.restype = c_int32
        L.trevs_sensitivity_workspace_size.argtypes = [ctypes.POINTER(SensitivityArgs)]
        L.trevs_sensitivity_workspace_size.restype = c_size_t
        L.trevs_text_sensitivity.argtypes = [ctypes.POINTER(SensitivityArgs), c_void_p, c_size_t,
                                             c_void_p]
        L.trevs_text_sensitivity.restype = ctypes.c_int
        L.trevs_spearman_workspace_size.argtypes = [c_int32, c_int32, c_int32]
        L.trevs_spearman_workspace_size.restype = c_size_t
        L.trevs_topk_spearman.argtypes = [c_void_p, c_void_p, c_int32, c_int32, c_int32, c_void_p,
                                          c_void_p, c_void_p, c_size_t, c_void_p]
        L.trevs_topk_spearman.restype = ctypes.c_int
        L.trevs_rope.argtypes = [ctypes.POINTER(RopeArgs), c_void_p]
        L.trevs_rope.restype = ctypes.c_int
        L.trevs_rope_frequencies.argtypes = [c_int32, c_double, c_int32, c_double, c_double, c_double,
                                             c_double, c_void_p]
        L.trevs_rope_frequencies.restype = ctypes.c_int
        cache = ctypes.POINTER(Kv8CacheArgs)
        L.trevs_pages_reserve.argtypes = [cache, c_int32] + [c_void_p] * 6
        L.trevs_pages_reserve.restype = ctypes.c_int
        L.trevs_pages_fork.argtypes = [cache, c_int32] + [c_void_p] * 5
        L.trevs_pages_fork.restype = ctypes.c_int
        L.trevs_pages_free.argtypes = [cache, c_int32] + [c_void_p] * 3
        L.trevs_pages_free.restype = ctypes.c_int
        L.trevs_kv8_copy_pages.argtypes = [cache, c_int32] + [c_void_p] * 3
        L.trevs_kv8_copy_pages.restype = ctypes.c_int
        L.trevs_kv8_write.argtypes = [cache, ctypes.POINTER(Kv8WriteArgs), c_void_p]
        L.trevs_kv8_write.restype = ctypes.c_int
        L.trevs_kv8_attention_workspace_size.argtypes = [cache, ctypes.POINTER(Kv8AttentionArgs)]
        L.trevs_kv8_attention_workspace_size.restype = c_size_t
        L.trevs_kv8_attention.argtypes = [cache, ctypes.POINTER(Kv8AttentionArgs), c_void_p, c_size_t,
                                          c_void_p]
        L.trevs_kv8_attention.restype = ctypes.c_int
        L.trevs_kv8_compact.argtypes = [cache, ctypes.POINTER(Kv8CompactArgs), c_void_p]
        L.trevs_kv8_compact.restype = ctypes.c_int
        L.trevs_norm_rope.argtypes = [ctypes.POINTER(NormRopeArgs), c_void_p]
        L.trevs_norm_rope.restype = ctypes.c_int
        L.trevs_kv8_weights_workspace_size.argtypes = [cache, ctypes.POINTER(Kv8WeightsArgs)]
        L.trevs_kv8_weights_workspace_size.restype = c_size_t
        L.trevs_kv8_weights.argtypes = [cache, ctypes.POINTER(Kv8WeightsArgs), c_void_p, c_size_t, c_void_p]
        L.trevs_kv8_weights.restype = ctypes.c_int
        L.trevs_kv8_evict_workspace_size.argtypes = [cache, ctypes.POINTER(Kv8EvictArgs)]
        L.trevs_kv8_evict_workspace_size.restype = c_size_t
        L.trevs_kv8_evict.argtypes = [cache, ctypes.POINTER(Kv8EvictArgs), c_void_p, c_size_t, c_void_p]
        L.trevs_kv8_evict.restype = ctypes.c_int
        L.trevs_beam_select_workspace_size.argtypes = [ctypes.POINTER(BeamSelectArgs)]
        L.trevs_beam_select_workspace_size.restype = c_size_t
        L.trevs_beam_select.argtypes = [ctypes.POINTER(BeamSelectArgs), c_void_p, c_size_t, c_void_p]
        L.trevs_beam_select.restype = ctypes.c_int
        L.trevs_pages_reorder.argtypes = [cache, c_int32, c_int32] + [c_void_p] * 4
        L.trevs_pages_reorder.restype = ctypes.c_int
        for size, struct in ((L.trevs_prellm_args_size, PrellmArgs), (L.trevs_inllm_args_size, InllmArgs),
                             (L.trevs_sensitivity_args_size, SensitivityArgs),
                             (L.trevs_rope_args_size, RopeArgs), (L.trevs_kv8_cache_size, Kv8CacheArgs),
                             (L.trevs_kv8_write_args_size, Kv8WriteArgs),
                             (L.trevs_kv8_attention_args_size, Kv8AttentionArgs),
                             (L.trevs_kv8_compact_args_size, Kv8CompactArgs),
                             (L.trevs_norm_rope_args_size, NormRopeArgs),
                             (L.trevs_kv8_weights_args_size, Kv8WeightsArgs),
                             (L.trevs_kv8_evict_args_size, Kv8EvictArgs),
                             (L.trevs_beam_select_args_size, BeamSelectArgs)):
            size.restype = c_size_t
            if size() == ctypes.sizeof(struct):
                continue
            raise RuntimeError("libtrevs.so argument structs do not match this binding")
        _lib = L
    return _lib


def keep_count(ratio, n):
    return int(lib().trevs_keep_count(ratio, n))


def _dtype_code(t):
    if t.dtype == torch.float32:
        return TREVS_F32
    if t.dtype == torch.bfloat16:
        return TREVS_BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _ptr(t):
    return None if t is None else t.data_ptr()


def _check(t, name, device, ndim=None, dtype=None):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a tensor")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if ndim is not None and t.dim() != ndim:
        raise ValueError(f"{name} must have {ndim} dims, got {tuple(t.shape)}")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")


def _stream(stream):
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _one_off(stream, device, run, *inputs):
    """run(), which makes a handle and calls it, on `stream` (None: torch's
    current one).  What it allocates is that stream's memory, so a workspace
    that is dropped on return is not taken by another stream's tensors while
    this one still works in it; the inputs, which may be dropped too, are kept
    from reuse until `stream` is past them, and the outputs until the caller's
    stream is."""
    if stream is None or stream == torch.cuda.current_stream(device):
        return run()
    if stream.device != device:
        raise ValueError(f"the stream is on {stream.device}, the tensors are on {device}")
    caller = torch.cuda.current_stream(device)
    with torch.cuda.stream(stream):
        out = run()
    for t in inputs:
        for x in t.tensors if isinstance(t, Kv8Cache) else (t,):
            if x is not None:
                x.record_stream(stream)
    for t in out if isinstance(out, tuple) else (out,):
        if t is not None:
            t.record_stream(caller)
    return out


class _EventArray:
    def __init__(self, events, n_kernels):
        if events is None:
            self.ptr = None
            return
        if len(events) != 2 * n_kernels:
            raise ValueError(f"events must hold {2 * n_kernels} handles (None allowed)")
        self.arr = (c_void_p * len(events))(*[e for e in events])
        self.ptr = ctypes.cast(self.arr, c_void_p)


class Prellm:
    """Stage 1 with outputs and workspace allocated once; call() enqueues it."""

    def __init__(self, cls_logits, vis_feats, text_emb, text_len=None, *, k_keep, n_seg=1,
                 k_div=0, textual_ratio=0.5, tau_v=1.4, tau_t=1.0, lambda_=1.0, eps=1e-8,
                 want_scores=False, ratio_mode="weights"):
        dev = vis_feats.device
        _check(vis_feats, "vis_feats", dev, 3)
        dt = vis_feats.dtype
        _check(cls_logits, "cls_logits", dev, 3, dt)
        _check(text_emb, "text_emb", dev, 3, dt)
        if text_len is not None:
            _check(text_len, "text_len", dev, 1, torch.int32)
        B, N, d = vis_feats.shape
        H_v = cls_logits.shape[1]
        M_max = text_emb.shape[1]
        if cls_logits.shape != (B, H_v, N) or text_emb.shape != (B, M_max, d):
            raise ValueError("inconsistent stage-1 shapes")
        if text_len is not None and text_len.shape != (B,):
            raise ValueError("text_len must be [B]")
        self.inputs = (cls_logits, vis_feats, text_emb, text_len)
        self.kept_idx = _empty((B, k_keep), torch.int32, dev)
        # farthest-point diversity tokens in pick order (k_div > 0)
        self.div_idx = _empty((B, k_div), torch.int32, dev) if k_div > 0 else None
        self.kept_feats = _empty((B, k_keep, d), dt, dev)
        if ratio_mode not in RATIO_MODES:
            raise ValueError(f"ratio_mode must be one of {sorted(RATIO_MODES)}")
        budget = ratio_mode == "budget"
        if want_scores:
            # the budget split ranks the raw scores: no fused score, no Med/MAD
            self.score = None if budget else _empty((B, N), torch.float32, dev)
            self.sal = _empty((B, N), torch.float32, dev)
            self.rel = _empty((B, N), torch.float32, dev)
            self.norm_stats = None if budget else _empty((B, 4), torch.float32, dev)
        else:
            self.score = self.sal = self.rel = self.norm_stats = None
        a = PrellmArgs()
        a.struct_size = ctypes.sizeof(PrellmArgs)
        a.B, a.N, a.n_seg, a.H_v, a.d, a.M_max = B, N, n_seg, H_v, d, M_max
        a.k_keep, a.k_div = k_keep, k_div
        a.textual_ratio, a.tau_v, a.tau_t, a.lambda_, a.eps = textual_ratio, tau_v, tau_t, lambda_, eps
        a.dtype = _dtype_code(vis_feats)
        a.cls_logits, a.vis_feats, a.text_emb = _ptr(cls_logits), _ptr(vis_feats), _ptr(text_emb)
        a.text_len = _ptr(text_len)
        a.kept_idx, a.kept_feats = _ptr(self.kept_idx), _ptr(self.kept_feats)
        a.score_out, a.sal_out, a.rel_out = _ptr(self.score), _ptr(self.sal), _ptr(self.rel)
        a.norm_stats = _ptr(self.norm_stats)
        a.ratio_mode = RATIO_MODES[ratio_mode]
        a.div_idx = _ptr(self.div_idx)
        self.args = a
        ws = lib().trevs_prellm_workspace_size(ctypes.byref(a))
        if ws == 0:
            # invalid arguments: let the call report the precise status
            st = lib().trevs_prellm_prune(ctypes.byref(a), None, 0, None)
            raise TrevsError(st, "trevs_prellm_prune")
        self.workspace = _empty((ws,), torch.uint8, dev)

    def __call__(self, stream=None, events=None):
        ev = _EventArray(events, PRELLM_NUM_KERNELS)
        self.args.events = ev.ptr
        st = lib().trevs_prellm_prune(ctypes.byref(self.args), self.workspace.data_ptr(),
                                      self.workspace.numel(), _stream(stream))
        self.args.events = None
        if st:
            raise TrevsError(st, "trevs_prellm_prune")
        return self.kept_idx, self.kept_feats


def prellm_prune(cls_logits, vis_feats, text_emb, text_len=None, **kw):
    """Stage 1 (Sec. 4.1): returns (kept_idx [B,K1] int32, kept_feats [B,K1,d]),
    plus a dict of scores when want_scores=True."""
    call = Prellm(cls_logits, vis_feats, text_emb, text_len, **kw)
    idx, feats = call()
    if kw.get("want_scores"):
        return idx, feats, dict(score=call.score, sal=call.sal, rel=call.rel,
                                norm_stats=call.norm_stats)
    return idx, feats


class Inllm:
    """Stage 2 with outputs and workspace allocated once; call() enqueues it."""

    def __init__(self, q, k, v, hidden, pos, text_len=None, *, P, K_in, n_keep_heads, k_keep,
                 scale=None, lse_rest=None, want_scores=False, softmax="visual", noalloc=False,
                 row_stats=None):
        dev = hidden.device
        _check(hidden, "hidden", dev, 3)
        dt = hidden.dtype
        _check(q, "q", dev, 4, dt)
        _check(k, "k", dev, 4, dt)
        _check(v, "v", dev, 4, dt)
        _check(pos, "pos", dev, 3, torch.int64)
        if text_len is not None:
            _check(text_len, "text_len", dev, 1, torch.int32)
        if lse_rest is not None:
            _check(lse_rest, "lse_rest", dev, 3, torch.float32)
        if row_stats is not None:
            _check(row_stats, "row_stats", dev, 4, torch.float32)
        B, S, D = hidden.shape
        H_q, d_head = q.shape[2], q.shape[3]
        H_kv = k.shape[2]
        n_pos = pos.shape[0]
        T_max = S - P - K_in
        if q.shape[:2] != (B, S) or k.shape != (B, S, H_kv, d_head) or v.shape != k.shape:
            raise ValueError("inconsistent stage-2 shapes")
        if pos.shape != (n_pos, B, S):
            raise ValueError("pos must be [n_pos,B,S]")
        if T_max < 1:
            raise ValueError("no text rows after the visual block")
        if lse_rest is not None and lse_rest.shape != (B, H_q, T_max):
            raise ValueError("lse_rest must be [B,H_q,T_max]")
        if row_stats is not None and row_stats.shape != (B, H_q, T_max, 3):
            raise ValueError("row_stats must be [B,H_q,T_max,3]")
        So = S - K_in + k_keep
        self.inputs = (q, k, v, hidden, pos, text_len, lse_rest, row_stats)
        self.kept_idx = _empty((B, k_keep), torch.int32, dev)
        self.hidden_out = _empty((B, So, D), dt, dev)
        self.k_out = _empty((B, So, H_kv, d_head), dt, dev)
        self.v_out = _empty((B, So, H_kv, d_head), dt, dev)
        self.pos_out = _empty((n_pos, B, So), torch.int64, dev)
        if want_scores:
            self.head_sel = _empty((B, n_keep_heads), torch.int32, dev)
            self.head_var = _empty((B, H_q), torch.float32, dev)
            self.score = _empty((B, K_in), torch.float32, dev)
        else:
            self.head_sel = self.head_var = self.score = None
        a = InllmArgs()
        a.struct_size = ctypes.sizeof(InllmArgs)
        a.B, a.S, a.P, a.K_in, a.T_max = B, S, P, K_in, T_max
        a.H_q, a.H_kv, a.d_head, a.D, a.n_pos = H_q, H_kv, d_head, D, n_pos
        a.n_keep_heads, a.k_keep = n_keep_heads, k_keep
        a.scale = float(scale) if scale is not None else d_head ** -0.5
        a.dtype = _dtype_code(hidden)
        a.q, a.k, a.v, a.hidden, a.pos = _ptr(q), _ptr(k), _ptr(v), _ptr(hidden), _ptr(pos)
        a.text_len, a.lse_rest = _ptr(text_len), _ptr(lse_rest)
        a.row_stats = _ptr(row_stats)
        a.softmax = SOFTMAX[softmax]
        a.kept_idx, a.hidden_out = _ptr(self.kept_idx), _ptr(self.hidden_out)
        a.k_out, a.v_out, a.pos_out = _ptr(self.k_out), _ptr(self.v_out), _ptr(self.pos_out)
        a.head_sel, a.head_var, a.score_out = _ptr(self.head_sel), _ptr(self.head_var), _ptr(self.score)
        self.args = a
        ws = lib().trevs_inllm_workspace_size(ctypes.byref(a))
        if ws == 0:
            st = lib().trevs_inllm_prune(ctypes.byref(a), None, 0, None)
            raise TrevsError(st, "trevs_inllm_prune")
        # noalloc: the library's static per-GPU workspace (trevs_inllm_prune_noalloc)
        self.noalloc = noalloc
        self.workspace = None if noalloc else _empty((ws,), torch.uint8, dev)

    def __call__(self, stream=None, events=None):
        ev = _EventArray(events, INLLM_NUM_KERNELS)
        self.args.events = ev.ptr
        if self.noalloc:
            st = lib().trevs_inllm_prune_noalloc(ctypes.byref(self.args), _stream(stream))
        else:
            st = lib().trevs_inllm_prune(ctypes.byref(self.args), self.workspace.data_ptr(),
                                         self.workspace.numel(), _stream(stream))
        self.args.events = None
        if st:
            raise TrevsError(st, "trevs_inllm_prune_noalloc" if self.noalloc else "trevs_inllm_prune")
        return self.kept_idx, self.hidden_out, self.k_out, self.v_out, self.pos_out


def inllm_prune(q, k, v, hidden, pos, text_len=None, **kw):
    """Stage 2 (Sec. 4.2): returns (kept_idx, hidden_out, k_out, v_out,
    pos_out), plus a dict of head_sel/head_var/score when want_scores=True."""
    call = Inllm(q, k, v, hidden, pos, text_len, **kw)
    out = call()
    if kw.get("want_scores"):
        return out + (dict(head_sel=call.head_sel, head_var=call.head_var, score=call.score),)
    return out


def topk_select(scores, k, stream=None):
    """Stable top-k of each row of scores [B,N] (fp32, device) -> int32 [B,k]
    ascending."""
    _check(scores, "scores", scores.device, 2, torch.float32)
    B, N = scores.shape

    def run():
        out = _empty((B, k), torch.int32, scores.device)
        st = lib().trevs_topk_select(scores.data_ptr(), B, N, k, out.data_ptr(), None, 0, _stream(None))
        if st:
            raise TrevsError(st, "trevs_topk_select")
        return out

    return _one_off(stream, scores.device, run, scores)


# ---------------------------------------------------------------- diagnostics
class TextSensitivity:
    """Eq. (1) for every head (Sec. 3): one image with two questions, each a
    stage-2 input (q [B,S,H_q,d_h], k [B,S,H_kv,d_h], same shapes).  Outputs
    ts [B,H_q] and, per question, the visual profiles [B,H_q,K_in] and head
    variances [B,H_q]; allocated once, call() enqueues the computation."""

    def __init__(self, q, k, q2, k2, text_len=None, text_len2=None, *, P, K_in, scale=None,
                 lse_rest=None, lse_rest2=None, softmax="visual"):
        dev = q.device
        dt = q.dtype
        for t, name in ((q, "q"), (k, "k"), (q2, "q2"), (k2, "k2")):
            _check(t, name, dev, 4, dt)
        for t, name in ((text_len, "text_len"), (text_len2, "text_len2")):
            if t is not None:
                _check(t, name, dev, 1, torch.int32)
        B, S, H_q, d_head = q.shape
        H_kv = k.shape[2]
        T_max = S - P - K_in
        if q2.shape != q.shape or k.shape != (B, S, H_kv, d_head) or k2.shape != k.shape:
            raise ValueError("inconsistent shapes of the two questions")
        if T_max < 1:
            raise ValueError("no text rows after the visual block")
        for t, name in ((lse_rest, "lse_rest"), (lse_rest2, "lse_rest2")):
            if t is not None:
                _check(t, name, dev, 3, torch.float32)
                if t.shape != (B, H_q, T_max):
                    raise ValueError(f"{name} must be [B,H_q,T_max]")
        self.inputs = (q, k, q2, k2, text_len, text_len2, lse_rest, lse_rest2)
        self.ts = _empty((B, H_q), torch.float32, dev)
        self.profile = [_empty((B, H_q, K_in), torch.float32, dev) for _ in range(2)]
        self.head_var = [_empty((B, H_q), torch.float32, dev) for _ in range(2)]
        a = SensitivityArgs()
        a.struct_size = ctypes.sizeof(SensitivityArgs)
        a.B, a.S, a.P, a.K_in, a.T_max = B, S, P, K_in, T_max
        a.H_q, a.H_kv, a.d_head = H_q, H_kv, d_head
        a.scale = float(scale) if scale is not None else d_head ** -0.5
        a.dtype = _dtype_code(q)
        a.q[0], a.q[1], a.k[0], a.k[1] = _ptr(q), _ptr(q2), _ptr(k), _ptr(k2)
        a.text_len[0], a.text_len[1] = _ptr(text_len), _ptr(text_len2)
        a.lse_rest[0], a.lse_rest[1] = _ptr(lse_rest), _ptr(lse_rest2)
        a.softmax = SOFTMAX[softmax]
        a.ts = _ptr(self.ts)
        a.profile[0], a.profile[1] = _ptr(self.profile[0]), _ptr(self.profile[1])
        a.head_var[0], a.head_var[1] = _ptr(self.head_var[0]), _ptr(self.head_var[1])
        self.args = a
        ws = lib().trevs_sensitivity_workspace_size(ctypes.byref(a))
        if ws == 0:
            st = lib().trevs_text_sensitivity(ctypes.byref(a), None, 0, None)
            raise TrevsError(st, "trevs_text_sensitivity")
        self.workspace = _empty((ws,), torch.uint8, dev)

    def __call__(self, stream=None, events=None):
        ev = _EventArray(events, SENSITIVITY_NUM_KERNELS)
        self.args.events = ev.ptr
        st = lib().trevs_text_sensitivity(ctypes.byref(self.args), self.workspace.data_ptr(),
                                          self.workspace.numel(), _stream(stream))
        self.args.events = None
        if st:
            raise TrevsError(st, "trevs_text_sensitivity")
        return self.ts


def text_sensitivity(q, k, q2, k2, text_len=None, text_len2=None, **kw):
    """Eq. (1): returns (ts [B,H_q], [profile0, profile1], [head_var0, head_var1])."""
    call = TextSensitivity(q, k, q2, k2, text_len, text_len2, **kw)
    call()
    return call.ts, call.profile, call.head_var


class TopkSpearman:
    """Spearman correlation of s^v and s^t within the top-k saliency set of
    each sample (Sec. 3), outputs and workspace allocated once.  sv, st
    [B,N] fp32 on the device; call() enqueues it and returns (rho float64
    [B], kept_idx int32 [B,k] ascending)."""

    def __init__(self, sv, st, k):
        _check(sv, "sv", sv.device, 2, torch.float32)
        _check(st, "st", sv.device, 2, torch.float32)
        if st.shape != sv.shape:
            raise ValueError("sv and st must have one shape")
        self.inputs = (sv, st)
        self.B, self.N = sv.shape
        self.k = k
        self.rho = _empty((self.B,), torch.float64, sv.device)
        self.kept_idx = _empty((self.B, k), torch.int32, sv.device)
        self.ws_bytes = lib().trevs_spearman_workspace_size(self.B, self.N, k)
        self.workspace = _empty((max(self.ws_bytes, 1),), torch.uint8, sv.device)

    def __call__(self, stream=None):
        sv, st = self.inputs
        stat = lib().trevs_topk_spearman(sv.data_ptr(), st.data_ptr(), self.B, self.N, self.k,
                                         self.rho.data_ptr(), self.kept_idx.data_ptr(),
                                         self.workspace.data_ptr(), self.ws_bytes, _stream(stream))
        if stat:
            raise TrevsError(stat, "trevs_topk_spearman")
        return self.rho, self.kept_idx


def topk_spearman(sv, st, k, stream=None):
    """Spearman correlation of s^v and s^t within the top-k saliency set of
    each sample (Sec. 3).  sv, st [B,N] fp32 on the device.  Returns
    (rho float64 [B], kept_idx int32 [B,k] ascending)."""
    return _one_off(stream, sv.device, lambda: TopkSpearman(sv, st, k)(), sv, st)


# ------------------------------------------------------------- serving cache
def _row_ld(t, name, device, dtype, heads=None):
    """Elements from one row of t [B,T,H,d] to the next: heads and channels
    dense, rows evenly spaced (a slice of a fused projection is)."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a tensor")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")
    if t.dim() != 4 or min(t.shape) < 1:
        raise ValueError(f"{name} must be a non-empty [B,T,H,d], got {tuple(t.shape)}")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    B, T, H, d = t.shape
    sb, st, sh, sd = t.stride()
    ld = st if T > 1 else sb if B > 1 else H * d
    if sd != 1 or (H > 1 and sh != d) or (B > 1 and sb != T * ld) or ld < H * d:
        raise ValueError(f"{name} must have dense heads and evenly spaced rows")
    return ld


def _check_list(t, name, device, n=None):
    if t is None:
        return
    _check(t, name, device, 1, torch.int32)
    if n is not None and t.shape != (n,):
        raise ValueError(f"{name} must be [{n}]")


def _call(fn, device, stream, *args):
    """fn(*args, stream) on the tensors' device: with torch's current stream
    there unless one is given (the raw handle: making a Stream object and
    switching to a device that is current already cost 4 us of a 9 us call)."""
    if device.index == torch.cuda.current_device():
        s = torch._C._cuda_getCurrentRawStream(device.index) if stream is None else stream.cuda_stream
        st = fn(*args, s)
    else:
        with torch.cuda.device(device):
            st = fn(*args, _stream(stream))
    if st:
        raise TrevsError(st, fn.__name__)


def rope_frequencies(rot_dim, *, base=10000.0, scaling="none", factor=1.0, original_len=0,
                     beta_fast=32.0, beta_slow=1.0):
    """Frequencies of Rope, float64 [rot_dim/2] on the host, in turns per
    position: base^(-2i/rot_dim) / 2 pi; for longer contexts divided by
    `factor` in every pair (scaling="linear") or by parts ("parts": pairs that
    turn beta_fast times or more over original_len positions not at all, those
    of beta_slow or less in full, between them in proportion)."""
    if scaling not in ROPE_SCALING:
        raise ValueError(f"scaling must be one of {sorted(ROPE_SCALING)}")
    out = torch.empty(max(int(rot_dim) // 2, 1), dtype=torch.float64)
    st = lib().trevs_rope_frequencies(rot_dim, base, ROPE_SCALING[scaling], factor, original_len,
                                      beta_fast, beta_slow, out.data_ptr())
    if st:
        raise TrevsError(st, "trevs_rope_frequencies")
    return out


def _fill_rope(a, q, k, pos, freqs, sections, interleaved, attn_factor, inplace):
    """The arguments of a rotation (inverse aside) and its outputs."""
    dev = q.device
    dt = q.dtype
    if dev.type != "cuda":
        raise ValueError("q must be on a GPU")
    a.struct_size = ctypes.sizeof(RopeArgs)
    a.dtype = _dtype_code(q)
    a.q_ld = _row_ld(q, "q", dev, dt)
    a.B, a.S, a.H_q, a.d_head = q.shape
    if k is not None:
        a.k_ld = _row_ld(k, "k", dev, dt)
        if k.shape[:2] != q.shape[:2] or k.shape[3] != q.shape[3]:
            raise ValueError("inconsistent shapes of q and k")
        a.H_k = k.shape[2]
    _check(pos, "pos", dev, 3, torch.int64)
    _check(freqs, "freqs", dev, 1, torch.float64)
    if pos.shape[1:] != q.shape[:2]:
        raise ValueError("pos must be [n_pos,B,S]")
    a.rot_dim, a.n_pos = 2 * freqs.shape[0], pos.shape[0]
    sections = [a.rot_dim // 2] if sections is None else [int(n) for n in sections]
    if len(sections) > MAX_POS_PLANES or len(sections) != a.n_pos:
        raise ValueError(f"sections must give the pairs of each of up to {MAX_POS_PLANES} planes")
    for i, n in enumerate(sections):
        a.section[i] = n
    a.interleaved, a.attn_factor = int(interleaved), attn_factor
    if inplace:
        q_out, k_out = q, k
        a.q_out_ld, a.k_out_ld = a.q_ld, a.k_ld
    else:
        q_out = _empty(q.shape, dt, dev)
        k_out = None if k is None else _empty(k.shape, dt, dev)
    a.freqs, a.pos, a.q, a.k = _ptr(freqs), _ptr(pos), _ptr(q), _ptr(k)
    a.q_out, a.k_out = _ptr(q_out), _ptr(k_out)
    return q_out, k_out


class Rope:
    """Rotary positions of query rows q [B,S,H_q,d] and, unless None, key rows
    k [B,S,H_k,d] at pos [n_pos,B,S] int64, with freqs [R/2] float64 on the
    device (rope_frequencies).  sections deals the R/2 pairs to the position
    planes (all to the first by default).  Outputs are allocated once, or are
    q and k themselves with inplace=True; call() enqueues the rotation and
    returns (q_out, k_out).  inverse=True turns back: the gradient of the
    rotation."""

    def __init__(self, q, k, pos, *, freqs, sections=None, interleaved=False, inverse=False,
                 attn_factor=1.0, inplace=False):
        self.device = q.device
        self.args = a = RopeArgs()
        self.q_out, self.k_out = _fill_rope(a, q, k, pos, freqs, sections, interleaved, attn_factor, inplace)
        a.inverse = int(inverse)
        self.inputs = (q, k, pos, freqs)

    def __call__(self, stream=None):
        _call(lib().trevs_rope, self.device, stream, ctypes.byref(self.args))
        return self.q_out, self.k_out


def rope(q, k, pos, stream=None, **kw):
    """Rotary positions: returns (q_out, k_out); see Rope."""
    return _one_off(stream, q.device, lambda: Rope(q, k, pos, **kw)(), q, k, pos, kw.get("freqs"))


class NormRope:
    """Rope after an RMS norm of every head: values over the root of their
    head's mean square (plus eps), times q_weight or k_weight (fp32 or bf16
    [d_head], or [H,d_head] for a weight a head; None: none) plus
    weight_offset.  The other arguments are those of Rope."""

    def __init__(self, q, k, pos, *, freqs, q_weight=None, k_weight=None, eps=1e-6, weight_offset=0.0,
                 sections=None, interleaved=False, attn_factor=1.0, inplace=False):
        self.device = dev = q.device
        self.args = a = NormRopeArgs()
        a.struct_size = ctypes.sizeof(NormRopeArgs)
        self.q_out, self.k_out = _fill_rope(a.rope, q, k, pos, freqs, sections, interleaved, attn_factor,
                                            inplace)
        if k is None and k_weight is not None:
            raise ValueError("k_weight without k")
        given = [(w, x, n) for w, x, n in ((q_weight, q, "q_weight"), (k_weight, k, "k_weight"))
                 if w is not None]
        for w, x, name in given:
            _check(w, name, dev, given[0][0].dim(), given[0][0].dtype)
            if w.shape not in (x.shape[3:], x.shape[2:]):
                raise ValueError(f"{name} must be [d_head] or [H,d_head]")
        if given:
            a.weight_dtype, a.per_head = _dtype_code(given[0][0]), given[0][0].dim() - 1
        a.eps, a.weight_offset = eps, weight_offset
        a.q_weight, a.k_weight = _ptr(q_weight), _ptr(k_weight)
        self.inputs = (q, k, pos, freqs, q_weight, k_weight)

    def __call__(self, stream=None):
        _call(lib().trevs_norm_rope, self.device, stream, ctypes.byref(self.args))
        return self.q_out, self.k_out


def norm_rope(q, k, pos, stream=None, **kw):
    """Norms of the heads, then rotary positions: returns (q_out, k_out); see NormRope."""
    return _one_off(stream, q.device, lambda: NormRope(q, k, pos, **kw)(), q, k, pos, kw.get("freqs"),
                    kw.get("q_weight"), kw.get("k_weight"))


class Kv8Cache:
    """A paged K/V cache of n_layers layers held in 8 bits (e4m3 values, one
    power-of-two scale for each page and KV head), empty at first:
      k, v              uint8 [n_layers,n_pages,H_kv,page_tokens,d_head] and
                        [n_layers,n_pages,H_kv,d_head,page_tokens]
      k_scale, v_scale  float32 [n_layers,n_pages,H_kv]
      table             int32 [n_slots,max_pages], the pages of each slot
      len, ref          int32 [n_slots], tokens; [n_pages], slots that hold a page
    """

    def __init__(self, *, n_pages, page_tokens, n_slots, max_pages, H_kv, d_head, n_layers=1,
                 device="cuda"):
        dev = torch.device(device)
        if dev.type != "cuda":
            raise ValueError("the cache lives on a GPU")
        if dev.index is None:
            dev = torch.device("cuda", torch.cuda.current_device())
        if min(n_pages, page_tokens, n_slots, max_pages, H_kv, d_head, n_layers) < 1:
            raise ValueError("every size of a cache is at least 1")
        self.device = dev
        self.k = _empty((n_layers, n_pages, H_kv, page_tokens, d_head), torch.uint8, dev)
        self.v = _empty((n_layers, n_pages, H_kv, d_head, page_tokens), torch.uint8, dev)
        self.k_scale = _empty((n_layers, n_pages, H_kv), torch.float32, dev)
        self.v_scale = _empty((n_layers, n_pages, H_kv), torch.float32, dev)
        self.table = _empty((n_slots, max_pages), torch.int32, dev)
        self.len = _empty((n_slots,), torch.int32, dev)
        self.ref = _empty((n_pages,), torch.int32, dev)
        for t in (self.k, self.v, self.k_scale, self.v_scale, self.len, self.ref):
            t.zero_()
        self.table.fill_(-1)
        self.tensors = (self.k, self.v, self.k_scale, self.v_scale, self.table, self.len, self.ref)
        a = Kv8CacheArgs()
        a.struct_size = ctypes.sizeof(Kv8CacheArgs)
        a.n_layers, a.n_pages, a.page_tokens, a.H_kv = n_layers, n_pages, page_tokens, H_kv
        a.d_head, a.n_slots, a.max_pages = d_head, n_slots, max_pages
        a.k, a.v, a.k_scale, a.v_scale = _ptr(self.k), _ptr(self.v), _ptr(self.k_scale), _ptr(self.v_scale)
        a.table, a.len, a.ref = _ptr(self.table), _ptr(self.len), _ptr(self.ref)
        self.args = a


class PagesReserve:
    """Room for n_new[i] more tokens in slots[i] (None: slot i): call() returns
    (granted, copy_src, copy_dst), int32 [n] on the device: n_new[i], or 0 where
    the pages did not suffice, and the shared page that Kv8Copy has to copy to
    the slot's own before rows are written, or -1."""

    def __init__(self, cache, n_new, slots=None):
        dev = cache.device
        _check(n_new, "n_new", dev, 1, torch.int32)
        n = n_new.shape[0]
        _check_list(slots, "slots", dev, n)
        self.cache, self.inputs, self.n = cache, (n_new, slots), n
        self.granted, self.copy_src, self.copy_dst = [_empty((n,), torch.int32, dev) for _ in range(3)]

    def __call__(self, stream=None):
        n_new, slots = self.inputs
        _call(lib().trevs_pages_reserve, self.cache.device, stream, ctypes.byref(self.cache.args), self.n,
              _ptr(slots), _ptr(n_new), _ptr(self.granted), _ptr(self.copy_src), _ptr(self.copy_dst))
        return self.granted, self.copy_src, self.copy_dst


def pages_reserve(cache, n_new, slots=None, stream=None):
    """Room for more tokens: returns (granted, copy_src, copy_dst); see PagesReserve."""
    return _one_off(stream, cache.device, lambda: PagesReserve(cache, n_new, slots)(), cache, n_new, slots)


class PagesFork:
    """Slot dst[i], empty before, shares the pages of the first n_tokens[i]
    tokens of slot src[i] (None: of all): call() returns done int32 [n], 1 or,
    where the request did nothing, 0."""

    def __init__(self, cache, src, dst, n_tokens=None):
        dev = cache.device
        _check(src, "src", dev, 1, torch.int32)
        n = src.shape[0]
        _check(dst, "dst", dev, 1, torch.int32)
        _check_list(dst, "dst", dev, n)
        _check_list(n_tokens, "n_tokens", dev, n)
        self.cache, self.inputs, self.n = cache, (src, dst, n_tokens), n
        self.done = _empty((n,), torch.int32, dev)

    def __call__(self, stream=None):
        src, dst, n_tokens = self.inputs
        _call(lib().trevs_pages_fork, self.cache.device, stream, ctypes.byref(self.cache.args), self.n,
              _ptr(src), _ptr(dst), _ptr(n_tokens), _ptr(self.done))
        return self.done


def pages_fork(cache, src, dst, n_tokens=None, stream=None):
    """Sequences that share another's pages: returns done; see PagesFork."""
    return _one_off(stream, cache.device, lambda: PagesFork(cache, src, dst, n_tokens)(), cache, src, dst,
                    n_tokens)


class PagesFree:
    """slots[i] (int32, device) keeps its first keep[i] tokens (None: none) and
    gives up its other pages."""

    def __init__(self, cache, slots, keep=None):
        _check(slots, "slots", cache.device, 1, torch.int32)
        _check_list(keep, "keep", cache.device, slots.shape[0])
        self.cache, self.inputs = cache, (slots, keep)

    def __call__(self, stream=None):
        slots, keep = self.inputs
        _call(lib().trevs_pages_free, self.cache.device, stream, ctypes.byref(self.cache.args),
              slots.shape[0], _ptr(slots), _ptr(keep))


def pages_free(cache, slots, keep=None, stream=None):
    """Pages given up; see PagesFree."""
    _one_off(stream, cache.device, lambda: PagesFree(cache, slots, keep)(), cache, slots, keep)


class Kv8Copy:
    """Pages src[i] copied to dst[i] in every layer; pairs with -1 are skipped."""

    def __init__(self, cache, src, dst):
        _check(src, "src", cache.device, 1, torch.int32)
        _check(dst, "dst", cache.device, 1, torch.int32)
        _check_list(dst, "dst", cache.device, src.shape[0])
        self.cache, self.inputs = cache, (src, dst)

    def __call__(self, stream=None):
        src, dst = self.inputs
        _call(lib().trevs_kv8_copy_pages, self.cache.device, stream, ctypes.byref(self.cache.args),
              src.shape[0], _ptr(src), _ptr(dst))


def kv8_copy(cache, src, dst, stream=None):
    """Pages copied in every layer; see Kv8Copy."""
    _one_off(stream, cache.device, lambda: Kv8Copy(cache, src, dst)(), cache, src, dst)


class Kv8Write:
    """Key and value rows k, v [B,T,H_kv,d] (fp32 or bf16) written as the last
    n_new[b] tokens (None: T) of slots[b] (None: slot b) in one layer, their
    room reserved before."""

    def __init__(self, cache, k, v, n_new=None, slots=None, *, layer=0):
        dev, dt = cache.device, k.dtype
        a = Kv8WriteArgs()
        a.struct_size = ctypes.sizeof(Kv8WriteArgs)
        a.dtype = _dtype_code(k)
        a.k_ld, a.v_ld = _row_ld(k, "k", dev, dt), _row_ld(v, "v", dev, dt)
        if v.shape != k.shape or k.shape[2:] != (cache.args.H_kv, cache.args.d_head):
            raise ValueError("k and v must be [B,T,H_kv,d_head] of the cache")
        a.B, a.T_max, a.layer = k.shape[0], k.shape[1], layer
        _check_list(n_new, "n_new", dev, a.B)
        _check_list(slots, "slots", dev, a.B)
        a.k, a.v, a.n_new, a.slots = _ptr(k), _ptr(v), _ptr(n_new), _ptr(slots)
        self.cache, self.inputs, self.args = cache, (k, v, n_new, slots), a

    def __call__(self, stream=None):
        _call(lib().trevs_kv8_write, self.cache.device, stream, ctypes.byref(self.cache.args),
              ctypes.byref(self.args))


def kv8_write(cache, k, v, n_new=None, slots=None, stream=None, **kw):
    """Rows written to the cache; see Kv8Write."""
    _one_off(stream, cache.device, lambda: Kv8Write(cache, k, v, n_new, slots, **kw)(), cache, k, v, n_new,
             slots)


class Kv8Attention:
    """Attention of query rows q [B,T,H_q,d] over one layer of the cache: the
    first q_len[b] rows (None: T) of slots[b] (None: slot b), with causal=True
    as the sequence's last ones, else over all its tokens.  kv_max bounds the
    lengths of the call (0: what the cache can hold).  Output, workspace and,
    with want_lse, the log-sum-exp of the logits [B,H_q,T] are allocated once;
    call() enqueues and returns the output [B,T,H_q,d].  Rows past q_len[b] are
    not written."""

    def __init__(self, cache, q, q_len=None, slots=None, *, layer=0, causal=True, scale=None, kv_max=0,
                 want_lse=False):
        dev, dt = cache.device, q.dtype
        a = Kv8AttentionArgs()
        a.struct_size = ctypes.sizeof(Kv8AttentionArgs)
        a.dtype = _dtype_code(q)
        a.q_ld = _row_ld(q, "q", dev, dt)
        if q.shape[3] != cache.args.d_head:
            raise ValueError("q must be [B,T,H_q,d_head] of the cache")
        a.B, a.T_max, a.H_q, _ = q.shape
        _check_list(q_len, "q_len", dev, a.B)
        _check_list(slots, "slots", dev, a.B)
        a.layer, a.causal, a.kv_max = layer, int(causal), kv_max
        a.scale = float(scale) if scale is not None else q.shape[3] ** -0.5
        self.out = _empty(q.shape, dt, dev)
        self.lse = _empty((a.B, a.H_q, a.T_max), torch.float32, dev) if want_lse else None
        a.q, a.q_len, a.slots = _ptr(q), _ptr(q_len), _ptr(slots)
        a.out, a.lse = _ptr(self.out), _ptr(self.lse)
        self.cache, self.inputs, self.args = cache, (q, q_len, slots), a
        ws = lib().trevs_kv8_attention_workspace_size(ctypes.byref(cache.args), ctypes.byref(a))
        if ws == 0:
            st = lib().trevs_kv8_attention(ctypes.byref(cache.args), ctypes.byref(a), None, 0, None)
            raise TrevsError(st, "trevs_kv8_attention")
        self.workspace = _empty((ws,), torch.uint8, dev)

    def __call__(self, stream=None):
        _call(lib().trevs_kv8_attention, self.cache.device, stream, ctypes.byref(self.cache.args),
              ctypes.byref(self.args), self.workspace.data_ptr(), self.workspace.numel())
        return self.out


def kv8_attention(cache, q, q_len=None, slots=None, stream=None, **kw):
    """Attention over the cache: returns out, or (out, lse) with want_lse=True;
    see Kv8Attention."""

    def run():
        call = Kv8Attention(cache, q, q_len, slots, **kw)
        out = call()
        return (out, call.lse) if kw.get("want_lse") else out

    return _one_off(stream, cache.device, run, cache, q, q_len, slots)


class Kv8Compact:
    """Stage 2's compaction inside the cache, in every layer: rows [0,P) ++
    (P + kept_idx[b]) ++ [P+K_in, len) of slot src_slots[b] become the tokens of
    slot dst_slots[b], whose room is reserved before."""

    def __init__(self, cache, kept_idx, src_slots, dst_slots, *, P, K_in):
        dev = cache.device
        _check(kept_idx, "kept_idx", dev, 2, torch.int32)
        for t, name in ((src_slots, "src_slots"), (dst_slots, "dst_slots")):
            _check(t, name, dev, 1, torch.int32)
            _check_list(t, name, dev, kept_idx.shape[0])
        a = Kv8CompactArgs()
        a.struct_size = ctypes.sizeof(Kv8CompactArgs)
        a.B, a.n_kept = kept_idx.shape
        a.P, a.K_in = P, K_in
        a.kept_idx, a.src_slots, a.dst_slots = _ptr(kept_idx), _ptr(src_slots), _ptr(dst_slots)
        self.cache, self.inputs, self.args = cache, (kept_idx, src_slots, dst_slots), a

    def __call__(self, stream=None):
        _call(lib().trevs_kv8_compact, self.cache.device, stream, ctypes.byref(self.cache.args),
              ctypes.byref(self.args))


def kv8_compact(cache, kept_idx, src_slots, dst_slots, stream=None, **kw):
    """Kept rows of cached sequences moved together; see Kv8Compact."""
    _one_off(stream, cache.device, lambda: Kv8Compact(cache, kept_idx, src_slots, dst_slots, **kw)(),
             cache, kept_idx, src_slots, dst_slots)


def kv8_scores(cache):
    """Scores of a cache's tokens for Kv8Weights: zeros, float32 [n_slots,
    max_pages * page_tokens]."""
    a = cache.args
    return _empty((a.n_slots, a.max_pages * a.page_tokens), torch.float32, cache.device).zero_()


def _check_scores(cache, score):
    _check(score, "score", cache.device, 2, torch.float32)
    if score.shape != (cache.args.n_slots, cache.args.max_pages * cache.args.page_tokens):
        raise ValueError("score must be [n_slots, max_pages * page_tokens] of the cache")


class Kv8Weights:
    """The attention weights that query rows q [B,T,H_q,d] give to the cached
    tokens of one layer, summed over rows and heads and added to decay * score,
    in place.  lse [B,H_q,T] is Kv8Attention's for the same q, q_len, slots,
    layer, causal, scale and kv_max; slots name no slot twice.  decay=0 begins
    a slot's scores anew (PagesFork and PagesFree leave them alone: copy a
    fork's, and zero those of tokens given up).  call() enqueues and returns
    score."""

    def __init__(self, cache, q, lse, score, q_len=None, slots=None, *, layer=0, causal=True, scale=None,
                 kv_max=0, decay=1.0):
        dev, dt = cache.device, q.dtype
        a = Kv8WeightsArgs()
        a.struct_size = ctypes.sizeof(Kv8WeightsArgs)
        a.dtype = _dtype_code(q)
        a.q_ld = _row_ld(q, "q", dev, dt)
        if q.shape[3] != cache.args.d_head:
            raise ValueError("q must be [B,T,H_q,d_head] of the cache")
        a.B, a.T_max, a.H_q, _ = q.shape
        _check(lse, "lse", dev, 3, torch.float32)
        if lse.shape != (a.B, a.H_q, a.T_max):
            raise ValueError("lse must be [B,H_q,T]")
        _check_scores(cache, score)
        _check_list(q_len, "q_len", dev, a.B)
        _check_list(slots, "slots", dev, a.B)
        a.layer, a.causal, a.kv_max, a.decay = layer, int(causal), kv_max, decay
        a.scale = float(scale) if scale is not None else q.shape[3] ** -0.5
        a.q, a.q_len, a.slots = _ptr(q), _ptr(q_len), _ptr(slots)
        a.lse, a.score = _ptr(lse), _ptr(score)
        self.cache, self.inputs, self.args, self.score = cache, (q, lse, q_len, slots), a, score
        ws = lib().trevs_kv8_weights_workspace_size(ctypes.byref(cache.args), ctypes.byref(a))
        if ws == 0:
            st = lib().trevs_kv8_weights(ctypes.byref(cache.args), ctypes.byref(a), None, 0, None)
            raise TrevsError(st, "trevs_kv8_weights")
        self.workspace = _empty((ws,), torch.uint8, dev)

    def __call__(self, stream=None):
        _call(lib().trevs_kv8_weights, self.cache.device, stream, ctypes.byref(self.cache.args),
              ctypes.byref(self.args), self.workspace.data_ptr(), self.workspace.numel())
        return self.score


def kv8_weights(cache, q, lse, score, q_len=None, slots=None, stream=None, **kw):
    """Attention weights added to the tokens' scores: returns score; see Kv8Weights."""
    return _one_off(stream, cache.device, lambda: Kv8Weights(cache, q, lse, score, q_len, slots, **kw)(),
                    cache, q, lse, score, q_len, slots)


class Kv8Evict:
    """Sequences of slots (None: slots 0..B-1, B given by keep or by `n`; else
    all) cut to n_keep tokens each, or keep[b] of them: the first n_first, the
    last n_last, and those of the highest scores between, in their order, in
    every layer.  Tables, lengths, counts and scores follow.  call() returns
    (n_evicted [B], kept_idx [B,n_keep]): how many tokens went (0: the sequence
    is short enough, or the free pages did not suffice), and the places that the
    kept ones had, -1 past them or where nothing went.  Kept tokens move to pages
    that are free before the call, up to n_keep tokens' a sequence: evict while
    there is that room."""

    def __init__(self, cache, score, slots=None, *, n_keep, n_first=0, n_last=0, keep=None, n=None):
        dev = cache.device
        _check_scores(cache, score)
        a = Kv8EvictArgs()
        a.struct_size = ctypes.sizeof(Kv8EvictArgs)
        given = [t.shape[0] for t in (slots, keep) if isinstance(t, torch.Tensor) and t.dim() == 1]
        a.B = given[0] if given else cache.args.n_slots if n is None else n
        if n is not None and a.B != n:
            raise ValueError("n differs from the lists' length")
        _check_list(slots, "slots", dev, a.B)
        _check_list(keep, "keep", dev, a.B)
        a.n_keep, a.n_first, a.n_last = n_keep, n_first, n_last
        if a.B < 1 or n_keep < 1:
            raise TrevsError(1, "trevs_kv8_evict")
        self.n_evicted = _empty((a.B,), torch.int32, dev)
        self.kept_idx = _empty((a.B, n_keep), torch.int32, dev)
        a.keep, a.slots, a.score = _ptr(keep), _ptr(slots), _ptr(score)
        a.n_evicted, a.kept_idx = _ptr(self.n_evicted), _ptr(self.kept_idx)
        self.cache, self.inputs, self.args = cache, (score, slots, keep), a
        ws = lib().trevs_kv8_evict_workspace_size(ctypes.byref(cache.args), ctypes.byref(a))
        if ws == 0:
            st = lib().trevs_kv8_evict(ctypes.byref(cache.args), ctypes.byref(a), None, 0, None)
            raise TrevsError(st, "trevs_kv8_evict")
        self.workspace = _empty((ws,), torch.uint8, dev)

    def __call__(self, stream=None):
        _call(lib().trevs_kv8_evict, self.cache.device, stream, ctypes.byref(self.cache.args),
              ctypes.byref(self.args), self.workspace.data_ptr(), self.workspace.numel())
        return self.n_evicted, self.kept_idx


def kv8_evict(cache, score, slots=None, stream=None, **kw):
    """Sequences cut to their best tokens: returns (n_evicted, kept_idx); see Kv8Evict."""
    return _one_off(stream, cache.device, lambda: Kv8Evict(cache, score, slots, **kw)(), cache, score, slots,
                    kw.get("keep"))


# --------------------------------------------------------------- beam search
class BeamSelect:
    """The n_out best continuations of each sequence over its beams and the
    vocabulary: logits [B,W,V] (fp32 or bf16; rows evenly spaced), score [B,W]
    float32, the beams' summed log probabilities; done [B,W] int32 or None:
    beams that go on by the token eos alone, with their score.  call() returns
    (score [B,n_out] float32, parent, token [B,n_out] int32), best first, ties
    to the lower beam and token; (-inf, -1, -1) where there are fewer."""

    def __init__(self, logits, score, done=None, *, n_out, eos=0):
        if not isinstance(logits, torch.Tensor) or logits.dim() != 3 or min(logits.shape) < 1:
            raise ValueError("logits must be a non-empty [B,W,V] tensor")
        self.device = dev = logits.device
        if dev.type != "cuda":
            raise ValueError("logits must be on a GPU")
        B, W, V = logits.shape
        sb, sw, sv = logits.stride()
        ld = sw if W > 1 else sb if B > 1 else V
        if (V > 1 and sv != 1) or (B > 1 and sb != W * ld) or ld < V:
            raise ValueError("logits must have dense, evenly spaced rows")
        _check(score, "score", dev, 2, torch.float32)
        if done is not None:
            _check(done, "done", dev, 2, torch.int32)
        if score.shape != (B, W) or (done is not None and done.shape != (B, W)):
            raise ValueError("score and done must be [B,W]")
        a = BeamSelectArgs()
        a.struct_size = ctypes.sizeof(BeamSelectArgs)
        a.B, a.W, a.V, a.n_out, a.eos = B, W, V, n_out, eos
        a.dtype, a.logits_ld = _dtype_code(logits), ld
        if n_out < 1:
            raise TrevsError(1, "trevs_beam_select")
        self.score_out = _empty((B, n_out), torch.float32, dev)
        self.parent, self.token = [_empty((B, n_out), torch.int32, dev) for _ in range(2)]
        a.logits, a.score, a.done = _ptr(logits), _ptr(score), _ptr(done)
        a.score_out, a.parent, a.token = _ptr(self.score_out), _ptr(self.parent), _ptr(self.token)
        self.inputs, self.args = (logits, score, done), a
        ws = lib().trevs_beam_select_workspace_size(ctypes.byref(a))
        if ws == 0:
            raise TrevsError(lib().trevs_beam_select(ctypes.byref(a), None, 0, None), "trevs_beam_select")
        self.workspace = _empty((ws,), torch.uint8, dev)

    def __call__(self, stream=None):
        _call(lib().trevs_beam_select, self.device, stream, ctypes.byref(self.args),
              self.workspace.data_ptr(), self.workspace.numel())
        return self.score_out, self.parent, self.token


def beam_select(logits, score, done=None, stream=None, **kw):
    """Beam search's selection: returns (score, parent, token); see BeamSelect."""
    return _one_off(stream, logits.device, lambda: BeamSelect(logits, score, done, **kw)(), logits, score,
                    done)


class PagesReorder:
    """The beams' sequences after a selection: slots[g * W + w] (int32, None:
    slot g * W + w) takes over the pages and length that the slot of beam
    parent[g, w] of its group had before, for all of parent [n_groups,W] int32
    at once; with score (Kv8Weights'), the scores too.  No page is copied:
    PagesReserve and Kv8Copy give beams that share a last page their own."""

    def __init__(self, cache, parent, slots=None, *, score=None):
        dev = cache.device
        _check(parent, "parent", dev, 2, torch.int32)
        _check_list(slots, "slots", dev, parent.numel())
        if score is not None:
            _check_scores(cache, score)
        self.cache, self.inputs = cache, (parent, slots, score)

    def __call__(self, stream=None):
        parent, slots, score = self.inputs
        _call(lib().trevs_pages_reorder, self.cache.device, stream, ctypes.byref(self.cache.args),
              parent.shape[0], parent.shape[1], _ptr(slots), _ptr(parent), _ptr(score))


def pages_reorder(cache, parent, slots=None, stream=None, **kw):
    """Sequences taken over from the beams' parents; see PagesReorder."""
    _one_off(stream, cache.device, lambda: PagesReorder(cache, parent, slots, **kw)(), cache, parent, slots,
             kw.get("score"))


# ---------------------------------------------------------------- HIP events
HIP_EVENT_DISABLE_SYSTEM_FENCE = 0x20000000  # hipEventDisableSystemFence


class HipEvents:
    """A pool of hipEvent_t handles created through the HIP runtime that torch
    has already loaded, for the per-kernel event slots of the entry points.

    The events serve timing only, so they are created without the
    system-scope release fence (hipEventDisableSystemFence): a fenced record
    between two kernels writes back and invalidates the caches, which adds
    several microseconds to the work it brackets.  Read the times only after
    a device or stream synchronisation."""

    def __init__(self, n):
        self.rt = ctypes.CDLL("libamdhip64.so")
        self.rt.hipEventCreateWithFlags.argtypes = [ctypes.POINTER(c_void_p), ctypes.c_uint]
        self.rt.hipEventElapsedTime.argtypes = [ctypes.POINTER(ctypes.c_float), c_void_p, c_void_p]
        self.rt.hipEventDestroy.argtypes = [c_void_p]
        self.rt.hipEventRecord.argtypes = [c_void_p, c_void_p]
        self.handles = []
        for _ in range(n):
            h = c_void_p()
            if self.rt.hipEventCreateWithFlags(ctypes.byref(h), HIP_EVENT_DISABLE_SYSTEM_FENCE):
                raise RuntimeError("hipEventCreateWithFlags failed")
            self.handles.append(h.value)

    def record(self, i, stream=None):
        """Record event i on the stream (torch's current stream by default)."""
        if self.rt.hipEventRecord(self.handles[i], _stream(stream)):
            raise RuntimeError("hipEventRecord failed")

    def elapsed_ms(self, i, j):
        ms = ctypes.c_float()
        if self.rt.hipEventElapsedTime(ctypes.byref(ms), self.handles[i], self.handles[j]):
            raise RuntimeError("hipEventElapsedTime failed")
        return ms.value

    def close(self):
        for h in self.handles:
            self.rt.hipEventDestroy(h)
        self.handles = []
