"""ctypes binding of libss_msa.so: the same entry points as include/ss_msa.h.

Argument marshalling only: every step of the path runs in the CUDA library.  PyTorch is used for
device memory and streams.  There is no fallback: if the library is missing or cannot be loaded
this module raises, it never computes anything itself.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence

import numpy as np
import torch

SS_MAX_NODES = 64
SS_MAX_GAMMA = 4
SS_PATH_STRIDE = SS_MAX_NODES

SS_OK = 0
SS_ERR_INVALID_ARG = -1
SS_ERR_BAD_TREE = -2
SS_ERR_UNSUPPORTED = -3
SS_ERR_WORKSPACE = -4
SS_ERR_CAPACITY = -5
SS_ERR_CUDA = -6
SS_ERR_DEVICE_TIMEOUT = -7

SS_ATTN_PREFIX_STABLE = 1

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libss_msa.so")
_lib = None
_native = None          # the _pycall module: takes the tensors of the per-step calls apart (see native())
_NATIVE_CALLS = ("ss_msa_attention", "ss_tree_verify", "ss_tree_verify_soft", "ss_tree_verify_sampled", "ss_tree_prune", "ss_next_draft",
                 "ss_kv_compact", "ss_stream_insert", "ss_value_rotate", "ss_msa_attention_kvq", "ss_kvq_write",
                 "ss_kvq_read")                                                 # in the order of _pycall.setup

# number of kernels each entry point enqueues per call (for launch accounting in the benchmark); ss_kv_compact enqueues a
# second one where kv_len_out overlaps one of its inputs, as does ss_kvq_write
LAUNCHES_PER_CALL = {"ss_msa_attention": 1, "ss_tree_verify": 1, "ss_kv_compact": 1, "ss_next_draft": 1,
                     "ss_tree_prune": 1, "ss_tree_verify_soft": 1, "ss_tree_verify_sampled": 1, "ss_stream_insert": 1,
                     "ss_value_rotate": 1, "ss_msa_attention_kvq": 1, "ss_kvq_write": 1, "ss_kvq_read": 1}


class SsError(RuntimeError):
    def __init__(self, what: str, status: int):
        self.status = status
        msg = lib().ss_error_string(C.c_int32(status)).decode() if _lib is not None else "?"
        super().__init__("%s failed: status %d (%s)" % (what, status, msg))


class TreeDesc(C.Structure):
    _fields_ = [("n_nodes", C.c_int32), ("gamma", C.c_int32), ("max_depth", C.c_int32), ("reserved", C.c_int32),
                ("parent", C.c_int32 * SS_MAX_NODES), ("depth", C.c_int32 * SS_MAX_NODES),
                ("anc_mask", C.c_uint64 * SS_MAX_NODES)]


class AttnParams(C.Structure):
    _fields_ = [("batch", C.c_int32), ("n_heads", C.c_int32), ("head_dim", C.c_int32), ("gamma", C.c_int32),
                ("max_nodes", C.c_int32), ("sm_scale", C.c_float),
                ("q_main", C.c_void_p), ("o_main", C.c_void_p), ("q_spec", C.c_void_p), ("k_spec", C.c_void_p),
                ("v_spec", C.c_void_p), ("o_spec", C.c_void_p), ("k_cache", C.c_void_p), ("v_cache", C.c_void_p),
                ("kv_slot_stride", C.c_int64), ("kv_head_stride", C.c_int64), ("kv_total_slots", C.c_int64),
                ("kv_start", C.c_void_p), ("kv_len", C.c_void_p), ("kv_capacity", C.c_void_p),
                ("trees", C.c_void_p), ("lse_main", C.c_void_p), ("lse_spec", C.c_void_p),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t), ("flags", C.c_uint32)]


class CacheLayout(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("n_heads", C.c_int32), ("head_dim", C.c_int32), ("reserved", C.c_int32),
                ("layer_stride", C.c_int64), ("slot_stride", C.c_int64), ("head_stride", C.c_int64)]


class KvqCache(C.Structure):
    """A cache in 4 bits (ss_kvq_cache); make_kvq_cache and empty_kvq_cache keep its tensors with it."""
    _fields_ = [("n_layers", C.c_int32), ("n_heads", C.c_int32), ("head_dim", C.c_int32), ("device", C.c_int32),
                ("k_codes", C.c_void_p), ("v_codes", C.c_void_p), ("k_params", C.c_void_p), ("v_params", C.c_void_p),
                ("layer_stride", C.c_int64), ("slot_stride", C.c_int64), ("head_stride", C.c_int64),
                ("param_layer_stride", C.c_int64), ("param_slot_stride", C.c_int64), ("param_head_stride", C.c_int64),
                ("total_slots", C.c_int64)]


class KvqAttnParams(C.Structure):
    _fields_ = [("batch", C.c_int32), ("gamma", C.c_int32), ("max_nodes", C.c_int32), ("layer", C.c_int32), ("sm_scale", C.c_float),
                ("q_main", C.c_void_p), ("o_main", C.c_void_p), ("k_tree", C.c_void_p), ("v_tree", C.c_void_p),
                ("q_spec", C.c_void_p), ("k_spec", C.c_void_p), ("v_spec", C.c_void_p), ("o_spec", C.c_void_p),
                ("cache", KvqCache), ("kv_start", C.c_void_p), ("kv_len", C.c_void_p), ("kv_capacity", C.c_void_p),
                ("trees", C.c_void_p), ("lse_main", C.c_void_p), ("lse_spec", C.c_void_p),
                ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)]


EXPORTS = ("ss_tree_build", "ss_msa_attention_workspace_bytes", "ss_msa_attention",
           "ss_tree_verify_workspace_bytes", "ss_tree_verify", "ss_tree_verify_static", "ss_kv_compact", "ss_status",
           "ss_version", "ss_error_string",
           "ss_next_draft_workspace_bytes", "ss_next_draft", "ss_tree_prune_workspace_bytes", "ss_tree_prune",
           "ss_tree_verify_soft", "ss_tree_verify_sampled_workspace_bytes", "ss_tree_verify_sampled",
           "ss_stream_insert", "ss_value_rotate", "ss_wait_selftest",
           "ss_kvq_write", "ss_kvq_read", "ss_msa_attention_kvq_workspace_bytes", "ss_msa_attention_kvq")
SS_MAX_TOPK = 8
SS_VERIFY_STATIC_SCRATCH_BYTES = 1 << 20


def lib() -> C.CDLL:
    """Loads libss_msa.so (built in-tree by paper_2402_11131_b200.build).  Raises if it is missing."""
    global _lib, _native
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError("CUDA library %s is missing: run `python -m paper_2402_11131_b200.build` "
                               "(there is no CPU fallback)" % _LIB_PATH)
        l = C.CDLL(_LIB_PATH)
        l.ss_tree_build.restype = C.c_int32
        l.ss_tree_build.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.POINTER(TreeDesc)]
        l.ss_msa_attention_workspace_bytes.restype = C.c_size_t
        l.ss_msa_attention_workspace_bytes.argtypes = [C.POINTER(AttnParams)]
        l.ss_msa_attention.restype = C.c_int32
        l.ss_msa_attention.argtypes = [C.POINTER(AttnParams), C.c_void_p]
        l.ss_tree_verify_workspace_bytes.restype = C.c_size_t
        l.ss_tree_verify_workspace_bytes.argtypes = [C.c_int32, C.c_int32, C.c_int32]
        l.ss_tree_verify.restype = C.c_int32
        l.ss_tree_verify.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32,
                                     C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                     C.c_size_t, C.c_void_p]
        l.ss_tree_verify_static.restype = C.c_int32
        l.ss_tree_verify_static.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32, C.c_int32, C.c_int32,
                                            C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        l.ss_kv_compact.restype = C.c_int32
        l.ss_kv_compact.argtypes = [C.c_void_p, C.c_void_p, C.POINTER(CacheLayout), C.c_int32, C.c_void_p,
                                    C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        vp, i32, f32 = C.c_void_p, C.c_int32, C.c_float
        for name in ("ss_next_draft_workspace_bytes", "ss_tree_prune_workspace_bytes", "ss_tree_verify_sampled_workspace_bytes"):
            getattr(l, name).restype = C.c_size_t
            getattr(l, name).argtypes = [i32, i32, i32]
        l.ss_next_draft.restype = i32
        l.ss_next_draft.argtypes = [vp, i32, vp, vp, i32, i32, i32, i32, i32, vp, vp, vp, C.c_size_t, vp]
        l.ss_tree_prune.restype = i32
        l.ss_tree_prune.argtypes = [vp, vp, vp, i32, i32, i32, f32, vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
        l.ss_tree_verify_soft.restype = i32
        l.ss_tree_verify_soft.argtypes = [vp, vp, vp, i32, i32, i32, f32, f32, vp, vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
        l.ss_tree_verify_sampled.restype = i32
        l.ss_tree_verify_sampled.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, C.c_size_t, vp]
        l.ss_stream_insert.restype = i32
        l.ss_stream_insert.argtypes = [vp, vp, vp, C.c_int64, i32, i32, vp]
        l.ss_value_rotate.restype = i32
        l.ss_value_rotate.argtypes = [vp, vp, C.c_int64, i32, i32, f32, vp]
        l.ss_kvq_write.restype = l.ss_kvq_read.restype = l.ss_msa_attention_kvq.restype = i32
        l.ss_kvq_write.argtypes = [vp, C.POINTER(KvqCache)] + [vp] * 8
        l.ss_kvq_read.argtypes = [C.POINTER(KvqCache)] + [vp] * 5
        l.ss_msa_attention_kvq_workspace_bytes.restype = C.c_size_t
        l.ss_msa_attention_kvq_workspace_bytes.argtypes = [C.POINTER(KvqAttnParams)]
        l.ss_msa_attention_kvq.argtypes = [C.POINTER(KvqAttnParams), vp]
        l.ss_wait_selftest.restype = C.c_int32
        l.ss_wait_selftest.argtypes = [C.c_void_p, C.c_size_t, C.c_void_p]
        l.ss_status.restype = C.c_int32
        l.ss_status.argtypes = [C.c_void_p, C.c_void_p, C.POINTER(C.c_int32)]
        l.ss_version.restype = C.c_int32
        l.ss_error_string.restype = C.c_char_p
        l.ss_error_string.argtypes = [C.c_int32]
        _lib, _native = l, None                           # (the native part takes the new library's addresses)
    return _lib


def native():
    """The CPython side of the binding, for the calls of a decode step: pointers, sizes and the current stream are collected
    in C (1 us of a call that costs 3 us through ctypes).  Raises like lib() if it has not been built."""
    global _native
    if _native is None:
        lib()
        try:
            from . import _pycall
        except ImportError as e:
            raise RuntimeError("the binding's native part is missing: run `python -m paper_2402_11131_b200.build`") from e
        if torch.cuda.is_available():
            torch.cuda.current_stream()                   # initialises CUDA if nothing has yet
        addresses = tuple(C.cast(getattr(lib(), name), C.c_void_p).value for name in _NATIVE_CALLS)
        _pycall.setup(SsError, torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice, AttnParams, CacheLayout, C.byref,
                      C.ArgumentError, addresses, KvqAttnParams, KvqCache, torch.int32, torch.int64, torch.bfloat16)
        _native = _pycall
    return _native


def _check(status: int, what: str) -> None:
    if status != SS_OK:
        raise SsError(what, status)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream: Optional[torch.cuda.Stream]) -> Optional[int]:
    s = torch.cuda.current_stream() if stream is None else stream
    return s.cuda_stream or None


# ---- host ---------------------------------------------------------------------------------------
def ss_tree_build(parent: Sequence[int], gamma: int) -> TreeDesc:
    """Host-side descriptor of one tree (depth, ancestor bit masks) from its parent array."""
    par = np.ascontiguousarray(parent, dtype=np.int32)
    out = TreeDesc()
    _check(lib().ss_tree_build(par.ctypes.data, C.c_int32(par.shape[0]), C.c_int32(gamma), C.byref(out)),
           "ss_tree_build")
    return out


def trees_to_device(descs: Sequence[TreeDesc], device="cuda") -> torch.Tensor:
    """Packs descriptors into one device byte tensor (the `trees` argument of the device calls)."""
    raw = b"".join(bytes(d) for d in descs)
    host = torch.frombuffer(bytearray(raw), dtype=torch.uint8)
    return host.to(device)


def workspace(n_bytes: int, device="cuda") -> torch.Tensor:
    """A zero-filled workspace of at least n_bytes (256-byte granularity)."""
    return torch.zeros((int(n_bytes) + 255) // 256 * 256, dtype=torch.uint8, device=device)


# ---- device -------------------------------------------------------------------------------------
def make_attn_params(*, q_main, o_main, k_cache, v_cache, kv_start, kv_len, trees, gamma, sm_scale,
                     q_spec=None, k_spec=None, v_spec=None, o_spec=None, kv_capacity=None, lse_main=None,
                     lse_spec=None, workspace=None, prefix_stable=False) -> AttnParams:
    """Fills ss_attn_params from tensors.  q_main/o_main: bf16 [B][Tmax][H][d]; *_spec: bf16
    [B][Tmax][gamma][H][d]; k_cache/v_cache: bf16 [slots][H][d] (any slot/head stride, d contiguous)."""
    B, Tmax, H, d = q_main.shape
    assert k_cache.dim() == 3 and k_cache.stride(2) == 1 and k_cache.stride() == v_cache.stride()
    p = AttnParams()
    p.batch, p.n_heads, p.head_dim, p.gamma, p.max_nodes = B, H, d, int(gamma), Tmax
    p.sm_scale = float(sm_scale)
    p.q_main, p.o_main = _ptr(q_main), _ptr(o_main)
    p.q_spec, p.k_spec, p.v_spec, p.o_spec = _ptr(q_spec), _ptr(k_spec), _ptr(v_spec), _ptr(o_spec)
    p.k_cache, p.v_cache = _ptr(k_cache), _ptr(v_cache)
    p.kv_slot_stride, p.kv_head_stride, p.kv_total_slots = k_cache.stride(0), k_cache.stride(1), k_cache.shape[0]
    p.kv_start, p.kv_len, p.kv_capacity = _ptr(kv_start), _ptr(kv_len), _ptr(kv_capacity)
    p.trees = _ptr(trees)
    p.lse_main, p.lse_spec = _ptr(lse_main), _ptr(lse_spec)
    p.workspace = _ptr(workspace)
    p.workspace_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    p.flags = SS_ATTN_PREFIX_STABLE if prefix_stable else 0
    return p


def ss_msa_attention_workspace_bytes(p: AttnParams) -> int:
    return int(lib().ss_msa_attention_workspace_bytes(C.byref(p)))


def ss_msa_attention(p: AttnParams, stream: Optional[torch.cuda.Stream] = None) -> None:
    """One layer of tree-masked multi-stream attention (asynchronous on `stream`)."""
    (_native or native()).msa_attention(p, stream)


def ss_tree_verify_workspace_bytes(batch: int, max_nodes: int, vocab: int) -> int:
    return int(lib().ss_tree_verify_workspace_bytes(batch, max_nodes, vocab))


def ss_tree_verify(logits, draft_tokens, trees, accept_len, accept_path, last_node, bonus_token,
                   node_argmax, workspace, stream=None) -> None:
    """Greedy verification.  logits f32 [B][Tmax][V]; the int32 outputs are written on the device."""
    (_native or native()).tree_verify(logits, draft_tokens, trees, accept_len, accept_path, last_node, bonus_token, node_argmax,
                                      workspace, stream)


def ss_tree_verify_static(logits, draft_tokens, trees, accept_len, accept_path, last_node, bonus_token,
                          node_argmax, stream=None) -> None:
    """ss_tree_verify for callers that cannot supply scratch memory (no allocator of their own, or
    allocation forbidden where they call): the scratch is a fixed array inside the library, shared
    by every call on the device, so overlapping calls race.  Raises SsError(SS_ERR_WORKSPACE) when
    the sizes need more than SS_VERIFY_STATIC_SCRATCH_BYTES.  Make the first call on a device
    outside any stream capture."""
    B, Tmax, V = logits.shape
    _check(lib().ss_tree_verify_static(_ptr(logits), _ptr(draft_tokens), _ptr(trees), B, Tmax, V,
                                       _ptr(accept_len), _ptr(accept_path), _ptr(last_node), _ptr(bonus_token),
                                       _ptr(node_argmax), _stream(stream)), "ss_tree_verify_static")


def empty_trees(batch: int, device="cuda") -> torch.Tensor:
    """Device storage for `batch` tree descriptors (written by ss_next_draft / ss_tree_prune)."""
    return torch.zeros(batch * C.sizeof(TreeDesc), dtype=torch.uint8, device=device)


def trees_from_device(trees: torch.Tensor):
    """Descriptors back on the host (tests)."""
    raw = trees.cpu().numpy().tobytes()
    n = len(raw) // C.sizeof(TreeDesc)
    return [TreeDesc.from_buffer_copy(raw[i * C.sizeof(TreeDesc):(i + 1) * C.sizeof(TreeDesc)]) for i in range(n)]


def ss_next_draft_workspace_bytes(batch: int, gamma: int, vocab: int) -> int:
    return int(lib().ss_next_draft_workspace_bytes(batch, gamma, vocab))


def ss_next_draft(stream_logits, row_index, bonus_token, top_k: int, max_nodes: int, draft_tokens, trees, workspace,
                  stream=None) -> None:
    """Next tree draft.  stream_logits f32 [B][n_rows][gamma][V]; row_index int32 [B] or None; bonus_token int32 [B];
    draft_tokens int32 [B][max_nodes] and trees (empty_trees(B)) are written on the device."""
    (_native or native()).next_draft(stream_logits, row_index, bonus_token, int(top_k), int(max_nodes), draft_tokens, trees,
                                     workspace, stream)


def ss_tree_prune_workspace_bytes(batch: int, max_nodes: int, vocab: int) -> int:
    return int(lib().ss_tree_prune_workspace_bytes(batch, max_nodes, vocab))


def ss_tree_prune(exit_logits, draft_tokens, trees, threshold: float, edge_prob, new_index, kept_nodes, kept_tokens,
                  pruned_trees, workspace, stream=None) -> None:
    """Parallel tree pruning.  exit_logits f32 [B][Tmax][V]; outputs are written on the device."""
    (_native or native()).tree_prune(exit_logits, draft_tokens, trees, threshold, edge_prob, new_index, kept_nodes, kept_tokens,
                                     pruned_trees, workspace, stream)


def ss_tree_verify_soft(logits, draft_tokens, trees, eps: float, delta: float, accept_len, accept_path, last_node,
                        bonus_token, edge_prob, node_entropy, workspace, stream=None) -> None:
    """Verification with the soft (typical-acceptance) criterion; workspace of ss_tree_prune_workspace_bytes."""
    (_native or native()).tree_verify_soft(logits, draft_tokens, trees, eps, delta, accept_len, accept_path, last_node,
                                           bonus_token, edge_prob, node_entropy, workspace, stream)


def ss_tree_verify_sampled_workspace_bytes(batch: int, max_nodes: int, vocab: int) -> int:
    return int(lib().ss_tree_verify_sampled_workspace_bytes(batch, max_nodes, vocab))


def ss_tree_verify_sampled(logits, draft_tokens, trees, uniforms, top_k: int, accept_len, accept_path, last_node,
                           bonus_token, node_token, workspace, stream=None) -> None:
    """Verification against tokens drawn from the top-k softmax (temperature 1) with the caller's uniforms f32 [B][Tmax]."""
    (_native or native()).tree_verify_sampled(logits, draft_tokens, trees, uniforms, int(top_k), accept_len, accept_path,
                                              last_node, bonus_token, node_token, workspace, stream)


def ss_stream_insert(main_hidden, stream_emb, out, stream=None) -> None:
    """out[t][j] = main_hidden[t] + stream_emb[j] (Eq. 3, identity transformation); bf16 [rows][hidden], [gamma][hidden]."""
    (_native or native()).stream_insert(main_hidden, stream_emb, out, stream)


def ss_value_rotate(v_main, v_streams, epsilon: float, stream=None) -> None:
    """v_streams[t][n-1] = v_main[t] rotated by epsilon * n on (re, im) pairs (Eq. 7); bf16 [rows][width], [rows][gamma][width]."""
    (_native or native()).value_rotate(v_main, v_streams, epsilon, stream)


def make_cache_layout(k_all: torch.Tensor) -> CacheLayout:
    """Layout of a bf16 cache tensor [n_layers][slots][H][d] (d contiguous)."""
    n_layers, _, H, d = k_all.shape
    assert k_all.stride(3) == 1
    lo = CacheLayout()
    lo.n_layers, lo.n_heads, lo.head_dim = n_layers, H, d
    lo.layer_stride, lo.slot_stride, lo.head_stride = k_all.stride(0), k_all.stride(1), k_all.stride(2)
    return lo


def ss_kv_compact(k_all, v_all, layout: CacheLayout, kv_start, kv_len_in, accept_len, accept_path, kv_len_out,
                  stream=None) -> None:
    """In-place gather of the accepted path's K/V in every layer (asynchronous on `stream`)."""
    (_native or native()).kv_compact(k_all, v_all, layout, kv_start, kv_len_in, accept_len, accept_path, kv_len_out, stream)


# ---- a cache in 4 bits --------------------------------------------------------------------------
def make_kvq_cache(k_codes: torch.Tensor, k_params: torch.Tensor, v_codes: torch.Tensor, v_params: torch.Tensor) -> KvqCache:
    """Describes a cache in 4 bits: codes uint8 [n_layers][slots][H][d / 2] (d / 2 contiguous), scales and zero points int32
    [n_layers][slots][H] (any strides; slots next to each other is the fast order); K and V laid out alike."""
    for t, dtype, dims in ((k_codes, torch.uint8, 4), (v_codes, torch.uint8, 4), (k_params, torch.int32, 3), (v_params, torch.int32, 3)):
        if t.dtype is not dtype or t.dim() != dims:
            raise ValueError("codes are uint8 [n_layers][slots][H][d / 2], scales and zero points int32 [n_layers][slots][H]")
    if (k_codes.shape != v_codes.shape or k_codes.stride() != v_codes.stride() or k_params.shape != v_params.shape
            or k_params.stride() != v_params.stride() or k_codes.shape[:3] != k_params.shape or k_codes.stride(3) != 1):
        raise ValueError("K and V are laid out alike, codes and their scales have the same layers, slots and heads, and a "
                         "head's codes are contiguous")
    if len({t.device for t in (k_codes, v_codes, k_params, v_params)}) != 1:
        raise ValueError("the parts of a cache lie on one device")
    c = KvqCache()
    c.n_layers, c.total_slots, c.n_heads, c.head_dim = k_codes.shape[0], k_codes.shape[1], k_codes.shape[2], 2 * k_codes.shape[3]
    c.device = k_codes.device.index if k_codes.is_cuda else -2          # (host memory: no call takes it)
    c.k_codes, c.v_codes, c.k_params, c.v_params = _ptr(k_codes), _ptr(v_codes), _ptr(k_params), _ptr(v_params)
    c.layer_stride, c.slot_stride, c.head_stride = k_codes.stride()[:3]
    c.param_layer_stride, c.param_slot_stride, c.param_head_stride = k_params.stride()
    c.tensors = (k_codes, k_params, v_codes, v_params)
    return c


def empty_kvq_cache(n_layers: int, slots: int, n_heads: int, head_dim: int, device="cuda") -> KvqCache:
    """A cache in 4 bits of its own memory: codes [n_layers][slots][H][d / 2], a head's scales and zero points slot after slot."""
    codes = [torch.zeros((n_layers, slots, n_heads, head_dim // 2), dtype=torch.uint8, device=device) for _ in "kv"]
    params = [torch.zeros((n_layers, n_heads, slots), dtype=torch.int32, device=device).transpose(1, 2) for _ in "kv"]
    return make_kvq_cache(codes[0], params[0], codes[1], params[1])


def ss_kvq_write(k_rows, v_rows, cache: KvqCache, kv_start, kv_len_in, n_rows=None, path=None, kv_capacity=None, kv_len_out=None,
                 status=None, stream=None) -> None:
    """Quantises rows into the cache, in every layer (asynchronous on `stream`).  k_rows, v_rows: bf16 [n_layers][B][rows][H][d] (d
    contiguous); row r < n_rows[b] (int32 [B], None: all) goes to slot kv_start[b] + kv_len_in[b] + r, taken from row path[b][r]
    where a path (int32 [B][SS_PATH_STRIDE], a verification's accept_path) is given; kv_len_out[b] = kv_len_in[b] + n_rows[b].
    Sequences that do not fit are skipped; word 0 of `status` (a workspace) then says so."""
    (_native or native()).kvq_write(k_rows, v_rows, cache, kv_start, kv_len_in, n_rows, path, kv_capacity, kv_len_out, status, stream)


def ss_kvq_read(cache: KvqCache, k_rows, v_rows, kv_start, first=None, n_rows=None, stream=None) -> None:
    """Rows of the cache as bf16, in every layer: k_rows[:, b, r] for r < n_rows[b] receives slot kv_start[b] + first[b] + r."""
    (_native or native()).kvq_read(cache, k_rows, v_rows, kv_start, first, n_rows, stream)


def make_kvq_attn_params(*, q_main, o_main, k_tree, v_tree, cache: KvqCache, kv_start, kv_len, trees, gamma, sm_scale, layer=0, q_spec=None,
                         k_spec=None, v_spec=None, o_spec=None, kv_capacity=None, lse_main=None, lse_spec=None,
                         workspace=None) -> KvqAttnParams:
    """Fills ss_kvq_attn_params from tensors.  q_main, o_main, k_tree, v_tree: bf16 [B][Tmax][H][d]; *_spec: bf16
    [B][Tmax][gamma][H][d]; contiguous, on the cache's device.  The parameters keep the cache's tensors, as the cache does, not the
    others."""
    B, Tmax, H, d = q_main.shape
    if (H, d) != (cache.n_heads, cache.head_dim):
        raise ValueError("the cache holds %d heads of %d, the queries have %d of %d" % (cache.n_heads, cache.head_dim, H, d))
    main, spec = (B, Tmax, H, d), (B, Tmax, int(gamma), H, d)
    for t, shape in ((q_main, main), (o_main, main), (k_tree, main), (v_tree, main), (q_spec, spec), (k_spec, spec), (v_spec, spec), (o_spec, spec)):
        if t is not None and (t.dtype is not torch.bfloat16 or tuple(t.shape) != shape or not t.is_contiguous()):
            raise ValueError("queries, outputs and the K/V of nodes and streams are contiguous bf16 tensors [B][Tmax][H][d] and [B][Tmax][gamma][H][d]")
    for t, shape in ((lse_main, main[:-1]), (lse_spec, spec[:-1])):
        if t is not None and (t.dtype is not torch.float32 or tuple(t.shape) != shape or not t.is_contiguous()):
            raise ValueError("log-sum-exps are contiguous fp32 tensors [B][Tmax][H] and [B][Tmax][gamma][H]")
    if cache.device >= 0:
        for t in (q_main, o_main, k_tree, v_tree, q_spec, k_spec, v_spec, o_spec, lse_main, lse_spec, kv_start, kv_len, kv_capacity, trees, workspace):
            if t is not None and t.get_device() != cache.device:
                raise ValueError("the call's tensors lie on the cache's device")
        for t, dtype in ((kv_start, torch.int64), (kv_len, torch.int32), (kv_capacity, torch.int32)):
            if t is not None and (t.dtype is not dtype or t.numel() < B or not t.is_contiguous()):
                raise ValueError("kv_start is a contiguous int64 tensor of [B], kv_len and kv_capacity are int32 ones")
        if trees.numel() * trees.element_size() < B * C.sizeof(TreeDesc) or not trees.is_contiguous():
            raise ValueError("trees holds a descriptor per sequence")
    p = KvqAttnParams()
    p.batch, p.gamma, p.max_nodes, p.layer, p.sm_scale = B, int(gamma), Tmax, int(layer), float(sm_scale)
    p.q_main, p.o_main, p.k_tree, p.v_tree = _ptr(q_main), _ptr(o_main), _ptr(k_tree), _ptr(v_tree)
    p.q_spec, p.k_spec, p.v_spec, p.o_spec = _ptr(q_spec), _ptr(k_spec), _ptr(v_spec), _ptr(o_spec)
    p.cache = cache
    p.cache_tensors = getattr(cache, "tensors", None)     # (the copy above has the pointers only)
    p.kv_start, p.kv_len, p.kv_capacity, p.trees = _ptr(kv_start), _ptr(kv_len), _ptr(kv_capacity), _ptr(trees)
    p.lse_main, p.lse_spec = _ptr(lse_main), _ptr(lse_spec)
    p.workspace = _ptr(workspace)
    p.workspace_bytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    return p


def ss_msa_attention_kvq_workspace_bytes(p: KvqAttnParams) -> int:
    return int(lib().ss_msa_attention_kvq_workspace_bytes(C.byref(p)))


def ss_msa_attention_kvq(p: KvqAttnParams, stream: Optional[torch.cuda.Stream] = None) -> None:
    """One layer of tree-masked multi-stream attention over a prefix in 4 bits (asynchronous on `stream`)."""
    (_native or native()).msa_attention_kvq(p, stream)


def ss_wait_selftest(workspace: torch.Tensor, stream=None) -> None:
    """Diagnostic: one warp waits (bounded by workspace word 1) for a partial row that cannot arrive."""
    _check(lib().ss_wait_selftest(_ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)),
           "ss_wait_selftest")


def ss_status(workspace: torch.Tensor, stream=None) -> int:
    """Synchronises the stream and returns (and clears) the workspace's device status word."""
    out = C.c_int32(0)
    _check(lib().ss_status(_ptr(workspace), _stream(stream), C.byref(out)), "ss_status")
    return int(out.value)


# ---- numpy <-> device helpers for bf16 bit patterns ----------------------------------------------
def bf16_to_device(bits: np.ndarray, device="cuda") -> torch.Tensor:
    """uint16 bit patterns -> bf16 tensor on the device (no value conversion)."""
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).view(torch.bfloat16).to(device)


def bf16_to_host_bits(t: torch.Tensor) -> np.ndarray:
    """bf16 device tensor -> uint16 bit patterns on the host."""
    return t.detach().contiguous().view(torch.int16).cpu().numpy().view(np.uint16)
