"""ctypes binding of ``librpx.so`` (the C ABI declared in ``include/rpx.h``).

Only argument marshalling happens here: torch tensors supply device pointers and the current
stream; every step of the scoring path runs inside the CUDA library.  If the library is missing
the functions raise — there is no fallback path.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Tuple

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "librpx.so")
_lib = None

RPX_BF16, RPX_F32 = 0, 1
BLOCK_SIZE = 16
STATIC_SCRATCH_BYTES = 8 << 20
TREE_MAX_NODES = 1024

EXPORTS = (
    "rpx_prefix_attn",
    "rpx_suffix_attn",
    "rpx_chunk_attn",
    "rpx_tree_attn",
    "rpx_tree_attn_workspace_bytes",
    "rpx_token_logprobs",
    "rpx_token_logprobs_entropy",
    "rpx_token_logprobs_shard",
    "rpx_token_logprobs_merge",
    "rpx_token_logprobs_static",
    "rpx_token_logprobs_backward",
    "rpx_token_logprobs_backward_full",
    "rpx_token_logprobs_backward_workspace_bytes",
    "rpx_set_lm_head_pairing",
    "rpx_get_lm_head_pairing",
    "rpx_attn_backward",
    "rpx_attn_backward_workspace_bytes",
    "rpx_pages_free",
    "rpx_pages_fork",
    "rpx_pages_fork_workspace_bytes",
    "rpx_pages_compact",
    "rpx_pages_compact_workspace_bytes",
    "rpx_cache_copy_pages",
    "rpx_cache_append",
    "rpx_qk_norm_rope",
    "rpx_qk_norm_rope_backward",
    "rpx_qk_norm_rope_backward_workspace_bytes",
    "rpx_prefix_attn_workspace_bytes",
    "rpx_suffix_attn_workspace_bytes",
    "rpx_token_logprobs_workspace_bytes",
    "rpx_selftest_bounded_wait",
    "rpx_set_sm_budget",
    "rpx_get_sm_budget",
    "rpx_status_string",
    "rpx_version",
)


class RpxError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {status_string(status)} ({status})")


class AttnDesc(ctypes.Structure):
    _fields_ = [
        ("num_q_heads", ctypes.c_int32),
        ("num_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("softmax_scale", ctypes.c_float),
        ("dtype", ctypes.c_int32),
    ]


class KvCache(ctypes.Structure):
    _fields_ = [
        ("k_cache", ctypes.c_void_p),
        ("v_cache", ctypes.c_void_p),
        ("num_blocks", ctypes.c_int64),
        ("block_size", ctypes.c_int32),
        ("block_table", ctypes.c_void_p),
        ("block_table_stride", ctypes.c_int32),
    ]


class PagePool(ctypes.Structure):
    _fields_ = [
        ("block_table", ctypes.c_void_p),
        ("block_table_stride", ctypes.c_int32),
        ("table_cols", ctypes.c_int32),
        ("rows", ctypes.c_int32),
        ("lens", ctypes.c_void_p),
        ("ref_counts", ctypes.c_void_p),
        ("num_blocks", ctypes.c_int32),
    ]


class RopeDesc(ctypes.Structure):
    _fields_ = [
        ("num_q_heads", ctypes.c_int32),
        ("num_kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("rot_dim", ctypes.c_int32),
        ("num_axes", ctypes.c_int32),
        ("pair_axis", ctypes.c_char_p),
        ("eps", ctypes.c_float),
        ("dtype", ctypes.c_int32),
    ]


def library_path() -> str:
    return _LIB_PATH


def load_library():
    """Load librpx.so (built in-tree by ``paper_2608_14498_b200.build``); raises if absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB_PATH):
        raise FileNotFoundError(
            f"{_LIB_PATH} is missing: build it with `python -m paper_2608_14498_b200.build` "
            "(there is no CPU or eager fallback)"
        )
    lib = ctypes.CDLL(_LIB_PATH)
    vp, i32, i64, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
    lib.rpx_prefix_attn.restype = i32
    lib.rpx_prefix_attn.argtypes = [ctypes.POINTER(AttnDesc), vp, vp, vp, i64, i64, i64, vp, i32, i64, i32,
                                    ctypes.POINTER(KvCache), vp, vp, vp, sz, vp, vp]
    lib.rpx_suffix_attn.restype = i32
    lib.rpx_suffix_attn.argtypes = [ctypes.POINTER(AttnDesc), vp, vp, vp, i64, i64, i64, vp, vp, i32, i64, i32,
                                    i32, ctypes.POINTER(KvCache), vp, vp, vp, sz, vp, vp]
    lib.rpx_chunk_attn.restype = i32
    lib.rpx_chunk_attn.argtypes = [ctypes.POINTER(AttnDesc), vp, vp, vp, i64, i64, i64, vp, vp, i32, i64, i32,
                                    i32, ctypes.POINTER(KvCache), vp, vp, vp, sz, vp, vp]
    lib.rpx_tree_attn.restype = i32
    lib.rpx_tree_attn.argtypes = [ctypes.POINTER(AttnDesc), vp, vp, vp, i64, i64, i64, vp, vp, vp, i32, i64, i32, i32,
                                  ctypes.POINTER(KvCache), vp, vp, vp, sz, vp, vp]
    lib.rpx_tree_attn_workspace_bytes.restype = sz
    lib.rpx_tree_attn_workspace_bytes.argtypes = [ctypes.POINTER(AttnDesc), i64, i32, i32]
    lib.rpx_token_logprobs.restype = i32
    lib.rpx_token_logprobs.argtypes = [vp, i64, vp, vp, i64, i32, i32, i32, vp, vp, vp, sz, vp, vp]
    lib.rpx_token_logprobs_entropy.restype = i32
    lib.rpx_token_logprobs_entropy.argtypes = [vp, i64, vp, vp, i64, i32, i32, i32, vp, vp, vp, vp, sz, vp, vp]
    lib.rpx_token_logprobs_shard.restype = i32
    lib.rpx_token_logprobs_shard.argtypes = [vp, i64, vp, vp, i64, i32, i32, i32, i32, vp, vp, sz, vp, vp]
    lib.rpx_token_logprobs_merge.restype = i32
    lib.rpx_token_logprobs_merge.argtypes = [vp, i32, vp, i64, i32, vp, vp, vp, vp, vp]
    lib.rpx_token_logprobs_static.restype = i32
    lib.rpx_token_logprobs_static.argtypes = [vp, i64, vp, vp, i64, i32, i32, vp, vp, vp, vp]
    lib.rpx_token_logprobs_backward.restype = i32
    lib.rpx_token_logprobs_backward.argtypes = [vp, i64, vp, vp, vp, vp, i64, i32, i32, i32, vp, vp, sz, vp, vp]
    lib.rpx_token_logprobs_backward_full.restype = i32
    lib.rpx_token_logprobs_backward_full.argtypes = [vp, i64, vp, vp, vp, vp, i64, i32, i32, i32, vp, vp, i32, vp, sz, vp, vp]
    lib.rpx_token_logprobs_backward_workspace_bytes.restype = sz
    lib.rpx_token_logprobs_backward_workspace_bytes.argtypes = [i64, i32, i32, i32]
    lib.rpx_attn_backward.restype = i32
    lib.rpx_attn_backward.argtypes = [ctypes.POINTER(AttnDesc), vp, vp, vp, i64, i64, i64, vp, vp, vp, vp, vp, vp, i32,
                                      i64, i32, vp, vp, vp, i32, vp, sz, vp, vp]
    lib.rpx_attn_backward_workspace_bytes.restype = sz
    lib.rpx_attn_backward_workspace_bytes.argtypes = [ctypes.POINTER(AttnDesc), i64]
    pool = ctypes.POINTER(PagePool)
    lib.rpx_pages_free.restype = i32
    lib.rpx_pages_free.argtypes = [pool, vp, i32, vp, vp]
    lib.rpx_pages_fork.restype = i32
    lib.rpx_pages_fork.argtypes = [pool, vp, vp, i32, i32, vp, vp, vp, sz, vp, vp]
    lib.rpx_pages_fork_workspace_bytes.restype = sz
    lib.rpx_pages_fork_workspace_bytes.argtypes = [pool, i32]
    lib.rpx_pages_compact.restype = i32
    lib.rpx_pages_compact.argtypes = [pool, vp, i32, vp, vp, vp, vp, vp, sz, vp, vp]
    lib.rpx_pages_compact_workspace_bytes.restype = sz
    lib.rpx_pages_compact_workspace_bytes.argtypes = [pool]
    lib.rpx_cache_copy_pages.restype = i32
    lib.rpx_cache_copy_pages.argtypes = [vp, vp, i32, i64, i64, i32, i32, vp, vp, i64, vp, vp]
    lib.rpx_cache_append.restype = i32
    lib.rpx_cache_append.argtypes = [vp, vp, i64, i64, i64, i32, i32, i32, vp, i64, vp, vp, i32, i32, ctypes.POINTER(KvCache), vp,
                                     vp]
    lib.rpx_qk_norm_rope.restype = i32
    lib.rpx_qk_norm_rope.argtypes = [ctypes.POINTER(RopeDesc), vp, vp, i64, i64, vp, vp, vp, i64, vp, i64, vp, vp, i64, i64, vp]
    lib.rpx_qk_norm_rope_backward.restype = i32
    lib.rpx_qk_norm_rope_backward.argtypes = [ctypes.POINTER(RopeDesc), vp, vp, i64, i64, vp, vp, vp, i64, vp, vp, vp, i64, vp,
                                              vp, i64, i64, vp, vp, i32, vp, sz, vp]
    lib.rpx_qk_norm_rope_backward_workspace_bytes.restype = sz
    lib.rpx_qk_norm_rope_backward_workspace_bytes.argtypes = [ctypes.POINTER(RopeDesc), i64]
    lib.rpx_prefix_attn_workspace_bytes.restype = sz
    lib.rpx_prefix_attn_workspace_bytes.argtypes = [ctypes.POINTER(AttnDesc), i64]
    lib.rpx_suffix_attn_workspace_bytes.restype = sz
    lib.rpx_suffix_attn_workspace_bytes.argtypes = [ctypes.POINTER(AttnDesc), i64]
    lib.rpx_token_logprobs_workspace_bytes.restype = sz
    lib.rpx_token_logprobs_workspace_bytes.argtypes = [i64, i32, i32, i32]
    lib.rpx_selftest_bounded_wait.restype = i32
    lib.rpx_selftest_bounded_wait.argtypes = [i64, vp, vp]
    lib.rpx_set_sm_budget.restype = i32
    lib.rpx_set_sm_budget.argtypes = [i32]
    lib.rpx_get_sm_budget.restype = i32
    lib.rpx_get_sm_budget.argtypes = []
    lib.rpx_set_lm_head_pairing.restype = i32
    lib.rpx_set_lm_head_pairing.argtypes = [i32]
    lib.rpx_get_lm_head_pairing.restype = i32
    lib.rpx_get_lm_head_pairing.argtypes = []
    lib.rpx_status_string.restype = ctypes.c_char_p
    lib.rpx_status_string.argtypes = [i32]
    lib.rpx_version.restype = i32
    lib.rpx_version.argtypes = []
    _lib = lib
    return lib


def status_string(status: int) -> str:
    return load_library().rpx_status_string(int(status)).decode()


def version() -> int:
    return int(load_library().rpx_version())


# ------------------------------------------------------------------ helpers (torch side)
_torch_module = None


def _torch():
    global _torch_module
    if _torch_module is None:
        import torch

        _torch_module = torch
    return _torch_module


def _dtype_code(t) -> int:
    torch = _torch()
    if t.dtype == torch.bfloat16:
        return RPX_BF16
    if t.dtype == torch.float32:
        return RPX_F32
    raise TypeError(f"rpx tensors are bfloat16 or float32, got {t.dtype}")


def _ptr(t) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream_ptr(stream) -> int:
    if stream is not None:
        return stream.cuda_stream
    c = _torch()._C  # the raw handles: torch.cuda's own functions take ten times as long
    return c._cuda_getCurrentRawStream(c._cuda_getDevice())


def _tok_stride(t) -> int:
    shape, stride = t.shape, t.stride()
    if len(shape) != 3:
        raise ValueError("expected a [tokens, heads, head_dim] tensor")
    if shape[0] == 0:
        return shape[1] * shape[2]
    if stride[2] != 1 or (stride[1] != shape[2] and shape[1] > 1):  # (one head has no neighbour)
        raise ValueError("expected a [tokens, heads, head_dim] tensor with contiguous heads")
    return stride[0] if shape[0] > 1 else shape[1] * shape[2]


def _workspace(nbytes: int, device, workspace):
    torch = _torch()
    if workspace is not None:
        if workspace.nbytes < nbytes:
            raise ValueError(f"workspace too small: need {nbytes} bytes")
        return workspace
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)


def _in_call_context(fn):
    """Runs a wrapper with its first tensor's device current (the library launches on the current device) and,
    when ``stream=`` is given, with that stream current, so that outputs and temporary workspaces the wrapper
    allocates belong to the stream the kernels run on."""
    import functools

    @functools.wraps(fn)
    def call(*args, **kwargs):
        torch = _torch()
        first = args[0] if args else next(x for x in kwargs.values() if isinstance(x, torch.Tensor))
        stream = kwargs.get("stream")
        if stream is None and first.is_cuda and first.get_device() == torch._C._cuda_getDevice():
            return fn(*args, **kwargs)  # the usual case, without the cost of entering a context
        with torch.cuda.device(first.device):
            if stream is None:
                return fn(*args, **kwargs)
            with torch.cuda.stream(stream):
                return fn(*args, **kwargs)
    return call


def _bound(x) -> int:
    """A bound or a count for the C ABI: any whole number, and nothing that 32 bits would cut."""
    x = int(x)
    if not 0 <= x < 1 << 31:
        raise ValueError(f"{x} is not a count of 32 bits")
    return x


def _one_device(first, *others) -> None:
    """Kernels take bare pointers: an index tensor left on the host, or on another GPU, would be read as this GPU's memory."""
    device = first.get_device()
    for t in others:
        if t is not None and t.get_device() != device:
            raise ValueError(f"all tensors of a call are on one device: {t.device} next to {first.device}")


def _desc(q, k, softmax_scale: float) -> AttnDesc:
    return AttnDesc(q.shape[1], k.shape[1], q.shape[2], float(softmax_scale), _dtype_code(q))


def _cache_struct(cache) -> KvCache:
    k_cache, v_cache, block_table = cache
    torch = _torch()
    if k_cache.dtype != torch.bfloat16 or v_cache.dtype != torch.bfloat16 or block_table.dtype != torch.int32:
        raise TypeError("cache pools are bfloat16 and the block table is int32")
    if not (k_cache.is_contiguous() and v_cache.is_contiguous()) or block_table.stride(1) != 1:
        raise ValueError("cache pools must be contiguous [blocks, kv_heads, 16, head_dim]")
    return KvCache(k_cache.data_ptr(), v_cache.data_ptr(), k_cache.shape[0], k_cache.shape[2],
                   block_table.data_ptr(), block_table.stride(0))


def prefix_attn_workspace_bytes(num_q_heads, num_kv_heads, head_dim, dtype_code, total_tokens) -> int:
    d = AttnDesc(num_q_heads, num_kv_heads, head_dim, 0.0, dtype_code)
    return int(load_library().rpx_prefix_attn_workspace_bytes(ctypes.byref(d), int(total_tokens)))


def suffix_attn_workspace_bytes(num_q_heads, num_kv_heads, head_dim, dtype_code, total_tokens) -> int:
    d = AttnDesc(num_q_heads, num_kv_heads, head_dim, 0.0, dtype_code)
    return int(load_library().rpx_suffix_attn_workspace_bytes(ctypes.byref(d), int(total_tokens)))


def attn_backward_workspace_bytes(num_q_heads, num_kv_heads, head_dim, total_tokens) -> int:
    desc = AttnDesc(num_q_heads, num_kv_heads, head_dim, 0.0, RPX_BF16)
    return int(load_library().rpx_attn_backward_workspace_bytes(ctypes.byref(desc), int(total_tokens)))


def token_logprobs_workspace_bytes(n_tokens, hidden_dim, vocab, dtype_code) -> int:
    return int(load_library().rpx_token_logprobs_workspace_bytes(int(n_tokens), int(hidden_dim), int(vocab),
                                                                 int(dtype_code)))


def selftest_bounded_wait(limit_cycles: int, device_status, stream=None) -> None:
    """rpx_selftest_bounded_wait: a wait that must time out and report RPX_ERR_TIMEOUT in device_status."""
    rc = load_library().rpx_selftest_bounded_wait(int(limit_cycles), _ptr(device_status), _stream_ptr(stream))
    if rc != 0:
        raise RpxError(rc, "rpx_selftest_bounded_wait")


def set_sm_budget(sms: int) -> None:
    """rpx_set_sm_budget: cap the persistent kernels' grids at ``sms`` CTAs (0 = no cap), process-wide."""
    rc = load_library().rpx_set_sm_budget(int(sms))
    if rc != 0:
        raise RpxError(rc, "rpx_set_sm_budget")


def set_lm_head_pairing(on: bool) -> None:
    """Process-wide choice of the LM-head kernel: CTA pairs (cta_group::2) when ``on``."""
    rc = load_library().rpx_set_lm_head_pairing(1 if on else 0)
    if rc != 0:
        raise RpxError(rc, "rpx_set_lm_head_pairing")


def get_lm_head_pairing() -> bool:
    return bool(load_library().rpx_get_lm_head_pairing())


def get_sm_budget() -> int:
    return int(load_library().rpx_get_sm_budget())


# ------------------------------------------------------------------ the three calls
@_in_call_context
def prefix_attn(q, k, v, cu_seqlens, max_seqlen: int, cache: Optional[Tuple] = None, softmax_scale: float = 0.0,
                out=None, lse=None, return_lse: bool = False, workspace=None, device_status=None, stream=None):
    """rpx_prefix_attn: causal GQA attention over packed prompts, writing the paged KV cache.

    q [T, H_q, d], k/v [T, H_kv, d] device tensors; cu_seqlens int32 [B+1] on the device;
    cache = (k_cache, v_cache, block_table) or None.  Returns out (and lse when asked).
    """
    torch = _torch()
    lib = load_library()
    desc = _desc(q, k, softmax_scale)
    total = q.shape[0]
    if out is None:
        out = torch.empty((total, q.shape[1], q.shape[2]), dtype=q.dtype, device=q.device)
    if lse is None and return_lse:
        lse = torch.empty((total, q.shape[1]), dtype=torch.float32, device=q.device)
    ws = _workspace(int(lib.rpx_prefix_attn_workspace_bytes(ctypes.byref(desc), total)), q.device, workspace)
    cs = _cache_struct(cache) if cache is not None else None
    rc = lib.rpx_prefix_attn(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _tok_stride(q), _tok_stride(k),
                             _tok_stride(v), _ptr(cu_seqlens), cu_seqlens.shape[0] - 1, total, int(max_seqlen),
                             ctypes.byref(cs) if cs is not None else None, _ptr(out), _ptr(lse), _ptr(ws),
                             ws.numel() * ws.element_size(), _ptr(device_status), _stream_ptr(stream))
    if rc != 0:
        raise RpxError(rc, "rpx_prefix_attn")
    return (out, lse) if return_lse else out


@_in_call_context
def suffix_attn(q, k, v, cu_seqlens_suffix, prefix_lens, max_suffix_len: int, max_prefix_len: int, cache: Tuple,
                softmax_scale: float = 0.0, out=None, lse=None, return_lse: bool = False, workspace=None,
                device_status=None, stream=None):
    """rpx_suffix_attn: response queries over [cached prefix KV ; causal self]."""
    torch = _torch()
    lib = load_library()
    desc = _desc(q, k, softmax_scale)
    total = q.shape[0]
    if out is None:
        out = torch.empty((total, q.shape[1], q.shape[2]), dtype=q.dtype, device=q.device)
    if lse is None and return_lse:
        lse = torch.empty((total, q.shape[1]), dtype=torch.float32, device=q.device)
    ws = _workspace(int(lib.rpx_suffix_attn_workspace_bytes(ctypes.byref(desc), total)), q.device, workspace)
    cs = _cache_struct(cache)
    rc = lib.rpx_suffix_attn(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _tok_stride(q), _tok_stride(k),
                             _tok_stride(v), _ptr(cu_seqlens_suffix), _ptr(prefix_lens),
                             cu_seqlens_suffix.shape[0] - 1, total, int(max_suffix_len), int(max_prefix_len),
                             ctypes.byref(cs), _ptr(out), _ptr(lse), _ptr(ws), ws.numel() * ws.element_size(),
                             _ptr(device_status), _stream_ptr(stream))
    if rc != 0:
        raise RpxError(rc, "rpx_suffix_attn")
    return (out, lse) if return_lse else out


@_in_call_context
def chunk_attn(q, k, v, cu_seqlens_chunk, cached_lens, max_chunk_len: int, max_cached_len: int, cache: Tuple,
                softmax_scale: float = 0.0, out=None, lse=None, return_lse: bool = False, workspace=None,
                device_status=None, stream=None):
    """rpx_chunk_attn: the next chunk of every prompt over [cached earlier chunks ; causal self], appending
    the chunk's K/V to the cache (cached_lens must be multiples of the 16-token block)."""
    torch = _torch()
    lib = load_library()
    desc = _desc(q, k, softmax_scale)
    total = q.shape[0]
    if out is None:
        out = torch.empty((total, q.shape[1], q.shape[2]), dtype=q.dtype, device=q.device)
    if lse is None and return_lse:
        lse = torch.empty((total, q.shape[1]), dtype=torch.float32, device=q.device)
    ws = _workspace(int(lib.rpx_suffix_attn_workspace_bytes(ctypes.byref(desc), total)), q.device, workspace)
    cs = _cache_struct(cache)
    rc = lib.rpx_chunk_attn(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _tok_stride(q), _tok_stride(k),
                             _tok_stride(v), _ptr(cu_seqlens_chunk), _ptr(cached_lens),
                             cu_seqlens_chunk.shape[0] - 1, total, int(max_chunk_len), int(max_cached_len),
                             ctypes.byref(cs), _ptr(out), _ptr(lse), _ptr(ws), ws.numel() * ws.element_size(),
                             _ptr(device_status), _stream_ptr(stream))
    if rc != 0:
        raise RpxError(rc, "rpx_chunk_attn")
    return (out, lse) if return_lse else out


def tree_attn_workspace_bytes(num_q_heads, num_kv_heads, head_dim, dtype_code, total_tokens, batch, max_tree_len) -> int:
    d = AttnDesc(num_q_heads, num_kv_heads, head_dim, 0.0, dtype_code)
    return int(load_library().rpx_tree_attn_workspace_bytes(ctypes.byref(d), int(total_tokens), int(batch), int(max_tree_len)))


@_in_call_context
def tree_attn(q, k, v, cu_seqlens_tree, parents, cached_lens, max_tree_len: int, max_cached_len: int, cache: Tuple,
              softmax_scale: float = 0.0, out=None, lse=None, return_lse: bool = False, workspace=None, device_status=None,
              stream=None):
    """rpx_tree_attn: nodes of a tree of drafted tokens over [cached keys ; ancestors and itself]; one node per sequence is a
    decoding step.

    parents int32 [T]: the node (numbered within its sequence) each node continues, -1 = the cached prefix, -2 = padding
    (out 0, lse -inf).  Other arguments as in ``suffix_attn``."""
    torch = _torch()
    lib = load_library()
    _one_device(q, k, v, cu_seqlens_tree, parents, cached_lens, *cache, out, lse, workspace, device_status)
    max_tree_len, max_cached_len = _bound(max_tree_len), _bound(max_cached_len)
    desc = ctypes.byref(_desc(q, k, softmax_scale))
    total, heads, _ = q.shape
    batch = cu_seqlens_tree.shape[0] - 1
    for t in (cu_seqlens_tree, parents, cached_lens):
        if t.dtype != torch.int32 or not t.is_contiguous():
            raise TypeError("cu_seqlens_tree, parents and cached_lens are contiguous int32 tensors")
    if parents.shape[0] != total or cached_lens.shape[0] != batch:
        raise ValueError("parents has one entry per token and cached_lens one per sequence")
    if v.shape != k.shape or k.dtype != q.dtype or v.dtype != q.dtype or k.shape[0] != total:
        raise ValueError("k and v are [tokens, kv_heads, head_dim] tensors with the tokens and the element type of q")
    if cache[0].shape[1:] != (k.shape[1], BLOCK_SIZE, k.shape[2]) or cache[1].shape != cache[0].shape or cache[2].shape[0] < batch:
        raise ValueError("the cache pools are [blocks, kv_heads, 16, head_dim], the block table has a row for each sequence")
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    elif out.shape != q.shape or out.dtype != q.dtype or not out.is_contiguous():
        raise ValueError("out is a contiguous tensor of the shape and element type of q")
    if lse is not None and (lse.shape != (total, heads) or lse.dtype != torch.float32 or not lse.is_contiguous()):
        raise ValueError("lse is a contiguous float32 [tokens, q_heads] tensor")
    if lse is None and return_lse:
        lse = torch.empty((total, heads), dtype=torch.float32, device=q.device)
    need = lib.rpx_tree_attn_workspace_bytes(desc, total, batch, max_tree_len)
    ws = _workspace(need, q.device, workspace)
    rc = lib.rpx_tree_attn(desc, q.data_ptr(), k.data_ptr(), v.data_ptr(), _tok_stride(q), _tok_stride(k), _tok_stride(v),
                           cu_seqlens_tree.data_ptr(), parents.data_ptr(), cached_lens.data_ptr(), batch, total, max_tree_len,
                           max_cached_len, ctypes.byref(_cache_struct(cache)), out.data_ptr(), _ptr(lse), ws.data_ptr(),
                           ws.nbytes, _ptr(device_status), _stream_ptr(stream))
    if rc != 0:
        raise RpxError(rc, "rpx_tree_attn")
    return (out, lse) if return_lse else out


@_in_call_context
def token_logprobs(hidden, w_vocab, target_ids, logprobs=None, lse=None, return_lse: bool = False, workspace=None,
                   device_status=None, stream=None, entropy=None):
    """rpx_token_logprobs: log p(target) per row from hidden [N, H] and W [V, H]; logits never stored.

    ``entropy`` (float32 [N], optional) additionally receives the entropy of each row's next-token
    distribution from the same pass (rpx_token_logprobs_entropy)."""
    torch = _torch()
    lib = load_library()
    code = _dtype_code(hidden)
    if _dtype_code(w_vocab) != code:
        raise TypeError("hidden and w_vocab must share an element type")
    if hidden.dim() != 2 or hidden.stride(1) != 1 or not w_vocab.is_contiguous():
        raise ValueError("hidden must be [N, H] with contiguous rows and w_vocab contiguous [V, H]")
    n, hdim = hidden.shape
    vocab = w_vocab.shape[0]
    if logprobs is None:
        logprobs = torch.empty((n,), dtype=torch.float32, device=hidden.device)
    if lse is None and return_lse:
        lse = torch.empty((n,), dtype=torch.float32, device=hidden.device)
    ws = _workspace(int(lib.rpx_token_logprobs_workspace_bytes(n, hdim, vocab, code)), hidden.device, workspace)
    row_stride = hidden.stride(0) if n > 1 else hdim
    if entropy is None:
        rc = lib.rpx_token_logprobs(_ptr(hidden), row_stride, _ptr(w_vocab), _ptr(target_ids), n, hdim, vocab, code,
                                    _ptr(logprobs), _ptr(lse), _ptr(ws), ws.numel() * ws.element_size(),
                                    _ptr(device_status), _stream_ptr(stream))
    else:
        rc = lib.rpx_token_logprobs_entropy(_ptr(hidden), row_stride, _ptr(w_vocab), _ptr(target_ids), n, hdim, vocab,
                                            code, _ptr(logprobs), _ptr(lse), _ptr(entropy), _ptr(ws),
                                            ws.numel() * ws.element_size(), _ptr(device_status), _stream_ptr(stream))
    if rc != 0:
        raise RpxError(rc, "rpx_token_logprobs")
    return (logprobs, lse) if return_lse else logprobs


def token_logprobs_backward_workspace_bytes(n_tokens, hidden_dim, vocab, dtype_code=RPX_BF16) -> int:
    return int(load_library().rpx_token_logprobs_backward_workspace_bytes(int(n_tokens), int(hidden_dim), int(vocab),
                                                                          int(dtype_code)))


@_in_call_context
def token_logprobs_backward(hidden, w_vocab, target_ids, lse, upstream, dhidden=None, workspace=None, device_status=None,
                            stream=None, dw=None, want_dw: bool = False, accumulate_dw: bool = False,
                            want_dhidden: bool = True):
    """rpx_token_logprobs_backward(_full): d(sum upstream * logprobs) / d hidden, bf16 [N, H], and - with ``want_dw`` or a
    ``dw`` buffer - d / d w_vocab, float32 [V, H] (added to ``dw`` when ``accumulate_dw``).

    ``lse`` is the forward call's lse output for the same rows, ``upstream`` float32 [N].  Returns dhidden, or
    (dhidden, dw) when the weight gradient was asked for (dhidden is None with ``want_dhidden=False``)."""
    torch = _torch()
    lib = load_library()
    if _dtype_code(hidden) != RPX_BF16 or _dtype_code(w_vocab) != RPX_BF16:
        raise TypeError("the LM-head backward pass takes bfloat16 tensors only")
    if hidden.dim() != 2 or hidden.stride(1) != 1 or not w_vocab.is_contiguous():
        raise ValueError("hidden must be [N, H] with contiguous rows and w_vocab contiguous [V, H]")
    if lse.dtype != torch.float32 or upstream.dtype != torch.float32:
        raise TypeError("lse and upstream are float32")
    n, hdim = hidden.shape
    vocab = w_vocab.shape[0]
    if dhidden is None and want_dhidden:
        dhidden = torch.empty((n, hdim), dtype=torch.bfloat16, device=hidden.device)
    with_dw = want_dw or dw is not None
    if with_dw:
        if dw is None:
            if accumulate_dw:
                raise ValueError("accumulate_dw needs the dw buffer to add to")
            dw = torch.empty((vocab, hdim), dtype=torch.float32, device=hidden.device)
        if dw.dtype != torch.float32 or not dw.is_contiguous() or tuple(dw.shape) != (vocab, hdim):
            raise ValueError("dw is a contiguous float32 [V, H] tensor")
    ws = _workspace(int(lib.rpx_token_logprobs_backward_workspace_bytes(n, hdim, vocab, RPX_BF16)), hidden.device, workspace)
    rc = lib.rpx_token_logprobs_backward_full(_ptr(hidden), hidden.stride(0) if n > 1 else hdim, _ptr(w_vocab),
                                              _ptr(target_ids), _ptr(lse), _ptr(upstream), n, hdim, vocab, RPX_BF16,
                                              _ptr(dhidden), _ptr(dw), 1 if accumulate_dw else 0, _ptr(ws),
                                              ws.numel() * ws.element_size(), _ptr(device_status), _stream_ptr(stream))
    if rc != 0:
        raise RpxError(rc, "rpx_token_logprobs_backward_full")
    return (dhidden, dw) if with_dw else dhidden


@_in_call_context
def attn_backward(q, k, v, out, dout, lse, cu_seqlens, max_seqlen: int, q_begin=None, q_end=None, softmax_scale: float = 0.0,
                  dq=None, dk=None, dv=None, accumulate_dkv: bool = False, workspace=None, device_status=None, stream=None):
    """rpx_attn_backward: gradients of causal GQA attention over packed whole sequences.

    q [T, H_q, d], k/v [T, H_kv, d], out/dout [T, H_q, d] bfloat16; lse float32 [T, H_q] from the forward pass;
    q_begin / q_end (int32 [B], optional) restrict the query rows that take part.  Returns float32 (dq, dk, dv);
    with ``accumulate_dkv`` the call's dk, dv are added to the given buffers."""
    torch = _torch()
    lib = load_library()
    if any(_dtype_code(t) != RPX_BF16 for t in (q, k, v, out, dout)):
        raise TypeError("the attention backward pass takes bfloat16 tensors only")
    if lse.dtype != torch.float32 or not lse.is_contiguous() or not out.is_contiguous() or not dout.is_contiguous():
        raise ValueError("out, dout and lse (float32) must be contiguous")
    desc = _desc(q, k, softmax_scale)
    total = q.shape[0]
    if dq is None:
        dq = torch.empty(tuple(q.shape), dtype=torch.float32, device=q.device)
    if accumulate_dkv and (dk is None or dv is None):
        raise ValueError("accumulate_dkv needs the dk and dv buffers to add to")
    if dk is None:
        dk = torch.empty(tuple(k.shape), dtype=torch.float32, device=q.device)
    if dv is None:
        dv = torch.empty(tuple(v.shape), dtype=torch.float32, device=q.device)
    for t in (dq, dk, dv):
        if t.dtype != torch.float32 or not t.is_contiguous():
            raise ValueError("dq, dk, dv are contiguous float32 tensors")
    ws = _workspace(int(lib.rpx_attn_backward_workspace_bytes(ctypes.byref(desc), total)), q.device, workspace)
    rc = lib.rpx_attn_backward(ctypes.byref(desc), _ptr(q), _ptr(k), _ptr(v), _tok_stride(q), _tok_stride(k),
                               _tok_stride(v), _ptr(out), _ptr(dout), _ptr(lse), _ptr(cu_seqlens), _ptr(q_begin),
                               _ptr(q_end), cu_seqlens.shape[0] - 1, total, int(max_seqlen), _ptr(dq), _ptr(dk), _ptr(dv),
                               1 if accumulate_dkv else 0, _ptr(ws), ws.numel() * ws.element_size(), _ptr(device_status),
                               _stream_ptr(stream))
    if rc != 0:
        raise RpxError(rc, "rpx_attn_backward")
    return dq, dk, dv


@_in_call_context
def token_logprobs_static(hidden, w_vocab, target_ids, logprobs, lse=None, device_status=None, stream=None):
    """rpx_token_logprobs_static: the same log-probs, for callers that cannot allocate device memory.

    Nothing is allocated on this path, not even by torch: ``logprobs`` (float32 [N]) must be passed
    in, and the partial records go to a fixed array inside the library.  Use it where the device
    allocator is out of reach (all HBM already reserved by the host engine, or a code section in
    which an allocator call could fail or stall the device).  bf16 only; the problem must fit
    ``STATIC_SCRATCH_BYTES`` (raises RpxError RPX_ERR_WORKSPACE otherwise); calls that overlap on
    the GPU race on the shared array.
    """
    lib = load_library()
    if _dtype_code(hidden) != RPX_BF16 or _dtype_code(w_vocab) != RPX_BF16:
        raise TypeError("the allocation-free entry point takes bfloat16 tensors only")
    if hidden.dim() != 2 or hidden.stride(1) != 1 or not w_vocab.is_contiguous():
        raise ValueError("hidden must be [N, H] with contiguous rows and w_vocab contiguous [V, H]")
    n, hdim = hidden.shape
    row_stride = hidden.stride(0) if n > 1 else hdim
    rc = lib.rpx_token_logprobs_static(_ptr(hidden), row_stride, _ptr(w_vocab), _ptr(target_ids), n, hdim,
                                       w_vocab.shape[0], _ptr(logprobs), _ptr(lse), _ptr(device_status),
                                       _stream_ptr(stream))
    if rc != 0:
        raise RpxError(rc, "rpx_token_logprobs_static")
    return logprobs


@_in_call_context
def token_logprobs_shard(hidden, w_shard, target_ids, vocab_begin: int, shard_stats=None, workspace=None,
                         device_status=None, stream=None):
    """rpx_token_logprobs_shard: this rank's share of a vocabulary-parallel LM head.

    w_shard holds rows vocab_begin .. vocab_begin + V_local - 1 of W_vocab; target_ids are global ids.
    Returns shard_stats float32 [N, 4] to be gathered over ranks and passed to token_logprobs_merge."""
    torch = _torch()
    lib = load_library()
    code = _dtype_code(hidden)
    if _dtype_code(w_shard) != code:
        raise TypeError("hidden and w_shard must share an element type")
    if hidden.dim() != 2 or hidden.stride(1) != 1 or not w_shard.is_contiguous():
        raise ValueError("hidden must be [N, H] with contiguous rows and w_shard contiguous [V_local, H]")
    n, hdim = hidden.shape
    v_local = w_shard.shape[0]
    if shard_stats is None:
        shard_stats = torch.empty((n, 4), dtype=torch.float32, device=hidden.device)
    ws = _workspace(int(lib.rpx_token_logprobs_workspace_bytes(n, hdim, v_local, code)), hidden.device, workspace)
    rc = lib.rpx_token_logprobs_shard(_ptr(hidden), hidden.stride(0) if n > 1 else hdim, _ptr(w_shard), _ptr(target_ids), n,
                                      hdim, v_local, int(vocab_begin), code, _ptr(shard_stats), _ptr(ws),
                                      ws.numel() * ws.element_size(), _ptr(device_status), _stream_ptr(stream))
    if rc != 0:
        raise RpxError(rc, "rpx_token_logprobs_shard")
    return shard_stats


@_in_call_context
def token_logprobs_merge(all_stats, target_ids, vocab_total: int, logprobs=None, return_lse: bool = False, entropy=None,
                         device_status=None, stream=None):
    """rpx_token_logprobs_merge: final log-probs from the gathered shard records float32 [R, N, 4]."""
    torch = _torch()
    lib = load_library()
    if all_stats.dim() != 3 or all_stats.shape[2] != 4 or all_stats.dtype != torch.float32 or not all_stats.is_contiguous():
        raise ValueError("all_stats must be a contiguous float32 [shards, N, 4] tensor")
    r, n, _ = all_stats.shape
    if logprobs is None:
        logprobs = torch.empty((n,), dtype=torch.float32, device=all_stats.device)
    lse = torch.empty((n,), dtype=torch.float32, device=all_stats.device) if return_lse else None
    rc = lib.rpx_token_logprobs_merge(_ptr(all_stats), r, _ptr(target_ids), n, int(vocab_total), _ptr(logprobs), _ptr(lse),
                                      _ptr(entropy), _ptr(device_status), _stream_ptr(stream))
    if rc != 0:
        raise RpxError(rc, "rpx_token_logprobs_merge")
    return (logprobs, lse) if return_lse else logprobs


# ------------------------------------------------------------------ norm + rotation in front of the attention calls
def mrope_pair_axis(sections, interleaved: bool = False):
    """Axis of every rotary pair for positions on several axes: ``sections[a]`` pairs for axis a, one run after the other,
    or - ``interleaved`` - the axes taking turns while they have pairs left (pair i goes to axis i mod n) and axis 0
    taking every other pair."""
    n, total = len(sections), sum(sections)
    if n < 1 or any(s < 0 for s in sections):
        raise ValueError("sections are pair counts, one per axis")
    if not interleaved:
        return [a for a, s in enumerate(sections) for _ in range(s)]
    axes = [i % n if i // n < sections[i % n] else 0 for i in range(total)]
    if [axes.count(a) for a in range(n)] != list(sections):
        raise ValueError("these sections cannot take turns: an axis other than 0 has more pairs than there are turns")
    return axes


def _axis_bytes(pair_axis, pairs: int) -> bytes:
    if not isinstance(pair_axis, (list, tuple, bytes)):
        # an array's numbers and not its memory, which is what bytes() takes from anything with a buffer
        if getattr(pair_axis, "is_cuda", False):
            raise TypeError("pair_axis is read on the host")
        pair_axis = pair_axis.tolist() if hasattr(pair_axis, "tolist") else list(pair_axis)
    if len(pair_axis) != pairs:
        raise ValueError("pair_axis has one axis number per entry of inv_freq")
    try:
        return bytes(pair_axis)
    except ValueError:
        raise ValueError("axis numbers of pair_axis are 0 .. num_axes - 1") from None


def _rope_desc(q, k, positions, inv_freq, q_weight, k_weight, pair_axis, eps) -> RopeDesc:
    torch = _torch()
    dtype = q.dtype
    code = _dtype_code(q)
    if k.dtype != dtype:
        raise TypeError("q, k and the norm weights must share an element type")
    if positions.dtype != torch.int32 or inv_freq.dtype != torch.float32:
        raise TypeError("positions are int32 and inv_freq float32")
    q_shape, k_shape, pos_shape = q.shape, k.shape, positions.shape
    if len(q_shape) != 3 or len(k_shape) != 3 or k_shape[0] != q_shape[0] or k_shape[2] != q_shape[2]:
        raise ValueError("expected q [tokens, q_heads, head_dim] and k [tokens, kv_heads, head_dim]")
    n, hq, d = q_shape
    axes = pos_shape[0] if len(pos_shape) == 2 else 1
    if len(pos_shape) not in (1, 2) or pos_shape[-1] != n or (n > 1 and positions.stride(-1) != 1):
        raise ValueError("positions are [tokens] or [axes, tokens] with contiguous tokens")
    if inv_freq.dim() != 1 or not inv_freq.is_contiguous():
        raise ValueError("inv_freq is a contiguous [rot_dim / 2] tensor")
    for w in (q_weight, k_weight):
        if w is not None:
            if w.dtype != dtype:
                raise TypeError("q, k and the norm weights must share an element type")
            if w.dim() != 1 or w.shape[0] != d or not w.is_contiguous():
                raise ValueError("norm weights are contiguous [head_dim] tensors")
    pairs = inv_freq.shape[0]
    if pair_axis is not None:
        pair_axis = _axis_bytes(pair_axis, pairs)
    return RopeDesc(hq, k_shape[1], d, 2 * pairs, axes, pair_axis, eps, code)


def _axis_stride(positions) -> int:
    return positions.stride(0) if positions.dim() == 2 and positions.shape[0] > 1 else positions.shape[-1]


def _rope_out(given, like):
    if given is None:
        return _torch().empty_like(like, memory_format=_torch().contiguous_format)
    if given.shape != like.shape or given.dtype != like.dtype:
        raise ValueError("an output has the shape and element type of its input")
    return given


@_in_call_context
def qk_norm_rope(q, k, positions, inv_freq, q_weight=None, k_weight=None, pair_axis=None, eps: float = 1e-6, q_out=None,
                 k_out=None, stream=None):
    """rpx_qk_norm_rope: RMS norm per head (with weights) and rotation by position of queries and keys, in one pass.

    q [T, H_q, d], k [T, H_kv, d]; positions int32 [T] or [axes, T]; inv_freq float32 [rot_dim / 2]; pair_axis: the axis of
    each pair, a sequence or array on the host (see ``mrope_pair_axis``), None = axis 0; weights [d] or both None (rotation only).  ``q_out`` / ``k_out``
    may be q / k themselves.  Returns (q_out, k_out)."""
    lib = load_library()
    _one_device(q, k, positions, inv_freq, q_weight, k_weight, q_out, k_out)
    desc = _rope_desc(q, k, positions, inv_freq, q_weight, k_weight, pair_axis, eps)
    q_out, k_out = _rope_out(q_out, q), _rope_out(k_out, k)
    rc = lib.rpx_qk_norm_rope(ctypes.byref(desc), q.data_ptr(), k.data_ptr(), _tok_stride(q), _tok_stride(k), _ptr(q_weight),
                              _ptr(k_weight), positions.data_ptr(), _axis_stride(positions), inv_freq.data_ptr(), q.shape[0],
                              q_out.data_ptr(), k_out.data_ptr(), _tok_stride(q_out), _tok_stride(k_out), _stream_ptr(stream))
    if rc != 0:
        raise RpxError(rc, "rpx_qk_norm_rope")
    return q_out, k_out


@_in_call_context
def qk_norm_rope_backward(q, k, dq, dk, positions, inv_freq, q_weight=None, k_weight=None, pair_axis=None, eps: float = 1e-6,
                          dq_in=None, dk_in=None, dq_weight=None, dk_weight=None, accumulate_dw: bool = False,
                          workspace=None, stream=None):
    """rpx_qk_norm_rope_backward: from float32 dq, dk with respect to the outputs (as ``attn_backward`` returns them) to the
    gradients of q, k (their element type) and of the norm weights (float32, added to the given buffers with
    ``accumulate_dw``).  Returns (dq_in, dk_in, dq_weight, dk_weight), the last two None without weights."""
    torch = _torch()
    lib = load_library()
    _one_device(q, k, dq, dk, positions, inv_freq, q_weight, k_weight, dq_in, dk_in, dq_weight, dk_weight, workspace)
    desc = ctypes.byref(_rope_desc(q, k, positions, inv_freq, q_weight, k_weight, pair_axis, eps))
    for g, x in ((dq, q), (dk, k)):
        if g.dtype != torch.float32 or g.shape != x.shape or not g.is_contiguous():
            raise ValueError("dq and dk are contiguous float32 tensors of the shapes of q and k")
    dq_in, dk_in = _rope_out(dq_in, q), _rope_out(dk_in, k)
    tokens, _, d = q.shape
    ws, ws_bytes = None, 0
    if q_weight is not None:
        if accumulate_dw and (dq_weight is None or dk_weight is None):
            raise ValueError("accumulate_dw needs the dq_weight and dk_weight buffers to add to")
        if dq_weight is None:
            dq_weight = torch.empty(d, dtype=torch.float32, device=q.device)
        if dk_weight is None:
            dk_weight = torch.empty(d, dtype=torch.float32, device=q.device)
        for w in (dq_weight, dk_weight):
            if w.dtype != torch.float32 or w.dim() != 1 or w.shape[0] != d or not w.is_contiguous():
                raise ValueError("weight gradients are contiguous float32 [head_dim] tensors")
        ws = _workspace(lib.rpx_qk_norm_rope_backward_workspace_bytes(desc, tokens), q.device, workspace)
        ws_bytes = ws.nbytes
    rc = lib.rpx_qk_norm_rope_backward(desc, q.data_ptr(), k.data_ptr(), _tok_stride(q), _tok_stride(k), _ptr(q_weight),
                                       _ptr(k_weight), positions.data_ptr(), _axis_stride(positions), inv_freq.data_ptr(),
                                       dq.data_ptr(), dk.data_ptr(), tokens, dq_in.data_ptr(), dk_in.data_ptr(),
                                       _tok_stride(dq_in), _tok_stride(dk_in), _ptr(dq_weight), _ptr(dk_weight),
                                       1 if accumulate_dw else 0, _ptr(ws), ws_bytes, _stream_ptr(stream))
    if rc != 0:
        raise RpxError(rc, "rpx_qk_norm_rope_backward")
    return dq_in, dk_in, dq_weight, dk_weight


# ------------------------------------------------------------------ pages of the cache
def _page_pool(block_table, lens, ref_counts) -> PagePool:
    i32 = _torch().int32
    if block_table.dtype != i32 or ref_counts.dtype != i32 or (lens is not None and lens.dtype != i32):
        raise TypeError("block_table, lens and ref_counts are int32")
    shape = block_table.shape
    if len(shape) != 2:
        raise ValueError("block_table is [rows, pages] with contiguous rows")
    rows, cols = shape
    stride = block_table.stride()
    if cols > 1 and stride[1] != 1:
        raise ValueError("block_table is [rows, pages] with contiguous rows")
    if not ref_counts.is_contiguous() or (lens is not None and (lens.numel() != rows or not lens.is_contiguous())):
        raise ValueError("ref_counts [num_blocks] and lens [rows] are contiguous")
    return PagePool(block_table.data_ptr(), stride[0] if rows > 1 else cols, cols, rows, _ptr(lens), ref_counts.data_ptr(),
                    ref_counts.numel())


def _row_list(t):
    if t.dtype != _torch().int32 or t.dim() != 1 or not t.is_contiguous():
        raise TypeError("row, page and token lists are contiguous int32 tensors")
    return t


def _first(t, n):
    """What a call wrote of a caller's buffer that may be longer: what lies behind is of an earlier call."""
    return t if t.numel() == n else t[:n]


@_in_call_context
def pages_free(block_table, lens, ref_counts, rows, device_status=None, stream=None) -> None:
    """rpx_pages_free: the listed rows give up their pages (reference counts go down, entries become -1, lens 0)."""
    _one_device(block_table, lens, ref_counts, rows, device_status)
    pool = ctypes.byref(_page_pool(block_table, lens, ref_counts))
    rc = load_library().rpx_pages_free(pool, _row_list(rows).data_ptr(), rows.numel(), _ptr(device_status), _stream_ptr(stream))
    if rc != 0:
        raise RpxError(rc, "rpx_pages_free")


@_in_call_context
def pages_fork(block_table, lens, ref_counts, src_rows, dst_rows, extra_tokens: int = 0, copy_src=None, copy_dst=None,
               workspace=None, device_status=None, stream=None):
    """rpx_pages_fork: empty rows ``dst`` become branches of rows ``src`` (-1: new sequences; src == dst: the row grows), whole
    pages shared, with fresh pages for the partial last one and ``extra_tokens`` more.

    Returns (copy_src, copy_dst) int32 [n], the first n entries of buffers that are given: the partial pages to copy in every
    layer (``cache_copy_pages``), -1 where none."""
    torch = _torch()
    lib = load_library()
    _one_device(block_table, lens, ref_counts, src_rows, dst_rows, copy_src, copy_dst, workspace, device_status)
    pool = ctypes.byref(_page_pool(block_table, lens, ref_counts))
    n = _row_list(src_rows).numel()
    if _row_list(dst_rows).numel() != n:
        raise ValueError("src_rows and dst_rows have one entry per request")
    if copy_src is None:
        copy_src = torch.empty_like(src_rows)
    elif _row_list(copy_src).numel() < n:
        raise ValueError("copy_src and copy_dst have one entry per request")
    if copy_dst is None:
        copy_dst = torch.empty_like(src_rows)
    elif _row_list(copy_dst).numel() < n:
        raise ValueError("copy_src and copy_dst have one entry per request")
    ws = _workspace(lib.rpx_pages_fork_workspace_bytes(pool, n), block_table.device, workspace)
    rc = lib.rpx_pages_fork(pool, src_rows.data_ptr(), dst_rows.data_ptr(), n, _bound(extra_tokens), copy_src.data_ptr(),
                            copy_dst.data_ptr(), ws.data_ptr(), ws.nbytes, _ptr(device_status), _stream_ptr(stream))
    if rc != 0:
        raise RpxError(rc, "rpx_pages_fork")
    return _first(copy_src, n), _first(copy_dst, n)


@_in_call_context
def pages_compact(block_table, ref_counts, table_out=None, ref_counts_out=None, copy_src=None, copy_dst=None, n_live=None,
                  workspace=None, device_status=None, stream=None):
    """rpx_pages_compact: live pages move to the low end of the pool; the table and the counts are rewritten, in place unless
    outputs are given.

    Returns (copy_src, copy_dst, n_live): the moves for ``cache_copy_pages`` (int32 [num_blocks // 2], -1 behind the last; the
    first entries of buffers that are given) and the number of live pages (int32 [1])."""
    torch = _torch()
    lib = load_library()
    _one_device(block_table, ref_counts, table_out, ref_counts_out, copy_src, copy_dst, n_live, workspace, device_status)
    pool = ctypes.byref(_page_pool(block_table, None, ref_counts))
    blocks = ref_counts.numel()
    table_out = block_table if table_out is None else table_out
    ref_counts_out = ref_counts if ref_counts_out is None else ref_counts_out
    out = _page_pool(table_out, None, ref_counts_out)
    if table_out.shape != block_table.shape or ref_counts_out.numel() != blocks:
        raise ValueError("table_out and ref_counts_out have the shapes of block_table and ref_counts")
    moves, dev = blocks // 2, block_table.device
    if copy_src is None:
        copy_src = torch.empty(moves, dtype=torch.int32, device=dev)
    if copy_dst is None:
        copy_dst = torch.empty(moves, dtype=torch.int32, device=dev)
    if n_live is None:
        n_live = torch.empty(1, dtype=torch.int32, device=dev)
    if _row_list(copy_src).numel() < moves or _row_list(copy_dst).numel() < moves or _row_list(n_live).numel() < 1:
        raise ValueError("copy_src and copy_dst have num_blocks // 2 entries, n_live one")
    ws = _workspace(lib.rpx_pages_compact_workspace_bytes(pool), dev, workspace)
    rc = lib.rpx_pages_compact(pool, out.block_table, out.block_table_stride, out.ref_counts, copy_src.data_ptr(),
                               copy_dst.data_ptr(), n_live.data_ptr(), ws.data_ptr(), ws.nbytes, _ptr(device_status),
                               _stream_ptr(stream))
    if rc != 0:
        raise RpxError(rc, "rpx_pages_compact")
    return _first(copy_src, moves), _first(copy_dst, moves), _first(n_live, 1)


@_in_call_context
def cache_copy_pages(k_cache, v_cache, src, dst, device_status=None, stream=None) -> None:
    """rpx_cache_copy_pages: page src[i] -> page dst[i] of both pools (pairs of -1 skipped).

    Pools bfloat16 [num_blocks, H_kv, 16, d], or [layers, num_blocks, H_kv, 16, d] for all layers at once."""
    bf16 = _torch().bfloat16
    _one_device(k_cache, v_cache, src, dst, device_status)
    if k_cache.dtype != bf16 or v_cache.dtype != bf16:
        raise TypeError("cache pools are bfloat16")
    shape = k_cache.shape
    if v_cache.shape != shape or len(shape) not in (4, 5) or shape[-2] != BLOCK_SIZE:
        raise ValueError("cache pools are [(layers,) blocks, kv_heads, 16, head_dim], K and V alike")
    if not (k_cache.is_contiguous() and v_cache.is_contiguous()):
        raise ValueError("cache pools must be contiguous")
    blocks, heads, _, d = shape[-4:]
    n = _row_list(src).numel()
    if _row_list(dst).numel() != n:
        raise ValueError("src and dst have one entry per pair")
    rc = load_library().rpx_cache_copy_pages(k_cache.data_ptr(), v_cache.data_ptr(), shape[0] if len(shape) == 5 else 1,
                                             blocks * heads * BLOCK_SIZE * d, blocks, heads, d, src.data_ptr(), dst.data_ptr(), n,
                                             _ptr(device_status), _stream_ptr(stream))
    if rc != 0:
        raise RpxError(rc, "rpx_cache_copy_pages")


@_in_call_context
def cache_append(k, v, cu_append, cached_lens, max_append: int, cache: Tuple, token_ids=None, device_status=None,
                 stream=None) -> None:
    """rpx_cache_append: K and V of tokens ``token_ids[cu_append[s]:cu_append[s + 1]]`` (or of the tokens of that range
    themselves) are stored at positions cached_lens[s], cached_lens[s] + 1, .. of sequence s; cached_lens stays as it is."""
    _one_device(k, v, cu_append, cached_lens, *cache, token_ids, device_status)
    cs = _cache_struct(cache)
    shape = k.shape
    if len(shape) != 3:
        raise ValueError("k and v are [tokens, kv_heads, head_dim] tensors that fit the cache pools")
    tokens, heads, d = shape
    if v.shape != shape or v.dtype != k.dtype or cache[0].shape[1:] != (heads, BLOCK_SIZE, d):
        raise ValueError("k and v are [tokens, kv_heads, head_dim] tensors that fit the cache pools")
    batch = _row_list(cached_lens).numel()
    if _row_list(cu_append).numel() != batch + 1 or cache[2].shape[0] < batch:
        raise ValueError("cu_append has one entry more than cached_lens, and the block table a row for each sequence")
    ids, n_ids = None, 0
    if token_ids is not None:
        # (an empty list has no pointer, and NULL stands for no list)
        ids, n_ids = _row_list(token_ids).data_ptr() or cu_append.data_ptr(), token_ids.numel()
    rc = load_library().rpx_cache_append(k.data_ptr(), v.data_ptr(), _tok_stride(k), _tok_stride(v), tokens, heads, d,
                                         _dtype_code(k), ids, n_ids, cu_append.data_ptr(), cached_lens.data_ptr(), batch,
                                         _bound(max_append), ctypes.byref(cs), _ptr(device_status), _stream_ptr(stream))
    if rc != 0:
        raise RpxError(rc, "rpx_cache_append")
