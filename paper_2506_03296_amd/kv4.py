"""Python binding of libapex_kv4.so: a 4-bit paged KV cache on MI355X.

Argument marshalling only, as in the package's decode-attention binding; the
names and semantics follow include/apex_kv4.h.

    cache = kv4.empty_cache(num_blocks, Hkv, device)         # uint8 [num_blocks][Hkv][2176]
    kv4.append(k_new, v_new, cache, slot_mapping)            # fp16 rows in, quantised
    out = kv4.attention(q, cache, block_table, context_lens, scale, lse_out=lse)
    kv4.accumulate_weights(q, cache, block_table, context_lens, scale, lse, weights)
    kv4.evict(cache, block_table, context_lens, weights, positions, keep, sinks, recent)
    k, v = kv4.gather(cache, slot_mapping)                   # fp16 rows back

block_table int32 [B][entries per row], context_lens int32 [B]; weights fp32
and positions int32, both [num_blocks][Hkv][16], belong to the cached tokens.
All tensors are on one GPU; a call works on ``stream``, by default that device's
current stream.  A result that the call allocates belongs to the stream it works
on: to use it on another one, wait for the call there, and record_stream before it
is dropped, as with any tensor of torch's.
"""
import ctypes
import os

from . import APEX_ERR_HIP, APEX_OK, ApexError, _on, _raw_stream, _require, _result, _torch

__all__ = ["LIB_PATH", "EXPORTED_SYMBOLS", "SLAB_BYTES", "BLOCK_SIZE", "HEAD_DIM", "load_library", "last_error",
           "empty_cache", "append", "gather", "attention", "accumulate_weights", "evict",
           "attention_workspace_bytes", "evict_workspace_bytes", "release_workspace"]

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libapex_kv4.so")
EXPORTED_SYMBOLS = (
    "apex_kv4_append", "apex_kv4_gather", "apex_kv4_attention", "apex_kv4_attention_workspace_bytes",
    "apex_kv4_accumulate_weights", "apex_kv4_evict", "apex_kv4_evict_workspace_bytes",
    "apex_kv4_last_error", "apex_kv4_release_workspace",
)
SLAB_BYTES = 2176
BLOCK_SIZE = 16
HEAD_DIM = 128

_LIB = None


def load_library(path=None):
    """Load (once) and return the ctypes handle of libapex_kv4.so."""
    global _LIB
    if _LIB is not None and path is None:
        return _LIB
    p = path or LIB_PATH
    try:
        import torch  # noqa: F401  (its HIP runtime is the one to bind to)
    except ImportError:
        pass
    if not os.path.exists(p):
        raise ApexError(APEX_ERR_HIP, f"{p} is not built; run __graft_entry__.build() "
                                      "(python -m paper_2506_03296_amd.build)")
    lib = ctypes.CDLL(p)
    vp, i32, i64, f32, size = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
    for name, res, args in (
            ("apex_kv4_append", i32, [vp, vp, i64, vp, vp, vp, vp, vp, i32, i32, i32, i32, i64, vp]),
            ("apex_kv4_gather", i32, [vp, vp, vp, vp, i32, i32, i32, i32, i64, vp]),
            ("apex_kv4_attention", i32, [vp, vp, vp, i64, vp, vp, vp, i32, i32, i32, i32, i32, i64, f32, vp, size, vp]),
            ("apex_kv4_attention_workspace_bytes", size, [i32, i32, i32]),
            ("apex_kv4_accumulate_weights", i32, [vp, vp, vp, i64, vp, vp, vp, i32, i32, i32, i32, i32, i64, f32, vp]),
            ("apex_kv4_evict", i32, [vp, vp, i64, vp, vp, vp, i32, i32, i32, i32, i64, i32, i32, i32, vp, size, vp]),
            ("apex_kv4_evict_workspace_bytes", size, [i32, i32, i64]),
            ("apex_kv4_last_error", ctypes.c_char_p, []),
            ("apex_kv4_release_workspace", i32, [])):
        f = getattr(lib, name)
        f.restype, f.argtypes = res, args
    if path is None:
        _LIB = lib
    return lib


def last_error():
    return load_library().apex_kv4_last_error().decode()


def _check(rc):
    if rc != APEX_OK:
        raise ApexError(rc, last_error())


def _call(name, index, *args):
    """The entry point, with the tensors' device (its index) current."""
    f = getattr(_LIB or load_library(), name)
    torch = _torch()
    if torch._C._cuda_getDevice() == index:
        rc = f(*args)
    else:
        with torch.cuda.device(index):
            rc = f(*args)
    if rc:
        _check(rc)


def release_workspace():
    _check(load_library().apex_kv4_release_workspace())


def attention_workspace_bytes(B, Hq, Hkv):
    """Bytes of an attention workspace on the current device (0: bad shapes)."""
    return int(load_library().apex_kv4_attention_workspace_bytes(B, Hq, Hkv))


def evict_workspace_bytes(B, Hkv, block_table_stride):
    return int(load_library().apex_kv4_evict_workspace_bytes(B, Hkv, block_table_stride))


def empty_cache(num_blocks, Hkv, device):
    """An uninitialised cache for num_blocks blocks of 16 tokens."""
    torch = _torch()
    return torch.empty((num_blocks, Hkv, SLAB_BYTES), dtype=torch.uint8, device=device)


def _want(t, name, dtype, shape, device, index):
    """An error unless t is a contiguous tensor of this dtype and shape on the
    device (of that index)."""
    if not (t.dtype is dtype and t.shape == shape and t.is_cuda and t.get_device() == index and t.is_contiguous()):
        _require(t, name, dtype, device, shape=shape)


def _cache(kv_cache):
    """(num_blocks, Hkv, device, index) of a cache."""
    torch = _torch()
    shape = kv_cache.shape
    if len(shape) != 3 or shape[2] != SLAB_BYTES:
        raise ValueError(f"kv_cache must be [num_blocks][Hkv][{SLAB_BYTES}], got {tuple(shape)}")
    if not kv_cache.is_cuda:
        raise ValueError(f"kv_cache must be a GPU tensor, got {kv_cache.device}")
    if kv_cache.dtype is not torch.uint8 or not kv_cache.is_contiguous():
        _require(kv_cache, "kv_cache", torch.uint8, kv_cache.device)
    return shape[0], shape[1], kv_cache.device, kv_cache.get_device()


def _batch(block_table, context_lens, device):
    """(B, entries per table row)."""
    i32 = _torch().int32
    if block_table.dim() != 2:
        raise ValueError(f"block_table must be [B][entries per row], got {tuple(block_table.shape)}")
    B, stride = block_table.shape
    _want(block_table, "block_table", i32, (B, stride), device, device.index)
    _want(context_lens, "context_lens", i32, (B,), device, device.index)
    return B, stride


def _queries(q, B, device):
    """Hq."""
    if q.dim() != 3 or q.shape[0] != B or q.shape[2] != HEAD_DIM:
        raise ValueError(f"q must be [B={B}][Hq][{HEAD_DIM}], got {tuple(q.shape)}")
    _want(q, "q", _torch().float16, q.shape, device, device.index)
    return q.shape[1]


# The checks above cost 2 us of Python where a decode step's calls take 8 in
# all.  _plain answers the common case -- everything as it must be -- with a few
# attribute reads; anything else goes through the checks, which raise what they
# find.

def _plain(q, kv_cache, block_table, context_lens):
    """(B, Hq, num_blocks, Hkv, entries per table row, device index) if the
    checks accept the tensors for sure, else None."""
    torch = _torch()
    qs, cs, bs = q.shape, kv_cache.shape, block_table.shape
    if (len(qs) == 3 and len(cs) == 3 and len(bs) == 2 and q.is_cuda and qs[2] == HEAD_DIM and cs[2] == SLAB_BYTES
            and bs[0] == qs[0] and context_lens.shape == (qs[0],) and q.dtype is torch.float16
            and kv_cache.dtype is torch.uint8 and block_table.dtype is torch.int32 and context_lens.dtype is torch.int32):
        i = q.get_device()
        if (kv_cache.get_device() == i and block_table.get_device() == i and context_lens.get_device() == i
                and q.is_contiguous() and kv_cache.is_contiguous() and block_table.is_contiguous()
                and context_lens.is_contiguous()):
            return qs[0], qs[1], cs[0], cs[1], bs[1], i
    return None


def _step(q, kv_cache, block_table, context_lens):
    """As _plain, with an error for what is not so."""
    plain = _plain(q, kv_cache, block_table, context_lens)
    if plain is not None:
        return plain
    nb, Hkv, dev, index = _cache(kv_cache)
    B, stride = _batch(block_table, context_lens, dev)
    return B, _queries(q, B, dev), nb, Hkv, stride, index


def _workspace(workspace, device):
    if not (_on(workspace, _torch().uint8, device.index) and workspace.is_contiguous()):
        _require(workspace, "workspace", _torch().uint8, device)
    return workspace.data_ptr(), workspace.numel()


def append(k_new, v_new, kv_cache, slot_mapping, token_positions=None, positions=None, weights=None, stream=None):
    """apex_kv4_append over torch tensors (in place on the cache).

    k_new/v_new: fp16 [T][Hkv][128] with unit strides inside a token (the token
    stride may be wider, e.g. views into a fused QKV buffer, but must be the
    same for both); slot_mapping int64 [T] (negative = padding);
    token_positions int32 [T] go to ``positions``; ``weights`` of the slots
    become 0."""
    torch = _torch()
    nb, Hkv, dev, index = _cache(kv_cache)
    f16 = torch.float16
    if k_new.dim() != 3 or v_new.shape != k_new.shape or k_new.shape[1] != Hkv or k_new.shape[2] != HEAD_DIM:
        raise ValueError(f"k_new and v_new must both be [T][Hkv={Hkv}][{HEAD_DIM}]")
    T = k_new.shape[0]
    if not (k_new.dtype is f16 and v_new.dtype is f16 and k_new.is_cuda and v_new.is_cuda
            and k_new.get_device() == index and v_new.get_device() == index):
        _require(k_new, "k_new", f16, dev, contiguous=False)
        _require(v_new, "v_new", f16, dev, contiguous=False)
    ks, vs = k_new.stride(), v_new.stride()
    if ks[2] != 1 or vs[2] != 1 or (Hkv > 1 and (ks[1] != HEAD_DIM or vs[1] != HEAD_DIM)):
        raise ValueError("each token's rows must be contiguous [Hkv][d]")
    if T > 1 and (ks[0] != vs[0] or ks[0] < Hkv * HEAD_DIM):
        raise ValueError("k_new and v_new must share the token stride, at least Hkv * d")
    if not (slot_mapping.dtype is torch.int64 and slot_mapping.shape == (T,) and slot_mapping.is_cuda
            and slot_mapping.get_device() == index and slot_mapping.is_contiguous()):
        _require(slot_mapping, "slot_mapping", torch.int64, dev, shape=(T,))
    if (positions is None) != (token_positions is None):
        raise ValueError("positions and token_positions go together")
    if positions is not None:
        _want(token_positions, "token_positions", torch.int32, (T,), dev, index)
        _want(positions, "positions", torch.int32, (nb, Hkv, BLOCK_SIZE), dev, index)
    if weights is not None:
        _want(weights, "weights", torch.float32, (nb, Hkv, BLOCK_SIZE), dev, index)
    _call("apex_kv4_append", index, k_new.data_ptr(), v_new.data_ptr(), ks[0] if T > 1 else 0, kv_cache.data_ptr(),
          slot_mapping.data_ptr(), None if positions is None else token_positions.data_ptr(),
          None if positions is None else positions.data_ptr(), None if weights is None else weights.data_ptr(),
          T, Hkv, HEAD_DIM, BLOCK_SIZE, nb, _raw_stream(stream, index))


def gather(kv_cache, slot_mapping, k_out=None, v_out=None, stream=None):
    """apex_kv4_gather over torch tensors; returns (k_out, v_out), fp16
    [T][Hkv][128]: the values of the slots (int64 [T]), zeros for a slot outside
    the pool."""
    torch = _torch()
    nb, Hkv, dev, index = _cache(kv_cache)
    T = slot_mapping.numel()
    _want(slot_mapping, "slot_mapping", torch.int64, (T,), dev, index)
    shape = (T, Hkv, HEAD_DIM)
    if k_out is None:
        k_out = torch.empty(shape, dtype=torch.float16, device=dev) if stream is None else _result(shape, dev, stream)
    else:
        _want(k_out, "k_out", torch.float16, shape, dev, index)
    if v_out is None:
        v_out = torch.empty_like(k_out) if stream is None else _result(shape, dev, stream)
    else:
        _want(v_out, "v_out", torch.float16, shape, dev, index)
    _call("apex_kv4_gather", index, kv_cache.data_ptr(), slot_mapping.data_ptr(), k_out.data_ptr(), v_out.data_ptr(),
          T, Hkv, HEAD_DIM, BLOCK_SIZE, nb, _raw_stream(stream, index))
    return k_out, v_out


def attention(q, kv_cache, block_table, context_lens, scale, out=None, lse_out=None, workspace=None, stream=None):
    """apex_kv4_attention over torch tensors; returns ``out``.

    ``workspace`` is an optional uint8 tensor of attention_workspace_bytes(B,
    Hq, Hkv) bytes or more, made by torch.zeros (calls of other shapes may share
    it, an eviction may not); calls that can overlap, and a captured graph, need one of their own."""
    torch = _torch()
    B, Hq, nb, Hkv, stride, index = _step(q, kv_cache, block_table, context_lens)
    if out is None:
        out = torch.empty_like(q) if stream is None else _result(q.shape, q.device, stream)
    else:
        _want(out, "out", torch.float16, q.shape, q.device, index)
    if lse_out is not None:
        _want(lse_out, "lse_out", torch.float32, (B, Hq), q.device, index)
    ws, ws_bytes = (None, 0) if workspace is None else _workspace(workspace, q.device)
    _call("apex_kv4_attention", index, q.data_ptr(), kv_cache.data_ptr(), block_table.data_ptr(), stride,
          context_lens.data_ptr(), out.data_ptr(), None if lse_out is None else lse_out.data_ptr(), B, Hq, Hkv,
          HEAD_DIM, BLOCK_SIZE, nb, scale, ws, ws_bytes, _raw_stream(stream, index))
    return out


def accumulate_weights(q, kv_cache, block_table, context_lens, scale, lse, weights, stream=None):
    """apex_kv4_accumulate_weights over torch tensors (in place on ``weights``);
    ``lse`` fp32 [B][Hq] is the ``lse_out`` of the step's attention."""
    torch = _torch()
    B, Hq, nb, Hkv, stride, index = _step(q, kv_cache, block_table, context_lens)
    dev = q.device
    _want(lse, "lse", torch.float32, (B, Hq), dev, index)
    _want(weights, "weights", torch.float32, (nb, Hkv, BLOCK_SIZE), dev, index)
    _call("apex_kv4_accumulate_weights", index, q.data_ptr(), kv_cache.data_ptr(), block_table.data_ptr(), stride,
          context_lens.data_ptr(), lse.data_ptr(), weights.data_ptr(), B, Hq, Hkv, HEAD_DIM, BLOCK_SIZE, nb, scale,
          _raw_stream(stream, index))


def evict(kv_cache, block_table, context_lens, weights, positions, keep, sinks=0, recent=0, workspace=None,
          stream=None):
    """apex_kv4_evict over torch tensors (in place on the cache, ``weights`` and
    ``positions``).  A request longer than ``keep`` has the length ``keep``
    afterwards; context_lens is left to the caller.  In a table row with block ids
    outside the pool only the tokens in the pool count: the first ``keep`` of their
    slots hold what is kept, and the length goes up to the last of these (a request
    with no more than ``keep`` tokens in the pool keeps its length).

    ``workspace`` is an optional uint8 tensor of evict_workspace_bytes(B, Hkv,
    block_table.shape[1]) bytes; calls that can overlap, and a captured graph,
    need one of their own."""
    torch = _torch()
    if not (0 < keep < 1 << 31 and sinks >= 0 and recent >= 0 and sinks + recent <= keep):
        raise ValueError(f"keep = {keep}, sinks = {sinks}, recent = {recent}: keep must be positive (below 2^31), "
                         "sinks + recent at most keep")
    nb, Hkv, dev, index = _cache(kv_cache)
    B, stride = _batch(block_table, context_lens, dev)
    _want(weights, "weights", torch.float32, (nb, Hkv, BLOCK_SIZE), dev, index)
    _want(positions, "positions", torch.int32, (nb, Hkv, BLOCK_SIZE), dev, index)
    ws, ws_bytes = (None, 0) if workspace is None else _workspace(workspace, dev)
    _call("apex_kv4_evict", index, kv_cache.data_ptr(), block_table.data_ptr(), stride, context_lens.data_ptr(),
          weights.data_ptr(), positions.data_ptr(), B, Hkv, HEAD_DIM, BLOCK_SIZE, nb, keep, sinks, recent, ws, ws_bytes,
          _raw_stream(stream, index))
