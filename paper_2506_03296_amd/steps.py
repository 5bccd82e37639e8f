"""Python binding of libapex_steps.so: steps with several new tokens a request
on MI355X -- prompts, trees of drafted tokens, and the cache blocks they take.

Argument marshalling only, as in the package's decode-attention binding; the
names and semantics follow include/apex_steps.h.

    free_blocks, free_state = steps.new_pool(num_blocks, device)      # every block is free
    plan = steps.extend(context_lens, new_lens, block_table, free_blocks, free_state, T)
    out = steps.prompt_attention(q, k, v, plan.token_offsets, scale)  # packed prompts
    kv_append(k, v, k_cache, v_cache, plan.slot_mapping)
    out = steps.tree_attention(q, k_new, v_new, token_offsets, tree_mask, k_cache, v_cache, block_table,
                               context_lens, max_nodes, scale)        # drafted tokens
    steps.release(context_lens, keep_lens, block_table, free_blocks, free_state)

q fp16 [T][Hq][128], K and V rows fp16 [T][Hkv][128], caches fp16
[num_blocks][Hkv][16][128], block_table int32 [B][entries per row], lengths int32
[B], token_offsets int32 [B + 1], tree_mask int64 [T].  All tensors are on one
GPU; a call works on ``stream``, by default that device's current stream.  A
result that the call allocates belongs to the stream it works on: to use it on
another one, wait for the call there, and record_stream before it is dropped, as
with any tensor of torch's.
"""
import ctypes
import os
from typing import NamedTuple

from . import APEX_ERR_HIP, APEX_OK, ApexError, _on, _raw_stream, _require, _result, _torch

__all__ = ["LIB_PATH", "EXPORTED_SYMBOLS", "BLOCK_SIZE", "HEAD_DIM", "MAX_NODES", "Plan", "load_library", "last_error",
           "new_pool", "empty_plan", "extend", "release", "prompt_attention", "tree_attention", "tree_workspace_bytes",
           "release_workspace"]

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libapex_steps.so")
EXPORTED_SYMBOLS = (
    "apex_steps_extend", "apex_steps_release", "apex_steps_prompt_attention", "apex_steps_tree_attention",
    "apex_steps_tree_workspace_bytes", "apex_steps_last_error", "apex_steps_release_workspace",
)
BLOCK_SIZE = 16
HEAD_DIM = 128
MAX_NODES = 64

_LIB = None


class Plan(NamedTuple):
    """What ``extend`` writes for a batch's new tokens."""
    token_offsets: object     # int32 [B + 1]
    total_lens: object        # int32 [B]
    slot_mapping: object      # int64 [T]
    token_positions: object   # int32 [T]


def load_library(path=None):
    """Load (once) and return the ctypes handle of libapex_steps.so."""
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
            ("apex_steps_extend", i32, [vp, vp, vp, i64, vp, vp, vp, vp, vp, vp, i32, i32, i32, i64, vp]),
            ("apex_steps_release", i32, [vp, vp, vp, i64, vp, vp, i32, i32, i64, vp]),
            ("apex_steps_prompt_attention", i32,
             [vp, i64, vp, vp, i64, vp, vp, vp, i32, i32, i32, i32, i32, f32, vp]),
            ("apex_steps_tree_attention", i32,
             [vp, i64, vp, vp, i64, vp, vp, vp, vp, vp, i64, vp, vp, vp, i32, i32, i32, i32, i32, i32, i32, i64, f32,
              vp, size, vp]),
            ("apex_steps_tree_workspace_bytes", size, [i32, i32, i32]),
            ("apex_steps_last_error", ctypes.c_char_p, []),
            ("apex_steps_release_workspace", i32, [])):
        f = getattr(lib, name)
        f.restype, f.argtypes = res, args
    if path is None:
        _LIB = lib
    return lib


def last_error():
    return load_library().apex_steps_last_error().decode()


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
    _check(load_library().apex_steps_release_workspace())


def tree_workspace_bytes(max_nodes, Hq, Hkv):
    """Bytes of a tree attention's workspace on the current device (0: bad shapes)."""
    for x, name in ((max_nodes, "max_nodes"), (Hq, "Hq"), (Hkv, "Hkv")):
        _c_int(x, name)
    return int(load_library().apex_steps_tree_workspace_bytes(max_nodes, Hq, Hkv))


def _c_int(x, name):
    """An error unless x fits a C int, which ctypes would cut it to."""
    if not -2 ** 31 <= x < 2 ** 31:
        raise ValueError(f"{name} = {x} does not fit 32 bits")


def _want(t, name, dtype, shape, device, index):
    """An error unless t is a contiguous tensor of this dtype and shape on the
    device (of that index)."""
    if not (t.dtype is dtype and t.shape == shape and t.is_cuda and t.get_device() == index and t.is_contiguous()):
        _require(t, name, dtype, device, shape=shape)


def _words(tensors, shapes, index):
    """True if all are contiguous int32 tensors of these shapes on GPU `index`."""
    i32 = _torch().int32
    for t, shape in zip(tensors, shapes):
        if not (t.dtype is i32 and t.shape == shape and t.get_device() == index and t.is_contiguous()):
            return False
    return True


def _gpu(t, name):
    """(device, index) of a tensor that has to be on a GPU."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a GPU tensor, got {t.device}")
    return t.device, t.get_device()


def _table(block_table, B, device, index):
    """Entries per row."""
    if block_table.dim() != 2 or block_table.shape[0] != B:
        raise ValueError(f"block_table must be [B={B}][entries per row], got {tuple(block_table.shape)}")
    _want(block_table, "block_table", _torch().int32, block_table.shape, device, index)
    return block_table.shape[1]


def _rows(t, name, heads, device, index):
    """Elements between the tokens of packed rows [T][heads][128], unit strides
    inside a token (0: one token or none)."""
    f16 = _torch().float16
    if t.dim() != 3 or t.shape[1] != heads or t.shape[2] != HEAD_DIM:
        raise ValueError(f"{name} must be [T][{heads}][{HEAD_DIM}], got {tuple(t.shape)}")
    if not _on(t, f16, index):
        _require(t, name, f16, device, contiguous=False)
    T = t.shape[0]
    s = t.stride()
    if T and (s[2] != 1 or (heads > 1 and s[1] != HEAD_DIM)):
        raise ValueError(f"each token's rows of {name} must be contiguous [heads][{HEAD_DIM}]")
    if T <= 1:
        return 0
    if s[0] < heads * HEAD_DIM:
        raise ValueError(f"the tokens of {name} overlap")
    return s[0]


def _blocks(context_lens, lens, name, block_table, free_blocks, free_state, block_size):
    """Checks common to extend and release: (device, index, B, entries per table row, blocks)."""
    dev, index = _gpu(block_table, "block_table")
    B, nb, shape = context_lens.numel(), free_blocks.numel(), block_table.shape
    _c_int(B, "B")
    _c_int(block_size, "block_size")
    if not (len(shape) == 2 and shape[0] == B
            and _words((block_table, context_lens, lens, free_blocks, free_state), (shape, (B,), (B,), (nb,), (2,)), index)):
        i32 = _torch().int32
        _want(context_lens, "context_lens", i32, (B,), dev, index)
        _want(lens, name, i32, (B,), dev, index)
        _table(block_table, B, dev, index)
        _want(free_blocks, "free_blocks", i32, (nb,), dev, index)
        _want(free_state, "free_state", i32, (2,), dev, index)
    return dev, index, B, shape[1], nb


def new_pool(num_blocks, device):
    """(free_blocks, free_state) of a cache whose num_blocks blocks are all unused;
    block 0 is given out first."""
    torch = _torch()
    return (torch.arange(num_blocks - 1, -1, -1, dtype=torch.int32, device=device),
            torch.tensor([num_blocks, 0], dtype=torch.int32, device=device))


def empty_plan(B, T, device):
    """An uninitialised plan for ``extend`` to write."""
    torch = _torch()
    i32 = torch.int32
    return Plan(torch.empty(B + 1, dtype=i32, device=device), torch.empty(B, dtype=i32, device=device),
                torch.empty(T, dtype=torch.int64, device=device), torch.empty(T, dtype=i32, device=device))


def extend(context_lens, new_lens, block_table, free_blocks, free_state, T, block_size=BLOCK_SIZE, plan=None,
           stream=None):
    """apex_steps_extend over torch tensors: blocks and slots for new_lens[b] new
    tokens of every request, in a packed batch of T rows; returns the Plan (``plan``
    if given, else a new one).  ``block_table`` and ``free_state`` are updated in
    place; a request whose total_lens is not context_lens + new_lens was refused."""
    torch = _torch()
    _c_int(T, "T")
    dev, index, B, stride, nb = _blocks(context_lens, new_lens, "new_lens", block_table, free_blocks, free_state, block_size)
    if plan is None:
        if T < 0:
            raise ValueError(f"T = {T} is negative")
        if stream is None:
            plan = empty_plan(B, T, dev)
        else:
            with torch.cuda.stream(stream):
                plan = empty_plan(B, T, dev)
    else:
        i32 = torch.int32
        _want(plan.token_offsets, "token_offsets", i32, (B + 1,), dev, index)
        _want(plan.total_lens, "total_lens", i32, (B,), dev, index)
        _want(plan.slot_mapping, "slot_mapping", torch.int64, (T,), dev, index)
        _want(plan.token_positions, "token_positions", i32, (T,), dev, index)
    _call("apex_steps_extend", index, context_lens.data_ptr(), new_lens.data_ptr(), block_table.data_ptr(), stride,
          free_blocks.data_ptr(), free_state.data_ptr(), plan.token_offsets.data_ptr(), plan.total_lens.data_ptr(),
          plan.slot_mapping.data_ptr(), plan.token_positions.data_ptr(), B, T, block_size, nb,
          _raw_stream(stream, index))
    return plan


def release(context_lens, keep_lens, block_table, free_blocks, free_state, block_size=BLOCK_SIZE, stream=None):
    """apex_steps_release over torch tensors: the blocks that keep_lens[b] of a
    request's context_lens[b] tokens do not need go back to ``free_blocks``.
    ``block_table``, ``free_blocks`` and ``free_state`` are updated in place."""
    _, index, B, stride, nb = _blocks(context_lens, keep_lens, "keep_lens", block_table, free_blocks, free_state, block_size)
    _call("apex_steps_release", index, context_lens.data_ptr(), keep_lens.data_ptr(), block_table.data_ptr(), stride,
          free_blocks.data_ptr(), free_state.data_ptr(), B, block_size, nb, _raw_stream(stream, index))


# The checks of tensors cost 4 us of Python where a small batch's kernel takes 6.
# _plain answers the common case -- everything as it must be -- with a few attribute
# reads; anything else goes through the checks, which raise what they find.

def _plain(q, k, v, token_offsets):
    """(index, B, T, Hq, Hkv, q's and k's elements between tokens) if the checks
    accept the tensors for sure, else None."""
    torch = _torch()
    f16 = torch.float16
    qs, ks, os_ = q.shape, k.shape, token_offsets.shape
    if (len(qs) == 3 and len(ks) == 3 and len(os_) == 1 and os_[0] > 0 and v.shape == ks and qs[0] == ks[0] > 1
            and qs[2] == HEAD_DIM and ks[2] == HEAD_DIM and q.is_cuda and q.dtype is f16 and k.dtype is f16
            and v.dtype is f16 and token_offsets.dtype is torch.int32):
        i = q.get_device()
        if k.get_device() == i and v.get_device() == i and token_offsets.get_device() == i:
            q0, q1, q2 = q.stride()
            kt = k.stride()
            if (v.stride() == kt and q1 == HEAD_DIM and kt[1] == HEAD_DIM and q2 == 1 and kt[2] == 1
                    and q0 >= qs[1] * HEAD_DIM and kt[0] >= ks[1] * HEAD_DIM and token_offsets.is_contiguous()):
                return i, os_[0] - 1, qs[0], qs[1], ks[1], q0, kt[0]
    return None


def _packed(q, k, v, names, token_offsets):
    """As _plain, with an error for what is not so."""
    plain = _plain(q, k, v, token_offsets)
    if plain is not None:
        return plain
    dev, index = _gpu(q, "q")
    if q.dim() != 3 or k.dim() != 3:
        raise ValueError(f"q, {names[0]} and {names[1]} must be [T][heads][{HEAD_DIM}]")
    T, Hq, Hkv = q.shape[0], q.shape[1], k.shape[1]
    q_stride = _rows(q, "q", Hq, dev, index)
    k_stride, v_stride = _rows(k, names[0], Hkv, dev, index), _rows(v, names[1], Hkv, dev, index)
    if k.shape[0] != T or v.shape[0] != T:
        raise ValueError(f"q, {names[0]} and {names[1]} must have as many rows")
    if k_stride != v_stride:
        raise ValueError(f"{names[0]} and {names[1]} must share the token stride")
    B = token_offsets.numel() - 1
    if B < 0:
        raise ValueError("token_offsets must be [B + 1]")
    _want(token_offsets, "token_offsets", _torch().int32, (B + 1,), dev, index)
    return index, B, T, Hq, Hkv, q_stride, k_stride


def _outputs(q, T, Hq, index, out, lse_out, stream):
    """(out, address of lse_out)."""
    torch = _torch()
    if out is None:
        if stream is None:
            out = torch.empty((T, Hq, HEAD_DIM), dtype=torch.float16, device=q.device)
        else:
            out = _result((T, Hq, HEAD_DIM), q.device, stream)
    else:
        _want(out, "out", torch.float16, (T, Hq, HEAD_DIM), q.device, index)
    if lse_out is None:
        return out, None
    _want(lse_out, "lse_out", torch.float32, (T, Hq), q.device, index)
    return out, lse_out.data_ptr()


def prompt_attention(q, k, v, token_offsets, scale, out=None, lse_out=None, stream=None):
    """apex_steps_prompt_attention over torch tensors; returns ``out``, fp16
    [T][Hq][128]: causal attention of packed prompts over themselves.

    q [T][Hq][128], k and v [T][Hkv][128] (fp16) with unit strides inside a token;
    the token strides may be wider (views into a fused QKV buffer), k's and v's the
    same.  Rows behind token_offsets[-1] are left as they are."""
    index, B, T, Hq, Hkv, qs, ks = _packed(q, k, v, ("k", "v"), token_offsets)
    out, lse = _outputs(q, T, Hq, index, out, lse_out, stream)
    _call("apex_steps_prompt_attention", index, q.data_ptr(), qs, k.data_ptr(), v.data_ptr(), ks,
          token_offsets.data_ptr(), out.data_ptr(), lse, B, T, Hq, Hkv, HEAD_DIM, scale, _raw_stream(stream, index))
    return out


def tree_attention(q, k_new, v_new, token_offsets, tree_mask, k_cache, v_cache, block_table, context_lens, max_nodes,
                   scale, out=None, lse_out=None, workspace=None, stream=None):
    """apex_steps_tree_attention over torch tensors; returns ``out``, fp16
    [T][Hq][128]: drafted tokens over the cached ones and those drafted ones of
    their request that tree_mask (int64 [T], a bit per drafted token) names.

    ``max_nodes`` is the most drafted tokens of a request, up to 64.  ``workspace``
    is an optional uint8 tensor of tree_workspace_bytes(max_nodes, Hq, Hkv) bytes;
    calls that can overlap, and a captured graph, need one of their own."""
    torch = _torch()
    _c_int(max_nodes, "max_nodes")
    index, B, T, Hq, Hkv, qs, ks = _packed(q, k_new, v_new, ("k_new", "v_new"), token_offsets)
    dev = q.device
    _want(tree_mask, "tree_mask", torch.int64, (T,), dev, index)
    shape = k_cache.shape
    if len(shape) != 4 or shape[1] != Hkv or shape[2] != BLOCK_SIZE or shape[3] != HEAD_DIM:
        raise ValueError(f"the caches must be [num_blocks][Hkv={Hkv}][{BLOCK_SIZE}][{HEAD_DIM}], got {tuple(shape)}")
    _want(k_cache, "k_cache", torch.float16, shape, dev, index)
    _want(v_cache, "v_cache", torch.float16, shape, dev, index)
    stride = _table(block_table, B, dev, index)
    _want(context_lens, "context_lens", torch.int32, (B,), dev, index)
    ws, ws_bytes = None, 0
    if workspace is not None:
        if not (_on(workspace, torch.uint8, index) and workspace.is_contiguous()):
            _require(workspace, "workspace", torch.uint8, dev)
        ws, ws_bytes = workspace.data_ptr(), workspace.numel()
    out, lse = _outputs(q, T, Hq, index, out, lse_out, stream)
    _call("apex_steps_tree_attention", index, q.data_ptr(), qs, k_new.data_ptr(), v_new.data_ptr(), ks,
          token_offsets.data_ptr(), tree_mask.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), block_table.data_ptr(),
          stride, context_lens.data_ptr(), out.data_ptr(), lse, B, T, max_nodes, Hq, Hkv, HEAD_DIM, BLOCK_SIZE, shape[0],
          scale, ws, ws_bytes, _raw_stream(stream, index))
    return out
