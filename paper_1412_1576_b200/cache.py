"""Operators on a paged cache of keys and values, for callers that hold torch tensors.

What the target model of drafted tokens needs before ``rows.verify_drafts`` can look at its probabilities: who sees whom in a tree of drafts
(``tree_mask``), their keys and values into the cache with the position rotation on the way (``append_cache``), and their attention over
the cache (``tree_attention``), which is also that of an ordinary decoding step, one token per sequence.  Argument checks and outputs only: the
work is done by the entry points of the same names in ``include/lda_b200.h``, queued on the current stream of the tensors' device.  There is no
fallback: tensors that are not on a GPU are refused, and so are tracing and tensors that autograd follows (there is no backward pass).

A cache is a pair of tensors [pages, page_size, kv_heads, dim] in float16 or bfloat16, of any strides that are multiples of 16 bytes and at most
2^31 elements (so one that lies head by head is handed over as a transposed view).  ``table``: int32 [sequences, most pages], the pages of each
sequence in order; ``starts``: int32 [sequences], the slots that a sequence has before its new tokens; ``offsets``: int64 [sequences + 1], where
each sequence's new tokens begin among those of the call (a sequence whose own two do not run upwards inside the tokens is left out).
"""

from __future__ import annotations

from struct import Struct

import torch
from torch.autograd import forward_ad
from torch.autograd.graph import increment_version

from . import binding as _b
from .rows import _call, _cuda as _on_gpu, _here, _vector

_DTYPES = {torch.float16: _b.LDA_F16, torch.bfloat16: _b.LDA_BF16}
# an lda_paged_cache (five microseconds less than filling the structure field by field, where a small call takes ten on the GPU)
_pack_cache = Struct("@PPiiiiqqqqqqqPqqPPi4x").pack
_WHAT = "operators on a cache"


def _cuda(x, name):
    return _on_gpu(x, name, _WHAT)


def _unfollowed(**tensors):
    """Refuses what autograd would have to follow."""
    grad, forward = torch.is_grad_enabled(), forward_ad._current_level >= 0
    if not grad and not forward:
        return
    for name, x in tensors.items():
        if x is not None and (grad and x.requires_grad or forward and forward_ad.unpack_dual(x).tangent is not None):
            raise ValueError(f"{name}: {_WHAT} are not differentiable (detach it)")


def _memory(x, name):
    """A tensor's address; it has one, on a multiple of 16 bytes."""
    address = x.data_ptr()
    if address % 16 or not address and x.numel():
        raise ValueError(f"{name}: must start at a multiple of 16 bytes, in memory of its own")
    return address


def _steps(x, name):
    """Strides but the last of a tensor whose last dimension is consecutive; those of dimensions of one are never taken."""
    *between, step = x.stride()
    if step != 1 and x.numel():
        raise ValueError(f"{name}: the values of a head must be consecutive in memory")
    steps = [s if n > 1 else 0 for s, n in zip(between, x.shape)]
    if any(s % 8 for s in steps):
        raise ValueError(f"{name}: strides must be multiples of 16 bytes, not {tuple(x.stride())}")
    return steps


def _heads(x, name, dtype, tokens, dim, device):
    """Checks rows of heads; returns (their number, address, token stride, head stride)."""
    shape = x.shape
    if x.dtype is dtype and len(shape) == 3 and x.device == device:
        n, heads, values = shape
        if values == dim and (tokens is None or n == tokens):
            # (what most calls bring)
            address, (between, step, one) = x.data_ptr(), x.stride()
            if one == 1 and not (between | step) & 7 and not address & 15 and address:
                return heads, address, between, step
    if x.dtype is not dtype:
        raise TypeError(f"{name}: the cache's {dtype} is needed, not {x.dtype}")
    if len(shape) != 3 or shape[2] != dim or tokens is not None and shape[0] != tokens:
        raise ValueError(f"{name}: [{'tokens' if tokens is None else tokens}, heads, {dim}] is needed, not {tuple(shape)}")
    _here(x, name, device)
    return (shape[1], _memory(x, name), *_steps(x, name))


def _cache(k_cache, v_cache, table, starts, offsets, device):
    """Checks a cache and its sequences; returns the library's description of them, and the cache's type, heads and their values."""
    dtype, shape = k_cache.dtype, k_cache.shape
    code = _DTYPES.get(dtype)
    if code is None:
        raise TypeError(f"k_cache: float16 or bfloat16 is needed, not {dtype}")
    if v_cache.dtype is not dtype:
        raise TypeError(f"v_cache: {dtype} is needed, not {v_cache.dtype}")
    if len(shape) != 4 or v_cache.shape != shape or 0 in shape[1:3]:
        raise ValueError(f"k_cache and v_cache: [pages, page_size, kv_heads, dim] is needed, not {tuple(shape)} and {tuple(v_cache.shape)}")
    pages, page_size, heads, dim = shape
    if dim < 8 or dim & 7 or dim > _b.LDA_HEAD_MAX_DIM:
        raise ValueError(f"k_cache: heads of a multiple of 8 values up to {_b.LDA_HEAD_MAX_DIM} are needed, not {dim}")
    if heads > _b.LDA_HEADS_MAX:
        raise ValueError(f"k_cache: up to {_b.LDA_HEADS_MAX} heads, not {heads}")
    if k_cache.device != device or v_cache.device != device or table.device != device:
        _here(k_cache, "k_cache", device), _here(v_cache, "v_cache", device), _here(table, "table", device)
    (k0, k1, k2, k3), (v0, v1, v2, v3) = k_cache.stride(), v_cache.stride()
    keys, values = k_cache.data_ptr(), v_cache.data_ptr()
    if k3 != 1 or v3 != 1 or (k0 | k1 | k2 | v0 | v1 | v2) & 7 or not keys or not values or (keys | values) & 15:
        (k0, k1, k2), (v0, v1, v2) = _steps(k_cache, "k_cache"), _steps(v_cache, "v_cache")
        keys, values = _memory(k_cache, "k_cache"), _memory(v_cache, "v_cache")
    n, grid = offsets.shape, table.shape
    if len(n) != 1 or n[0] < 1:
        raise ValueError("offsets: one more than there are sequences is needed")
    n = n[0] - 1
    if table.dtype is not torch.int32:
        raise TypeError(f"table: int32 is needed, not {table.dtype}")
    if len(grid) != 2 or grid[0] != n:
        raise ValueError(f"table: a row for each of {n} sequences is needed, not {tuple(grid)}")
    width, (between, step) = grid[1], table.stride()
    if width > 1 and step != 1:
        raise ValueError("table: the pages of a sequence must be consecutive in memory")
    if width * page_size > 0x7FFFFFFF:
        raise ValueError("table: a sequence has less than 2^31 slots")
    return _pack_cache(keys, values, code, heads, dim, page_size, pages, k0, k1, k2, v0, v1, v2, table.data_ptr(), between if n > 1 else 0, n,
                       _vector(starts, "starts", torch.int32, n, device), _vector(offsets, "offsets", torch.int64, n + 1, device),
                       width), dtype, heads, dim


def tree_mask(parents, offsets, starts, nodes: int):
    """Who sees whom in trees of drafted tokens, and the tokens' positions: (mask int64 [tokens, words], positions int32 [tokens]).

    parents: int32 [tokens], a token's parent by its place in its own sequence; a parent stands before its children, and any
    other number marks a token that follows the context itself.  nodes: as many tokens as the longest sequence has, or more; words =
    ceil(nodes / 64) and bit j % 64 of word j / 64 stands for the token at place j.  A token sees itself and all above it;
    its position is starts[sequence] and one for each above it.  starts: int32 [sequences], None for 0.  Rows of tokens that belong to no
    sequence are undefined.
    """
    device = _cuda(parents, "parents")
    if not 1 <= nodes <= 64 * _b.LDA_MASK_MAX_WORDS:
        raise ValueError(f"nodes: 1 to {64 * _b.LDA_MASK_MAX_WORDS}, not {nodes}")
    if offsets.dim() != 1 or offsets.shape[0] < 1:
        raise ValueError("offsets: one more than there are sequences is needed")
    n, tokens, words = offsets.shape[0] - 1, parents.numel(), (nodes + 63) // 64
    parents_ptr = _vector(parents, "parents", torch.int32, tokens, device)
    offsets_ptr = _vector(offsets, "offsets", torch.int64, n + 1, device)
    starts_ptr = None
    if starts is not None:
        starts_ptr = _vector(starts, "starts", torch.int32, n, device)
        if not starts_ptr and n:
            raise ValueError("starts: a tensor without memory of its own")
    mask = parents.new_empty((tokens, words), dtype=torch.int64)
    positions = torch.empty_like(parents)
    _call("lda_tree_mask", device, parents_ptr, offsets_ptr, n, tokens, starts_ptr, words, mask.data_ptr(), positions.data_ptr())
    return mask, positions


def append_cache(k, v, k_cache, v_cache, table, starts, offsets, positions=None, inv_freq=None, interleaved: bool = False, q=None, q_out=None):
    """New tokens' keys and values into the cache, in the slots from ``starts`` on; keys and queries rotated by their positions on the way.

    k, v: [tokens, kv_heads, dim] in the cache's type.  inv_freq: float32 [n], None for no rotation: of a head's first 2 n values pair i is
    turned by positions[token] * inv_freq[i]; a pair lies n values apart, or side by side (interleaved).  positions: int32 [tokens], None
    for the tokens' slots.  q: [tokens, heads, dim], rotated like the keys; q_out: where to, None for a new tensor, q itself is allowed, any other
    overlap is not.  Neither the cache nor q_out may be an expanded tensor, whose elements share their places.
    Returns the rotated queries (None without q).  Tokens of no sequence, and slots that the table has no page for, are left alone.
    """
    device = _cuda(k, "k")
    _unfollowed(k=k, v=v, q=q)
    if k_cache.requires_grad or v_cache.requires_grad or q_out is not None and q_out.requires_grad:
        raise ValueError("k_cache, v_cache and q_out: tensors that autograd follows cannot be written to (detach them)")
    cache, dtype, kv_heads, dim = _cache(k_cache, v_cache, table, starts, offsets, device)
    k_heads, *from_k = _heads(k, "k", dtype, None, dim, device)
    tokens = k.shape[0]
    v_heads, *from_v = _heads(v, "v", dtype, tokens, dim, device)
    if k_heads != kv_heads or v_heads != kv_heads:
        raise ValueError(f"k and v: the cache's {kv_heads} heads are needed, not {k_heads} and {v_heads}")
    positions_ptr = inv_freq_ptr = None
    rotated = 0
    if positions is not None:
        positions_ptr = _vector(positions, "positions", torch.int32, tokens, device)
        if not positions_ptr and tokens:
            raise ValueError("positions: a tensor without memory of its own")
    if inv_freq is not None and (pairs := inv_freq.numel()):
        inv_freq_ptr = _vector(inv_freq, "inv_freq", torch.float32, pairs, device)
        rotated = 2 * pairs
        if rotated > dim:
            raise ValueError(f"inv_freq: {dim // 2} values at most, not {pairs}")
    queries = (None, 0, 0, 0, None, 0, 0)
    given = q_out is not None
    if q is None and given:
        raise ValueError("q_out: there are no queries")
    if q is not None:
        if not given:
            q_out = torch.empty_like(q)
        elif q_out.shape != q.shape:
            raise ValueError(f"q_out: must have the queries' shape, not {tuple(q_out.shape)}")
        heads, *from_q = _heads(q, "q", dtype, tokens, dim, device)
        _, *to = _heads(q_out, "q_out", dtype, tokens, dim, device)
        if not 1 <= heads <= _b.LDA_HEADS_MAX:
            raise ValueError(f"q: 1 to {_b.LDA_HEADS_MAX} heads, not {heads}")
        queries = (*from_q, heads, *to)
    _call("lda_append_cache", device, cache, tokens, *from_k, *from_v, positions_ptr, inv_freq_ptr, rotated, int(interleaved), *queries)
    increment_version((k_cache, v_cache, q_out) if given else (k_cache, v_cache))  # (a graph that has saved them finds out)
    return q_out


def tree_attention(q, k_cache, v_cache, table, starts, offsets, mask=None, scale: float | None = None, out=None):
    """Attention of new tokens, whose keys and values ``append_cache`` has put into the cache, over the cache: [tokens, heads, dim].

    A token sees its sequence's slots before the new tokens, and of the new tokens those that its row of ``mask`` (int64 [tokens, words], as
    ``tree_mask`` makes it) names; mask None: those up to itself.  Head h of q reads head h // (heads // kv_heads) of the cache.  scale: of the scores,
    None for dim ** -0.5.  out: where to, None for a new tensor; q itself is allowed, any other overlap and expanded tensors are not.  What a token
    does not see does not touch its row, whatever it holds; a token that sees nothing gets zeros.  Rows of tokens that belong to no sequence
    stay as they are (in a new tensor: undefined).
    Waits inside the kernel are bounded; should one ever give up, the rows concerned are NaN.
    """
    device = _cuda(q, "q")
    _unfollowed(q=q, k_cache=k_cache, v_cache=v_cache)
    cache, dtype, kv_heads, dim = _cache(k_cache, v_cache, table, starts, offsets, device)
    heads, *rows = _heads(q, "q", dtype, None, dim, device)
    tokens = q.shape[0]
    if not 1 <= heads <= _b.LDA_HEADS_MAX or heads % kv_heads:
        raise ValueError(f"q: a multiple of the cache's {kv_heads} heads up to {_b.LDA_HEADS_MAX} is needed, not {heads}")
    if scale is None:
        scale = dim ** -0.5
    elif not 1e-6 <= scale <= 1e6:
        raise ValueError(f"scale: 1e-6 to 1e6, not {scale}")
    mask_ptr, mask_stride, words = None, 0, 0
    if mask is not None:
        if mask.dtype is not torch.int64:
            raise TypeError(f"mask: int64 is needed, not {mask.dtype}")
        if mask.dim() != 2 or mask.shape[0] != tokens or not 1 <= mask.shape[1] <= _b.LDA_MASK_MAX_WORDS:
            raise ValueError(f"mask: [{tokens}, 1 to {_b.LDA_MASK_MAX_WORDS} words] is needed, not {tuple(mask.shape)}")
        words = mask.shape[1]
        if words > 1 and mask.stride(1) != 1:
            raise ValueError("mask: the words of a token must be consecutive in memory")
        _here(mask, "mask", device)
        mask_ptr, mask_stride = mask.data_ptr(), mask.stride(0) if tokens > 1 else 0
        if not mask_ptr and tokens:
            raise ValueError("mask: a tensor without memory of its own")
    given = out is not None
    if not given:
        out = torch.empty_like(q)
    elif out.shape != q.shape or out.requires_grad:
        raise ValueError("out: must have the queries' shape, and autograd must not follow it")
    _, *to = _heads(out, "out", dtype, tokens, dim, device)
    size = _b.load_library().lda_tree_attention_workspace(cache, tokens, heads)
    if size < 0:
        raise _b.LdaError(size, "lda_tree_attention_workspace")
    workspace = q.new_empty(size, dtype=torch.uint8)
    _call("lda_tree_attention", device, cache, tokens, *rows, heads, mask_ptr, mask_stride, words, scale, *to, workspace.data_ptr(), size)
    if given:
        increment_version(out)
    return out
