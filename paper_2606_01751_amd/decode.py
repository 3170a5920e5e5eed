"""Python binding of decoding over a 4-bit KV cache (declared in include/sx_decode.h).

As in the package's other calls, the functions only marshal arguments: shapes, strides, types and the device are
checked here (ValueError), everything else by the library (SxError).  One step of a serving loop, all on one
stream:

    append_slots(ctx_lens, new_lens, free_blocks, block_table, seq_lens, cu_new, positions, slots, state)
    for every layer:
        qk_norm_rope(desc, q, k, positions, q_out, k_out, gamma_q, gamma_k, eps)
        kv4_write(desc, k_out, v, slots, pool[layer])
        kv4_attn(desc, q_out, cu_new, seq_lens, block_table, pool[layer], out, max_q, max_seqlen, workspace)

and after a request's prefill kv4_pack(desc, k_cache, v_cache, cache_blocks, pool, pool_blocks) takes its paged
cache over.
"""
from __future__ import annotations

import ctypes

import torch

from . import BF16, F32, LayerDesc, Plan, _check, _stream, lib

_TYPES = {F32: torch.float32, BF16: torch.bfloat16}


def _need(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


def _elsewhere(t) -> bool:
    at = t.get_device()      # -1: host memory
    return at < 0 or at != torch.cuda.current_device()


def _ptr(t, dtype, what: str):
    """Device pointer of a contiguous tensor of this type on the current device."""
    if t.dtype is not dtype or not t.is_contiguous() or _elsewhere(t):
        _need(t.dtype is dtype, f"{what} must be {dtype}, not {t.dtype}")
        _need(t.is_contiguous(), f"{what} must be contiguous")
        raise ValueError(f"{what} is on {t.device}, not on the current GPU")
    return t.data_ptr()


def _ints(t, what: str):
    return _ptr(t, torch.int32, what)


def _rows(desc: LayerDesc, t, heads: int, what: str):
    """(pointer, elements between rows) of [n][heads][head_dim] rows, each contiguous."""
    d = desc.head_dim
    if t.dim() != 3 or t.shape[1] != heads or t.shape[2] != d:
        raise ValueError(f"{what} must be [n][{heads}][{d}], not {list(t.shape)}")
    _need(t.dtype is _TYPES.get(desc.dtype), f"{what} is {t.dtype}, the descriptor says {_TYPES.get(desc.dtype)}")
    _need(t.stride(2) == 1 and (heads == 1 or t.stride(1) == d), f"{what}'s rows must be contiguous")
    if _elsewhere(t):
        raise ValueError(f"{what} is on {t.device}, not on the current GPU")
    return t.data_ptr(), t.stride(0) if t.shape[0] > 1 else heads * d


def _gamma(desc: LayerDesc, t, what: str):
    if t is None:
        return None
    _need(t.numel() == desc.head_dim, f"{what} must have {desc.head_dim} elements")
    return _ptr(t, _TYPES.get(desc.dtype), what)


def _pool(desc: LayerDesc, t):
    """(pointer, blocks) of a 4-bit pool [n_blocks][Hkv][17 head_dim]."""
    if t.dim() != 3 or t.shape[1] != desc.n_kv_heads or t.shape[2] != 17 * desc.head_dim:
        raise ValueError(f"pool must be [n_blocks][{desc.n_kv_heads}][{17 * desc.head_dim}], not {list(t.shape)}")
    return _ptr(t, torch.uint8, "pool"), t.shape[0]


def _cache(desc: LayerDesc, t, what: str):
    if t.dim() != 4 or t.shape[1:] != (desc.n_kv_heads, desc.block_size, desc.head_dim):
        raise ValueError(f"{what} must be [n_blocks][{desc.n_kv_heads}][{desc.block_size}][{desc.head_dim}], "
                         f"not {list(t.shape)}")
    return _ptr(t, _TYPES.get(desc.dtype), what)


def append_slots(ctx_lens, new_lens, free_blocks, block_table, seq_lens, cu_new, positions, slots, state,
                 free_head=None, block_size: int = 16, stream=None):
    """Block tables and slot maps of a step in which request r, holding ctx_lens[r] tokens, appends new_lens[r]
    (None: one each).  int32 tensors; writes block_table, seq_lens, cu_new, positions, slots and state = (next
    entry of free_blocks, tokens without a slot)."""
    n = ctx_lens.numel()
    _need(new_lens is None or new_lens.numel() == n, "new_lens and ctx_lens differ in length")
    _need(seq_lens.numel() == n and cu_new.numel() == n + 1, "seq_lens needs n and cu_new n + 1 entries")
    _need(block_table.dim() == 2 and block_table.shape[0] == n, "block_table must be [n_requests][max_blocks]")
    _need(positions.numel() == slots.numel(), "positions and slots differ in length")
    _need(state.numel() >= 2 and (free_head is None or free_head.numel() >= 1), "state needs two entries, free_head one")
    _check(lib().sx_append_slots(
        _ints(ctx_lens, "ctx_lens"), None if new_lens is None else _ints(new_lens, "new_lens"), n, block_size,
        _ints(free_blocks, "free_blocks"), free_blocks.numel(),
        None if free_head is None else _ints(free_head, "free_head"), _ints(block_table, "block_table"),
        block_table.shape[1], positions.numel(), _ints(seq_lens, "seq_lens"), _ints(cu_new, "cu_new"),
        _ints(positions, "positions"), _ints(slots, "slots"), _ints(state, "state"), _stream(stream)))


def qk_norm_rope(desc: LayerDesc, q, k, positions, q_out, k_out, gamma_q=None, gamma_k=None, eps: float = 1e-6,
                 stream=None):
    """q_out, k_out = the rows of q [n][Hq][d] and k [n][Hkv][d], normalised per head (gamma None: not) and rotated to
    positions; rows at negative positions are left alone.  Rows may lie apart (parts of one projection)."""
    n = positions.numel()
    _need(q.shape[0] == n and k.shape[0] == n and q_out.shape[0] == n and k_out.shape[0] == n,
          "q, k, positions, q_out and k_out differ in length")
    qp, q_ld = _rows(desc, q, desc.n_q_heads, "q")
    kp, k_ld = _rows(desc, k, desc.n_kv_heads, "k")
    qo, qo_ld = _rows(desc, q_out, desc.n_q_heads, "q_out")
    ko, ko_ld = _rows(desc, k_out, desc.n_kv_heads, "k_out")
    _check(lib().sx_qk_norm_rope(ctypes.byref(desc), qp, q_ld, kp, k_ld, _gamma(desc, gamma_q, "gamma_q"),
                                 _gamma(desc, gamma_k, "gamma_k"), eps, _ints(positions, "positions"), n, qo, qo_ld,
                                 ko, ko_ld, _stream(stream)))


def qk_norm_rope_rows(plan: Plan, rows, n_rows, max_rows: int, q, k, gamma_q=None, gamma_k=None, eps: float = 1e-6,
                      stream=None):
    """The same in place on the listed rows of a plan, at their positions in the new sequence (beside rope_rows)."""
    dt = _TYPES.get(plan.desc.dtype)
    _check(lib().sx_qk_norm_rope_rows(plan.handle, rows if isinstance(rows, int) else _ints(rows, "rows"),
                                      n_rows if isinstance(n_rows, int) else _ints(n_rows, "n_rows"), int(max_rows),
                                      _ptr(q, dt, "q"), _ptr(k, dt, "k"), _gamma(plan.desc, gamma_q, "gamma_q"),
                                      _gamma(plan.desc, gamma_k, "gamma_k"), eps, _stream(stream)))


def kv4_record_bytes(desc: LayerDesc) -> int:
    """Bytes of one KV head of one block: a pool is a uint8 tensor [n_blocks][Hkv][this]."""
    n = ctypes.c_int64()
    _check(lib().sx_kv4_record_bytes(ctypes.byref(desc), ctypes.byref(n)))
    return n.value


def kv4_write(desc: LayerDesc, k, v, slots, pool, stream=None):
    """Rows k, v [n][Hkv][d] rounded to 4 bits into slots of the pool (negative: skipped)."""
    n = slots.numel()
    _need(k.shape[0] == n and v.shape[0] == n, "k, v and slots differ in length")
    kp, k_ld = _rows(desc, k, desc.n_kv_heads, "k")
    vp, v_ld = _rows(desc, v, desc.n_kv_heads, "v")
    pp, nb = _pool(desc, pool)
    _check(lib().sx_kv4_write(ctypes.byref(desc), kp, k_ld, vp, v_ld, _ints(slots, "slots"), n, pp, nb, _stream(stream)))


def kv4_read(desc: LayerDesc, pool, slots, k, v, stream=None):
    """The rows that slots hold into k, v [n][Hkv][d], exactly; rows of negative slots are left alone."""
    n = slots.numel()
    _need(k.shape[0] == n and v.shape[0] == n, "k, v and slots differ in length")
    kp, k_ld = _rows(desc, k, desc.n_kv_heads, "k")
    vp, v_ld = _rows(desc, v, desc.n_kv_heads, "v")
    pp, nb = _pool(desc, pool)
    _check(lib().sx_kv4_read(ctypes.byref(desc), pp, nb, _ints(slots, "slots"), n, kp, k_ld, vp, v_ld, _stream(stream)))


def _block_args(desc, k_cache, v_cache, cache_blocks, pool, pool_blocks):
    n = cache_blocks.numel()
    _need(pool_blocks.numel() == n, "cache_blocks and pool_blocks differ in length")
    _need(k_cache.shape == v_cache.shape, "k_cache and v_cache differ in shape")
    pp, nb = _pool(desc, pool)
    return (_cache(desc, k_cache, "k_cache"), _cache(desc, v_cache, "v_cache"), k_cache.shape[0],
            _ints(cache_blocks, "cache_blocks"), n, pp, nb, _ints(pool_blocks, "pool_blocks"))


def kv4_pack(desc: LayerDesc, k_cache, v_cache, cache_blocks, pool, pool_blocks, stream=None):
    """Blocks cache_blocks[i] of a paged cache rounded to 4 bits into blocks pool_blocks[i] of the pool."""
    kc, vc, nc, cb, n, pp, nb, pb = _block_args(desc, k_cache, v_cache, cache_blocks, pool, pool_blocks)
    _check(lib().sx_kv4_pack(ctypes.byref(desc), kc, vc, nc, cb, n, pp, nb, pb, _stream(stream)))


def kv4_unpack(desc: LayerDesc, pool, pool_blocks, k_cache, v_cache, cache_blocks, stream=None):
    """Blocks pool_blocks[i] of the pool into blocks cache_blocks[i] of a paged cache, exactly."""
    kc, vc, nc, cb, n, pp, nb, pb = _block_args(desc, k_cache, v_cache, cache_blocks, pool, pool_blocks)
    _check(lib().sx_kv4_unpack(ctypes.byref(desc), pp, nb, pb, n, kc, vc, nc, cb, _stream(stream)))


def kv4_attn_workspace(desc: LayerDesc, n_requests: int, max_q: int, max_seqlen: int) -> int:
    """Bytes of workspace that kv4_attn needs for these bounds."""
    n = ctypes.c_int64()
    _check(lib().sx_kv4_attn_workspace(ctypes.byref(desc), n_requests, max_q, max_seqlen, ctypes.byref(n)))
    return n.value


def kv4_attn(desc: LayerDesc, q, cu_q, seq_lens, block_table, pool, out, max_q: int, max_seqlen: int, workspace,
             lse=None, stream=None):
    """out = causal attention of every request's last tokens (rows cu_q[r] .. cu_q[r + 1] of q) over its seq_lens[r] keys
    in the pool; lse (float32 [total_q][Hq]) their natural-log sums.  workspace: uint8, kv4_attn_workspace bytes."""
    n, total = seq_lens.numel(), q.shape[0]
    _need(cu_q.numel() == n + 1, "cu_q needs one entry more than seq_lens")
    _need(block_table.dim() == 2 and block_table.shape[0] == n, "block_table must be [n_requests][max_blocks]")
    _need(out.shape == q.shape, "out must have q's shape")
    _need(lse is None or lse.shape == q.shape[:2], "lse must be [total_q][Hq]")
    qp, q_ld = _rows(desc, q, desc.n_q_heads, "q")
    pp, nb = _pool(desc, pool)
    _check(lib().sx_kv4_attn(
        ctypes.byref(desc), qp, q_ld, _ints(cu_q, "cu_q"), _ints(seq_lens, "seq_lens"),
        _ints(block_table, "block_table"), block_table.shape[1], n, total, max_q, max_seqlen, pp, nb,
        _ptr(out, q.dtype, "out"), None if lse is None else _ptr(lse, torch.float32, "lse"),
        None if workspace is None else _ptr(workspace, torch.uint8, "workspace"),
        0 if workspace is None else workspace.numel(), _stream(stream)))
