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
import operator

import torch

from . import BF16, F32, LayerDesc, Plan, _check, _stream, lib

_TYPES = {F32: torch.float32, BF16: torch.bfloat16}
_I32, _U8 = torch.int32, torch.uint8
# the current stream's handle on a GPU without a Stream object (2.5 us), where torch offers it
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _need(ok: bool, what: str):
    if not ok:
        raise ValueError(what)


def _int(v, what: str) -> int:
    """A host number that the C call takes as int32 (ctypes would take it modulo 2^32)."""
    v = operator.index(v)
    if -0x80000000 <= v <= 0x7fffffff:
        return v
    raise ValueError(f"{what} ({v}) does not fit into 32 bits")


def _device(t) -> int:
    """The GPU that a call's tensors have to be on: the current one, where its first tensor is."""
    at = t.get_device()      # -1: host memory
    if at < 0 or at != torch.cuda.current_device():
        raise ValueError(f"a tensor is on {t.device}, not on the current GPU")
    return at


def _on(stream, at: int):
    return _raw_stream(at) if stream is None and _raw_stream is not None else _stream(stream)


def _ptr(t, dtype, at: int, what: str):
    """Device pointer of a contiguous tensor of this type on GPU `at`."""
    if t.dtype is dtype and t.get_device() == at and t.is_contiguous():
        return t.data_ptr()
    _need(t.dtype is dtype, f"{what} must be {dtype}, not {t.dtype}")
    _need(t.is_contiguous(), f"{what} must be contiguous")
    raise ValueError(f"{what} is on {t.device}, not on the current GPU")


def _opt(t, dtype, at: int, what: str):
    return None if t is None else _ptr(t, dtype, at, what)


def _rows(dtype, d: int, t, heads: int, at: int, what: str):
    """(pointer, elements between rows) of [n][heads][head_dim] rows, each contiguous."""
    shape = t.shape
    if len(shape) != 3 or shape[1] != heads or shape[2] != d:
        raise ValueError(f"{what} must be [n][{heads}][{d}], not {list(shape)}")
    ld, head, one = t.stride()
    if t.dtype is not dtype or one != 1 or (head != d and heads > 1) or t.get_device() != at:
        _need(t.dtype is dtype, f"{what} is {t.dtype}, the descriptor says {dtype}")
        _need(one == 1 and (heads == 1 or head == d), f"{what}'s rows must be contiguous")
        raise ValueError(f"{what} is on {t.device}, not on the current GPU")
    return t.data_ptr(), ld if shape[0] > 1 else heads * d


def _gamma(dtype, d: int, t, at: int, what: str):
    if t is None:
        return None
    _need(t.numel() == d, f"{what} must have {d} elements")
    return _ptr(t, dtype, at, what)


def _pool(desc: LayerDesc, t, at: int):
    """(pointer, blocks) of a 4-bit pool [n_blocks][Hkv][17 head_dim]."""
    shape = t.shape
    if len(shape) != 3 or shape[1] != desc.n_kv_heads or shape[2] != 17 * desc.head_dim:
        raise ValueError(f"pool must be [n_blocks][{desc.n_kv_heads}][{17 * desc.head_dim}], not {list(shape)}")
    return _ptr(t, _U8, at, "pool"), shape[0]


def _cache(desc: LayerDesc, t, at: int, what: str):
    if t.dim() != 4 or t.shape[1:] != (desc.n_kv_heads, desc.block_size, desc.head_dim):
        raise ValueError(f"{what} must be [n_blocks][{desc.n_kv_heads}][{desc.block_size}][{desc.head_dim}], "
                         f"not {list(t.shape)}")
    return _ptr(t, _TYPES.get(desc.dtype), at, what)


def append_slots(ctx_lens, new_lens, free_blocks, block_table, seq_lens, cu_new, positions, slots, state,
                 free_head=None, block_size: int = 16, stream=None):
    """Block tables and slot maps of a step in which request r, holding ctx_lens[r] tokens, appends new_lens[r]
    (None: one each).  int32 tensors; writes block_table, seq_lens, cu_new, positions, slots and state = (next
    entry of free_blocks, tokens without a slot)."""
    block_size = _int(block_size, "block_size")
    n, at = ctx_lens.numel(), _device(ctx_lens)
    _need(new_lens is None or new_lens.numel() == n, "new_lens and ctx_lens differ in length")
    _need(seq_lens.numel() == n and cu_new.numel() == n + 1, "seq_lens needs n and cu_new n + 1 entries")
    _need(block_table.dim() == 2 and block_table.shape[0] == n, "block_table must be [n_requests][max_blocks]")
    room, n_free = _int(positions.numel(), "positions"), _int(free_blocks.numel(), "free_blocks")
    _need(slots.numel() == room, "positions and slots differ in length")
    _need(state.numel() >= 2 and (free_head is None or free_head.numel() >= 1), "state needs two entries, free_head one")
    _check(lib().sx_append_slots(
        _ptr(ctx_lens, _I32, at, "ctx_lens"), _opt(new_lens, _I32, at, "new_lens"), n, block_size,
        _ptr(free_blocks, _I32, at, "free_blocks"), n_free, _opt(free_head, _I32, at, "free_head"),
        _ptr(block_table, _I32, at, "block_table"), block_table.shape[1], room, _ptr(seq_lens, _I32, at, "seq_lens"),
        _ptr(cu_new, _I32, at, "cu_new"), _ptr(positions, _I32, at, "positions"), _ptr(slots, _I32, at, "slots"),
        _ptr(state, _I32, at, "state"), _on(stream, at)))


def qk_norm_rope(desc: LayerDesc, q, k, positions, q_out, k_out, gamma_q=None, gamma_k=None, eps: float = 1e-6,
                 stream=None):
    """q_out, k_out = the rows of q [n][Hq][d] and k [n][Hkv][d], normalised per head (gamma None: not) and rotated to
    positions; rows at negative positions are left alone.  Rows may lie apart (parts of one projection)."""
    n, at, d, hq, hkv = positions.numel(), _device(positions), desc.head_dim, desc.n_q_heads, desc.n_kv_heads
    _need(q.shape[0] == n and k.shape[0] == n and q_out.shape[0] == n and k_out.shape[0] == n,
          "q, k, positions, q_out and k_out differ in length")
    dt = _TYPES.get(desc.dtype)
    qp, q_ld = _rows(dt, d, q, hq, at, "q")
    kp, k_ld = _rows(dt, d, k, hkv, at, "k")
    qo, qo_ld = _rows(dt, d, q_out, hq, at, "q_out")
    ko, ko_ld = _rows(dt, d, k_out, hkv, at, "k_out")
    _check(lib().sx_qk_norm_rope(ctypes.byref(desc), qp, q_ld, kp, k_ld, _gamma(dt, d, gamma_q, at, "gamma_q"),
                                 _gamma(dt, d, gamma_k, at, "gamma_k"), eps, _ptr(positions, _I32, at, "positions"), n,
                                 qo, qo_ld, ko, ko_ld, _on(stream, at)))


def qk_norm_rope_rows(plan: Plan, rows, n_rows, max_rows: int, q, k, gamma_q=None, gamma_k=None, eps: float = 1e-6,
                      stream=None):
    """The same in place on the listed rows of a plan, at their positions in the new sequence (beside rope_rows)."""
    max_rows = _int(int(max_rows), "max_rows")
    dt, d, at = _TYPES.get(plan.desc.dtype), plan.desc.head_dim, _device(q)
    tokens = plan.info()["total_tokens"]
    for t, heads, what in ((q, plan.desc.n_q_heads, "q"), (k, plan.desc.n_kv_heads, "k")):
        _need(t.numel() == tokens * heads * d, f"{what} must be [{tokens}][{heads}][{d}], not {list(t.shape)}")
    for t, n, what in ((rows, tokens, "rows"), (n_rows, plan.info()["n_requests"], "n_rows")):
        _need(isinstance(t, int) or t.numel() >= n, f"{what} needs {n} entries")
    _check(lib().sx_qk_norm_rope_rows(plan.handle, rows if isinstance(rows, int) else _ptr(rows, _I32, at, "rows"),
                                      n_rows if isinstance(n_rows, int) else _ptr(n_rows, _I32, at, "n_rows"),
                                      max_rows, _ptr(q, dt, at, "q"), _ptr(k, dt, at, "k"),
                                      _gamma(dt, d, gamma_q, at, "gamma_q"), _gamma(dt, d, gamma_k, at, "gamma_k"), eps,
                                      _on(stream, at)))


def kv4_record_bytes(desc: LayerDesc) -> int:
    """Bytes of one KV head of one block: a pool is a uint8 tensor [n_blocks][Hkv][this]."""
    n = ctypes.c_int64()
    _check(lib().sx_kv4_record_bytes(ctypes.byref(desc), ctypes.byref(n)))
    return n.value


def _row_args(desc, k, v, slots, pool):
    n, at, d, hkv = slots.numel(), _device(slots), desc.head_dim, desc.n_kv_heads
    _need(k.shape[0] == n and v.shape[0] == n, "k, v and slots differ in length")
    dt = _TYPES.get(desc.dtype)
    return (_rows(dt, d, k, hkv, at, "k"), _rows(dt, d, v, hkv, at, "v"), _ptr(slots, _I32, at, "slots"), n,
            _pool(desc, pool, at), at)


def kv4_write(desc: LayerDesc, k, v, slots, pool, stream=None):
    """Rows k, v [n][Hkv][d] rounded to 4 bits into slots of the pool (negative: skipped)."""
    (kp, k_ld), (vp, v_ld), sp, n, (pp, nb), at = _row_args(desc, k, v, slots, pool)
    _check(lib().sx_kv4_write(ctypes.byref(desc), kp, k_ld, vp, v_ld, sp, n, pp, nb, _on(stream, at)))


def kv4_read(desc: LayerDesc, pool, slots, k, v, stream=None):
    """The rows that slots hold into k, v [n][Hkv][d], exactly; rows of negative slots are left alone."""
    (kp, k_ld), (vp, v_ld), sp, n, (pp, nb), at = _row_args(desc, k, v, slots, pool)
    _check(lib().sx_kv4_read(ctypes.byref(desc), pp, nb, sp, n, kp, k_ld, vp, v_ld, _on(stream, at)))


def _block_args(desc, k_cache, v_cache, cache_blocks, pool, pool_blocks):
    n, at = cache_blocks.numel(), _device(cache_blocks)
    _need(pool_blocks.numel() == n, "cache_blocks and pool_blocks differ in length")
    _need(k_cache.shape == v_cache.shape, "k_cache and v_cache differ in shape")
    return (_cache(desc, k_cache, at, "k_cache"), _cache(desc, v_cache, at, "v_cache"), k_cache.shape[0],
            _ptr(cache_blocks, _I32, at, "cache_blocks"), n, *_pool(desc, pool, at),
            _ptr(pool_blocks, _I32, at, "pool_blocks"), at)


def kv4_pack(desc: LayerDesc, k_cache, v_cache, cache_blocks, pool, pool_blocks, stream=None):
    """Blocks cache_blocks[i] of a paged cache rounded to 4 bits into blocks pool_blocks[i] of the pool."""
    kc, vc, nc, cb, n, pp, nb, pb, at = _block_args(desc, k_cache, v_cache, cache_blocks, pool, pool_blocks)
    _check(lib().sx_kv4_pack(ctypes.byref(desc), kc, vc, nc, cb, n, pp, nb, pb, _on(stream, at)))


def kv4_unpack(desc: LayerDesc, pool, pool_blocks, k_cache, v_cache, cache_blocks, stream=None):
    """Blocks pool_blocks[i] of the pool into blocks cache_blocks[i] of a paged cache, exactly."""
    kc, vc, nc, cb, n, pp, nb, pb, at = _block_args(desc, k_cache, v_cache, cache_blocks, pool, pool_blocks)
    _check(lib().sx_kv4_unpack(ctypes.byref(desc), pp, nb, pb, n, kc, vc, nc, cb, _on(stream, at)))


def kv4_attn_workspace(desc: LayerDesc, n_requests: int, max_q: int, max_seqlen: int) -> int:
    """Bytes of workspace that kv4_attn needs for these bounds."""
    n = ctypes.c_int64()
    _check(lib().sx_kv4_attn_workspace(ctypes.byref(desc), _int(n_requests, "n_requests"), _int(max_q, "max_q"),
                                       _int(max_seqlen, "max_seqlen"), ctypes.byref(n)))
    return n.value


def kv4_attn(desc: LayerDesc, q, cu_q, seq_lens, block_table, pool, out, max_q: int, max_seqlen: int, workspace,
             lse=None, stream=None):
    """out = causal attention of every request's last tokens (rows cu_q[r] .. cu_q[r + 1] of q) over its seq_lens[r] keys
    in the pool; lse (float32 [total_q][Hq]) their natural-log sums.  out may be q itself where its rows are contiguous.
    workspace: uint8, kv4_attn_workspace bytes."""
    max_q, max_seqlen = _int(max_q, "max_q"), _int(max_seqlen, "max_seqlen")
    n, total, at, dt = seq_lens.numel(), q.shape[0], _device(seq_lens), _TYPES.get(desc.dtype)
    _need(cu_q.numel() == n + 1, "cu_q needs one entry more than seq_lens")
    _need(block_table.dim() == 2 and block_table.shape[0] == n, "block_table must be [n_requests][max_blocks]")
    _need(out.shape == q.shape, "out must have q's shape")
    _need(lse is None or lse.shape == q.shape[:2], "lse must be [total_q][Hq]")
    qp, q_ld = _rows(dt, desc.head_dim, q, desc.n_q_heads, at, "q")
    pp, nb = _pool(desc, pool, at)
    _check(lib().sx_kv4_attn(
        ctypes.byref(desc), qp, q_ld, _ptr(cu_q, _I32, at, "cu_q"), _ptr(seq_lens, _I32, at, "seq_lens"),
        _ptr(block_table, _I32, at, "block_table"), block_table.shape[1], n, total, max_q, max_seqlen, pp, nb,
        _ptr(out, dt, at, "out"), _opt(lse, torch.float32, at, "lse"), _opt(workspace, _U8, at, "workspace"),
        0 if workspace is None else workspace.numel(), _on(stream, at)))
