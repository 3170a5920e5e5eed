"""Refusals of the decoding calls without a GPU, beside test_decode_cpu.py: arguments that overlap, and sizes that the C types
do not hold."""
import ctypes

import pytest
import torch

import paper_2606_01751_amd as sx
from test_decode_cpu import A, attn_args, desc, err, qk_args


def qk(status=sx.SX_EINVAL, text="overlap", dtype="bf16", **kw):
    err(sx.lib().sx_qk_norm_rope(ctypes.byref(desc(dtype=dtype)), *qk_args(**kw)), status, text)


# bf16, 8 / 2 heads of 128: a row of q has 2048 bytes, a row of k 512; a row of stacked parts 3584
@pytest.mark.parametrize("kw", [
    dict(qo=A + 2048), dict(qo=A + 4096 + 2032), dict(qo=A - 4096 - 2032), dict(qo=A + 0x10000), dict(qo=A + 0x10000 + 1520),
    dict(qo=A + 0x20000), dict(qo=A + 0x21000 - 6128), dict(qo=A + 0x22000), dict(ko=A), dict(ko=A + 6128), dict(ko=A + 0x10200),
    dict(ko=A + 0x30000 + 2048), dict(ko=A + 0x21000), dict(ko=A + 0x22000 - 16),
    # parts of stacked rows, 1792 elements apart: one row behind, the part of q, one head into the other's part
    dict(qld=1792, kld=1792, k=A + 2048, qo=A + 3584, qold=1792), dict(qld=1792, kld=1792, k=A + 2048, ko=A + 1536, kold=1792),
    dict(qld=1792, kld=1792, k=A + 2048, qo=A, qold=1792, ko=A + 2048 + 256, kold=1792),
    # rows of different distances
    dict(qld=1792, qo=A + 3584 + 1024, qold=1800), dict(qld=1792, kld=256, k=A + 2048, ko=A + 2560, kold=2048),
])
def test_qk_norm_rope_refuses_overlapping_rows(kw):
    qk(**kw)


def test_qk_norm_rope_refuses_bases_whose_angles_it_cannot_reduce():
    # angles up to 2^31 / base: from 2^56 on the reduced angle was no longer one, and cos and sin came out beyond 1
    for base in (1e-9, 2.0 ** -20 * (1 - 2.0 ** -52), 5e-324):
        err(sx.lib().sx_qk_norm_rope(ctypes.byref(desc(rope_base=base)), *qk_args()), sx.SX_EUNSUPPORTED, "rope_base")


def _rows_meet(x, y):
    return any(a < d and c < b for a, b in x for c, d in y)


def test_overlap_is_that_of_the_rows():
    # every offset of a short k_out over the rows of q: refused where a row meets a row, else the call goes on to its next
    # check (eps, which comes before, is valid; a negative position pointer is not there to be read: n_tokens rows only)
    for qld, kold, n in ((1792, 1792, 3), (1792, 256, 3), (1024, 1792, 2), (2048, 1792, 3), (1792, 1800, 4)):
        q = [(A + i * qld * 2, A + i * qld * 2 + 2048) for i in range(n)]
        for off in range(-4096, 3 * n * 4096, 1008):
            at = A + off // 16 * 16
            ko = [(at + i * kold * 2, at + i * kold * 2 + 512) for i in range(n)]
            if _rows_meet(q, ko):
                qk(qld=qld, ko=at, kold=kold, n=n, k=A + (1 << 24), gq=None, gk=None, pos=A + (1 << 25), qo=A + (1 << 26))


def attn(**kw):
    # 2 rows of 2048 bytes, 4 blocks of 2 x 2176 bytes, up to 131072 keys; nothing overlaps unless kw says so
    a = dict(q=A, out=A + 0x30000, pool=A + (1 << 24), nb=4, ws=A + (1 << 28), lse=A + 0x50000)
    a.update(kw)
    err(sx.lib().sx_kv4_attn(ctypes.byref(desc()), *attn_args(**a)), sx.SX_EINVAL, "overlap")


@pytest.mark.parametrize("kw", [
    dict(out=A + 2048), dict(out=A - 2048 - 16), dict(out=A, qld=1792), dict(out=A + 2048 + 16, qld=1792), dict(out=A + 0x10000),
    dict(out=A + 0x11000 - 4080), dict(out=A + 0x12000 + 496), dict(out=A + (1 << 24) + 17392), dict(out=A + (1 << 28) + 4096),
    dict(lse=A), dict(lse=A + 0x30000 + 4092), dict(lse=A + 0x12000 - 60), dict(lse=A + (1 << 24)), dict(lse=A + (1 << 28) + 64),
    dict(ws=A), dict(ws=A + 0x10000), dict(ws=A + (1 << 24)),
])
def test_kv4_attn_refuses_overlapping_outputs(kw):
    attn(**kw)


# 3 rows of 512 bytes, or 4 blocks of 8192; a pool of 4 blocks of 4352
@pytest.mark.parametrize("kw", [dict(pool=A), dict(pool=A + 0x10000 + 1024), dict(pool=A + 0x20000 - 16), dict(pool=A - 17392)])
def test_kv4_write_refuses_a_pool_over_its_inputs(kw):
    a = dict(k=A, v=A + 0x10000, slots=A + 0x20000, pool=A + 0x30000)
    a.update(kw)
    err(sx.lib().sx_kv4_write(ctypes.byref(desc()), a["k"], 256, a["v"], 256, a["slots"], 3, a["pool"], 4, None), sx.SX_EINVAL, "overlap")


@pytest.mark.parametrize("kw", [
    dict(v=A), dict(v=A + 1024), dict(k=A + 0x30000 + 17392), dict(v=A + 0x30000 - 1520), dict(k=A + 0x20000), dict(v=A + 0x20000 - 1520),
    dict(kld=768, vld=768, v=A + 496),
])
def test_kv4_read_refuses_outputs_over_arguments(kw):
    a = dict(k=A, kld=256, v=A + 0x10000, vld=256, slots=A + 0x20000, pool=A + 0x30000)
    a.update(kw)
    err(sx.lib().sx_kv4_read(ctypes.byref(desc()), a["pool"], 4, a["slots"], 3, a["k"], a["kld"], a["v"], a["vld"], None), sx.SX_EINVAL,
        "overlap")


@pytest.mark.parametrize("name,kw", [
    ("pack", dict(pool=A + 32752)), ("pack", dict(pool=A + 0x10000 - 16)), ("pack", dict(pool=A + 0x20000)), ("pack", dict(pb=A + 0x30000)),
    ("unpack", dict(v=A + 32752)), ("unpack", dict(k=A + 0x30000)), ("unpack", dict(v=A + 0x20000 - 16)), ("unpack", dict(pb=A + 4)),
])
def test_kv4_blocks_refuse_outputs_over_arguments(name, kw):
    a = dict(k=A, v=A + 0x10000, cb=A + 0x20000, pool=A + 0x30000, pb=A + 0x40000)
    a.update(kw)
    if name == "pack":
        st = sx.lib().sx_kv4_pack(ctypes.byref(desc()), a["k"], a["v"], 4, a["cb"], 2, a["pool"], 4, a["pb"], None)
    else:
        st = sx.lib().sx_kv4_unpack(ctypes.byref(desc()), a["pool"], 4, a["pb"], 2, a["k"], a["v"], 4, a["cb"], None)
    err(st, sx.SX_EINVAL, "overlap")


def test_binding_refuses_sizes_that_the_c_types_do_not_hold():
    # ctypes takes them modulo 2^32: a bound of 2^32 + 512 keys came out as one of 512
    for bad in ((8, 1, (1 << 32) + 512), (8, (1 << 32) + 1, 4096), ((1 << 32) + 8, 1, 4096), (8, 1, 1 << 31), (8, -1 << 40, 1)):
        with pytest.raises(ValueError, match="32 bits"):
            sx.kv4_attn_workspace(desc(), *bad)
    with pytest.raises(sx.SxError):
        sx.kv4_attn_workspace(desc(), 8, -1, 4096)
    with pytest.raises(TypeError):
        sx.kv4_attn_workspace(desc(), 8, 1.5, 4096)
    z = torch.zeros(4, 2, 128, dtype=torch.int32)
    with pytest.raises(ValueError, match="32 bits"):
        sx.append_slots(*[z] * 9, block_size=(1 << 32) + 16)
    for bound in (dict(max_q=1, max_seqlen=1 << 32), dict(max_q=1 << 31, max_seqlen=7)):
        with pytest.raises(ValueError, match="32 bits"):
            sx.kv4_attn(desc(), z, z, z, z, z, z, workspace=z, **bound)
