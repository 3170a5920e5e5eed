"""Decoding calls without a GPU: refusals of the C entry points and of the binding, and the references' own checks."""
import ctypes
import math

import pytest
import torch

import kv4ref as R
import paper_2606_01751_amd as sx

P = ctypes.c_void_p
A = 1 << 20          # an address that no refused call reads


def desc(**kw):
    base = dict(n_q_heads=8, n_kv_heads=2, head_dim=128, dtype="bf16", rope_base=1e6)
    base.update(kw)
    return sx.make_desc(**base)


def err(status, want, text):
    assert status == want
    assert text in sx.lib().sx_last_error().decode()


def slots_args(**kw):
    a = dict(ctx=A, new=A + 0x1000, n=4, b=16, free=A + 0x2000, nf=8, head=None, table=A + 0x3000, width=4, room=16,
             seq=A + 0x4000, cu=A + 0x5000, pos=A + 0x6000, slot=A + 0x7000, state=A + 0x8000)
    a.update(kw)
    return [a[k] for k in ("ctx", "new", "n", "b", "free", "nf", "head", "table", "width", "room", "seq", "cu", "pos",
                           "slot", "state")] + [None]


@pytest.mark.parametrize("kw,want,text", [
    (dict(ctx=None), sx.SX_EINVAL, "NULL"), (dict(table=None), sx.SX_EINVAL, "NULL"), (dict(slot=None), sx.SX_EINVAL, "NULL"),
    (dict(free=None), sx.SX_EINVAL, "free list"), (dict(nf=-1), sx.SX_EINVAL, "free list"), (dict(n=0), sx.SX_EINVAL, ">= 1"),
    (dict(b=0), sx.SX_EINVAL, ">= 1"), (dict(width=0), sx.SX_EINVAL, ">= 1"), (dict(room=-1), sx.SX_EINVAL, ">= 1"),
    (dict(n=65537), sx.SX_EUNSUPPORTED, "requests"), (dict(room=(1 << 30) + 1), sx.SX_EUNSUPPORTED, "max_tokens"),
    (dict(seq=A), sx.SX_EINVAL, "overlaps"), (dict(state=A + 0x2004), sx.SX_EINVAL, "overlaps"),
    (dict(head=A + 0x8004), sx.SX_EINVAL, "overlaps"), (dict(pos=A + 0x7000 - 60), sx.SX_EINVAL, "overlaps"),
    (dict(table=A + 0x4000 - 16), sx.SX_EINVAL, "overlaps"),
])
def test_append_slots_refusals(kw, want, text):
    err(sx.lib().sx_append_slots(*slots_args(**kw)), want, text)


def test_append_slots_allows_no_room():
    # positions and slots may be NULL where there is no room for any; the arguments are otherwise refused first
    err(sx.lib().sx_append_slots(*slots_args(room=0, pos=None, slot=None, n=0)), sx.SX_EINVAL, ">= 1")


def qk_args(**kw):
    a = dict(q=A, qld=1024, k=A + 0x10000, kld=256, gq=A + 0x20000, gk=A + 0x21000, eps=1e-6, pos=A + 0x22000, n=3,
             qo=A + 0x30000, qold=1024, ko=A + 0x40000, kold=256)
    a.update(kw)
    return [a[k] for k in ("q", "qld", "k", "kld", "gq", "gk", "eps", "pos", "n", "qo", "qold", "ko", "kold")] + [None]


@pytest.mark.parametrize("kw,want,text", [
    (dict(q=None), sx.SX_EINVAL, "q is NULL"), (dict(ko=None), sx.SX_EINVAL, "k_out is NULL"),
    (dict(pos=None), sx.SX_EINVAL, "positions"), (dict(qld=1016), sx.SX_ESHAPE, "between rows"),
    (dict(kld=257), sx.SX_ESHAPE, "between rows"), (dict(q=A + 8), sx.SX_EINVAL, "aligned"),
    (dict(gk=A + 4), sx.SX_EINVAL, "gamma"), (dict(eps=0.0), sx.SX_EINVAL, "eps"), (dict(eps=math.nan), sx.SX_EINVAL, "eps"),
    (dict(n=-1), sx.SX_EINVAL, "n_tokens"), (dict(n=(1 << 31) - 1), sx.SX_EUNSUPPORTED, "one launch"), (dict(qo=A, qold=2048), sx.SX_EINVAL, "in place"),
])
def test_qk_norm_rope_refusals(kw, want, text):
    err(sx.lib().sx_qk_norm_rope(ctypes.byref(desc()), *qk_args(**kw)), want, text)


def test_qk_norm_rope_descriptor_and_empty():
    L = sx.lib()
    assert L.sx_qk_norm_rope(ctypes.byref(desc(head_dim=96)), *qk_args()) == sx.SX_EUNSUPPORTED
    assert L.sx_qk_norm_rope(None, *qk_args()) == sx.SX_EINVAL
    assert L.sx_qk_norm_rope(ctypes.byref(desc()), *qk_args(n=0, q=None, pos=None)) == sx.SX_OK
    assert L.sx_qk_norm_rope_rows(None, A, A, 1, A, A, None, None, 1e-6, None) == sx.SX_EINVAL


def test_kv4_sizes():
    n = ctypes.c_int64()
    for d in (64, 128):
        assert sx.kv4_record_bytes(desc(head_dim=d)) == 17 * d
    assert sx.lib().sx_kv4_record_bytes(ctypes.byref(desc(head_dim=80)), ctypes.byref(n)) == sx.SX_EUNSUPPORTED
    assert sx.lib().sx_kv4_record_bytes(ctypes.byref(desc()), None) == sx.SX_EINVAL
    # no split, no workspace; it grows with every bound
    assert sx.kv4_attn_workspace(desc(), 8, 1, 256) == 0
    last = 0
    for q, s in ((1, 512), (1, 8192), (4, 8192), (64, 8192), (64, 131072)):
        w = sx.kv4_attn_workspace(desc(), 8, q, s)
        assert w >= last and w % 8 == 0
        last = w
    assert sx.lib().sx_kv4_attn_workspace(ctypes.byref(desc()), -1, 1, 1, ctypes.byref(n)) == sx.SX_EINVAL


@pytest.mark.parametrize("name", ["sx_kv4_write", "sx_kv4_read"])
def test_kv4_rows_refusals(name):
    f = getattr(sx.lib(), name)

    def call(d=desc(), k=A, kld=256, v=A + 0x10000, vld=256, slots=A + 0x20000, n=3, pool=A + 0x30000, nb=4):
        args = (k, kld, v, vld, slots, n, pool, nb) if name == "sx_kv4_write" else (pool, nb, slots, n, k, kld, v, vld)
        return f(ctypes.byref(d), *args, None)

    err(call(k=None), sx.SX_EINVAL, "k is NULL")
    err(call(v=A + 2), sx.SX_EINVAL, "aligned")
    err(call(vld=128), sx.SX_ESHAPE, "between rows")
    err(call(slots=None), sx.SX_EINVAL, "index")
    err(call(pool=None), sx.SX_EINVAL, "pool")
    err(call(pool=A + 8), sx.SX_EINVAL, "aligned")
    err(call(nb=0), sx.SX_ESHAPE, "n_blocks")
    err(call(nb=1 << 28), sx.SX_ESHAPE, "n_blocks")
    err(call(n=-1), sx.SX_EINVAL, "negative")
    err(call(d=desc(dtype=3)), sx.SX_EUNSUPPORTED, "dtype")
    assert call(n=0, k=None, slots=None) == sx.SX_OK


@pytest.mark.parametrize("name", ["sx_kv4_pack", "sx_kv4_unpack"])
def test_kv4_blocks_refusals(name):
    f = getattr(sx.lib(), name)

    def call(d=desc(), k=A, v=A + 0x10000, nc=4, cb=A + 0x20000, n=2, pool=A + 0x30000, nb=4, pb=A + 0x40000):
        args = (k, v, nc, cb, n, pool, nb, pb) if name == "sx_kv4_pack" else (pool, nb, pb, n, k, v, nc, cb)
        return f(ctypes.byref(d), *args, None)

    err(call(k=None), sx.SX_EINVAL, "NULL")
    err(call(cb=None), sx.SX_EINVAL, "NULL")
    err(call(pb=None), sx.SX_EINVAL, "index")
    err(call(v=A + 4), sx.SX_EINVAL, "aligned")
    err(call(nc=0), sx.SX_ESHAPE, "n_cache_blocks")
    err(call(n=-5), sx.SX_EINVAL, "negative")
    err(call(n=(1 << 31) - 1), sx.SX_EUNSUPPORTED, "one launch")
    assert call(n=0, k=None, pb=None) == sx.SX_OK


def attn_args(**kw):
    a = dict(q=A, qld=1024, cu=A + 0x10000, lens=A + 0x11000, table=A + 0x12000, width=64, nr=2, tq=2, mq=1, ms=131072,
             pool=A + 0x20000, nb=64, out=A + 0x30000, lse=None, ws=A + 0x40000, wb=1 << 28)
    a.update(kw)
    return [a[k] for k in ("q", "qld", "cu", "lens", "table", "width", "nr", "tq", "mq", "ms", "pool", "nb", "out", "lse",
                           "ws", "wb")] + [None]


@pytest.mark.parametrize("kw,want,text", [
    (dict(q=None), sx.SX_EINVAL, "q is NULL"), (dict(q=A + 4), sx.SX_EINVAL, "aligned"), (dict(qld=512), sx.SX_ESHAPE, "rows"),
    (dict(cu=None), sx.SX_EINVAL, "NULL"), (dict(lens=None), sx.SX_EINVAL, "NULL"), (dict(table=None), sx.SX_EINVAL, "NULL"),
    (dict(out=None), sx.SX_EINVAL, "NULL"), (dict(out=A + 0x30008), sx.SX_EINVAL, "aligned"),
    (dict(pool=None), sx.SX_EINVAL, "pool"), (dict(nb=0), sx.SX_ESHAPE, "n_blocks"), (dict(ws=None), sx.SX_EINVAL, "workspace"),
    (dict(wb=64), sx.SX_ESHAPE, "workspace"), (dict(ws=A + 0x40004), sx.SX_EINVAL, "aligned"),
    (dict(nr=-1), sx.SX_EINVAL, "negative"), (dict(mq=-1), sx.SX_EINVAL, "negative"), (dict(width=-1), sx.SX_EINVAL, "negative"),
    (dict(nr=65536, wb=1 << 40), sx.SX_EUNSUPPORTED, "requests"), (dict(ms=(1 << 30) + 1), sx.SX_EUNSUPPORTED, "max_seqlen"),
    (dict(tq=1 << 30, mq=1 << 30), sx.SX_EUNSUPPORTED, "too large"),
])
def test_kv4_attn_refusals(kw, want, text):
    err(sx.lib().sx_kv4_attn(ctypes.byref(desc()), *attn_args(**kw)), want, text)


def test_kv4_attn_empty_calls_do_nothing():
    for kw in (dict(nr=0), dict(tq=0, q=None, out=None), dict(mq=0)):
        assert sx.lib().sx_kv4_attn(ctypes.byref(desc()), *attn_args(**kw)) == sx.SX_OK


def test_binding_refuses_wrong_tensors():
    d = desc()
    k = torch.zeros(3, 2, 128, dtype=torch.bfloat16)
    slots = torch.zeros(3, dtype=torch.int32)
    pool = torch.zeros(2, 2, 17 * 128, dtype=torch.uint8)
    for bad in (dict(k=k[:, :1]), dict(k=k.float()), dict(k=k.transpose(1, 2).contiguous().transpose(1, 2)),
                dict(slots=slots[:2]), dict(pool=pool[:, :, :64])):
        a = {**dict(k=k, v=k, slots=slots, pool=pool), **bad}
        with pytest.raises(ValueError):
            sx.kv4_write(d, a["k"], a["v"], a["slots"], a["pool"])


def test_reference_rounding_is_the_nearest_value():
    # round4 against a plain search over all 15 values of a group's own scale
    g = torch.Generator().manual_seed(1)
    x = torch.randn(64, 32, generator=g) * torch.exp(3 * torch.randn(64, 1, generator=g))
    val, code, byte = R.round4(x)
    s = torch.ldexp(torch.ones(64), byte[:, 0].int() - 127).double()
    amax = x.abs().amax(-1).double()
    assert (amax <= 7 * s).all() and (amax > 3.5 * s).all()
    near = (x.double()[..., None] / s[:, None, None] - torch.cat([R.MAG, -R.MAG])).abs().amin(-1) * s[:, None]
    assert torch.equal((x.double() - val).abs(), near)
    assert (x.double() - val).abs().le(s[:, None]).all()     # half of the widest step
    pool = torch.zeros(2, 1, R.record(64), dtype=torch.uint8)
    y = torch.randn(5, 1, 64, generator=g)
    slots = torch.tensor([3, 17, 31, 0, 30])
    kv, vv = R.put_rows(pool, y, y + 1, slots)
    k2, v2 = R.get_rows(pool, slots, 64)
    assert torch.equal(kv, k2) and torch.equal(vv, v2)
