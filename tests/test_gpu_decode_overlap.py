"""Arguments of the decoding calls that share an allocation, on the GPU: what is allowed gives the same bits, the rest is refused
on the host."""
import pytest
import torch

import paper_2606_01751_amd as sx
import workloads as W
from sxgpu import desc_of
from test_gpu_decode import DT, Batch, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    sx.lib()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_qk_norm_rope_into_parts_of_one_allocation(dtype):
    n, hq, hkv, d, dt = 7, 4, 2, 64, DT[dtype]
    g = torch.Generator().manual_seed(2)
    x = torch.randn(n, 2 * (hq + hkv), d, generator=g).to(dt).cuda()
    pos, gam, desc = i32(range(3, 3 + n)), torch.ones(d, dtype=dt, device="cuda"), sx.make_desc(hq, hkv, d, dtype, 1e4)
    qo, ko = torch.empty(n, hq, d, dtype=dt, device="cuda"), torch.empty(n, hkv, d, dtype=dt, device="cuda")
    q, k = x[:, :hq], x[:, hq:hq + hkv]
    sx.qk_norm_rope(desc, q, k, pos, qo, ko, gam, gam)
    # the outputs as further parts of the same rows
    sx.qk_norm_rope(desc, q, k, pos, x[:, hq + hkv:2 * hq + hkv], x[:, 2 * hq + hkv:], gam, gam)
    assert torch.equal(x[:, hq + hkv:2 * hq + hkv], qo) and torch.equal(x[:, 2 * hq + hkv:], ko)
    # rows of k_out between those of q, at another distance: two rows of q 4096 elements apart, k_out's in the gap
    flat = torch.zeros(16384, dtype=dt, device="cuda")
    q2, ko2 = flat.as_strided((2, hq, d), (4096, d, 1)), flat.as_strided((2, hkv, d), (1024, d, 1), 512)
    q2.copy_(q[:2])
    sx.qk_norm_rope(desc, q2, k[:2], pos[:2].clone(), torch.empty_like(qo[:2]), ko2, gam, gam)
    assert torch.equal(ko2, ko[:2]) and torch.equal(q2, q[:2])
    for bad in (dict(q_out=x[:, hq - 1:2 * hq - 1]), dict(k_out=q[:, :hkv]), dict(q_out=x.view(-1, d)[1:1 + n * hq].view(n, hq, d)),
                dict(q_out=qo, k_out=qo[:, :hkv])):
        a = {"q_out": qo, "k_out": ko, **bad}
        with pytest.raises(sx.SxError, match="overlap"):
            sx.qk_norm_rope(desc, q, k, pos, a["q_out"], a["k_out"], gam, gam)


def test_qk_norm_rope_rows_refuses_shared_tensors():
    w = W.custom_workload([[(37, False, 0, None), (25, True, 900, None)]], n_q_heads=8, n_kv_heads=2, head_dim=64, dtype="bf16",
                          rope_base=5e5, seed=7, name="rows")
    plan = sx.Plan(desc_of(w), w.requests, w.n_dst_blocks, w.n_src_blocks)
    T = w.total_tokens
    x = torch.randn(T * 10 * 64 + 64).bfloat16().cuda()
    q, k = x[:T * 512].view(T, 8, 64), x[T * 512:T * 640].view(T, 2, 64)
    rows, n = i32(range(T)), i32([T])
    sx.qk_norm_rope_rows(plan, rows, n, T, q, k, x[T * 640:])
    for bad in (dict(k=x[T * 512 - 64:T * 640 - 64].view(T, 2, 64)), dict(gamma_q=k[3, 1]), dict(rows=q.view(torch.int32).flatten()[:T])):
        a = {"k": k, "gamma_q": None, "rows": rows, **bad}
        with pytest.raises(sx.SxError, match="overlap"):
            sx.qk_norm_rope_rows(plan, a["rows"], n, T, q, a["k"], a["gamma_q"])
    plan.close()


@pytest.mark.parametrize("hq,hkv,d,dtype,sizes", [
    (8, 2, 128, "bf16", [(1, 40), (1, 3000), (9, 700), (3, 5000)]), (4, 1, 64, "bf16", [(300, 700), (1, 9000), (200, 4000)]),
    (6, 2, 64, "f32", [(1, 40), (45, 2500), (7, 300)]),
])
def test_kv4_attn_in_place(hq, hkv, d, dtype, sizes):
    b = Batch(sizes, hq, hkv, d, dtype, seed=hq)
    want, want_lse = b.run()
    n, q = b.cu[-1], b.q.clone()
    size = sx.kv4_attn_workspace(b.desc, len(sizes), max(b.nq), max(b.nk))
    ws, lse = torch.empty(size, dtype=torch.uint8, device="cuda"), torch.empty(n + 2, hq, device="cuda")
    sx.kv4_attn(b.desc, q, i32(b.cu), i32(b.nk), b.table.cuda(), b.pool, q, max(b.nq), max(b.nk), ws, lse=lse)
    assert torch.equal(q[:n], want[:n]) and torch.equal(q[n:], b.q[n:]) and torch.equal(lse[:n], want_lse[:n])


def test_kv4_moves_between_parts_of_one_allocation():
    # K and V of stacked rows, read into further parts of them; the pool and the cache as parts of one tensor
    n, hkv, d = 5, 2, 64
    x = torch.randn(n, 4 * hkv, d, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    desc, slots = sx.make_desc(hkv, hkv, d, "bf16", 1e4), i32([3, 17, 1, 30, 8])
    whole = torch.zeros(2 * hkv * 17 * d + 2 * 2 * hkv * 16 * d * 2, dtype=torch.uint8, device="cuda")
    pool = whole[:2 * hkv * 17 * d].view(2, hkv, 17 * d)
    kc, vc = whole[2 * hkv * 17 * d:].view(torch.bfloat16).view(2, 2, hkv, 16, d)
    sx.kv4_write(desc, x[:, :hkv], x[:, hkv:2 * hkv], slots, pool)
    sx.kv4_read(desc, pool, slots, x[:, 2 * hkv:3 * hkv], x[:, 3 * hkv:])
    sx.kv4_unpack(desc, pool, i32([0, 1]), kc, vc, i32([1, 0]))
    for i, s in enumerate(slots.tolist()):
        assert torch.equal(x[i, 2 * hkv:3 * hkv], kc[1 - s // 16, :, s % 16]) and torch.equal(x[i, 3 * hkv:], vc[1 - s // 16, :, s % 16])
    with pytest.raises(sx.SxError, match="overlap"):
        sx.kv4_read(desc, pool, slots, x[:, 2 * hkv:3 * hkv], x[:, 2 * hkv:3 * hkv])
    with pytest.raises(sx.SxError, match="overlap"):
        sx.kv4_unpack(desc, pool, i32([0, 1]), kc, kc, i32([1, 0]))
