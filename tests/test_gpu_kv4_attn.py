"""The 4-bit attention on the GPU, beside test_gpu_decode.py: what a row's result may not depend on, the precision of each
route, and long chunks of keys."""
import math

import pytest
import torch

import paper_2606_01751_amd as sx
from test_gpu_decode import Batch, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    sx.lib()


def put(b, r, at, k, v):
    """Keys k and values v [n][Hkv][d] of request r's tokens `at`, rounded to 4 bits."""
    t = torch.as_tensor(at)
    slots = i32(b.table[r, t // 16] * 16 + t % 16)
    sx.kv4_write(sx.make_desc(b.hkv, b.hkv, b.d, "f32", 1e4), k.float().cuda().contiguous(), v.float().cuda().contiguous(), slots, b.pool)


# (query tokens, keys, token from which the key is seen): one step or tile, the middle of a wave's columns, split keys
@pytest.mark.parametrize("hq,hkv,d,dtype,nq,nk,first", [
    (8, 2, 128, "bf16", 4, 60, 2), (8, 2, 128, "bf16", 9, 60, 4), (4, 1, 64, "bf16", 9, 2500, 4), (8, 2, 64, "f32", 9, 60, 4),
    (4, 1, 128, "f32", 40, 1500, 17), (8, 2, 128, "bf16", 300, 700, 204), (4, 1, 64, "bf16", 300, 700, 203),
    (2, 1, 128, "bf16", 200, 9000, 100),
])
@pytest.mark.parametrize("what", ["large", "nan"])
def test_a_key_behind_a_row_leaves_its_bits(hq, hkv, d, dtype, nq, nk, first, what):
    # the maximum of a row is raised by its own keys alone: the rows before a very large key, and before a NaN, keep every bit
    b = Batch([(nq, nk), (1, 40)], hq, hkv, d, dtype, seed=nq + d)
    out, lse = b.run()
    p = nk - nq + first
    k = torch.randn(1, hkv, d, generator=torch.Generator().manual_seed(1)) * (100.0 if what == "large" else math.nan)
    put(b, 0, [p], k, torch.ones(1, hkv, d))
    out2, lse2 = b.run()
    assert torch.equal(out2[:first], out[:first]) and torch.equal(lse2[:first], lse[:first])
    assert torch.equal(out2[nq:], out[nq:]) and torch.equal(lse2[nq:], lse[nq:])
    if what == "nan":
        assert out2[first:nq].isnan().all() and lse2[first:nq].isnan().all()
    else:
        assert not torch.equal(out2[first:nq], out[first:nq]) and torch.isfinite(out2).all()


def one_part_reference(b, r, extra=0.0):
    """(out, bound) in float64 of request r of more than 128 rows in bfloat16.  A probability p_j goes into the product as
    p_j (1 + e_j), |e_j| <= 2^-8, and the row is divided by the sum of these: off by at most 2^-8 sum w_j |v_j - out| over the
    softmax weights w (times 1 + 2^-7 for the divisor's own error).  The float32 arithmetic as in kv4ref.attention, without
    parts of a probability; `extra` on top of the relative error of a score."""
    import kv4ref as R
    q0, n, m, grp = b.cu[r], b.nq[r], b.nk[r], b.hq // b.hkv
    k, v, ok = (x.cuda() for x in R.rows_of(b.pool.cpu(), b.table[r], m, b.d))
    see = (torch.arange(m, device="cuda")[None] <= torch.arange(m - n, m, device="cuda")[:, None]) & ok[None]
    out = torch.zeros(n, b.hq, b.d, dtype=torch.float64, device="cuda")
    bound = torch.zeros_like(out)
    scale = b.d ** -0.5
    for h in range(b.hq):
        kh, vh, qh = k[:, h // grp], v[:, h // grp], b.q[q0:q0 + n, h].double()
        s = (qh @ kh.t().contiguous() * scale).masked_fill(~see, -math.inf)
        w = s.softmax(-1)
        out[:, h] = w @ vh
        mag = (qh.abs() @ kh.abs().t().contiguous()).masked_fill(~see, 0).amax(-1) * scale
        ds = mag * (b.d + 4) * 2.0 ** -24 + 2.0 ** -22 * (s.abs().masked_fill(~see, 0).amax(-1) + 1) + extra
        fine = 2 * (ds + m * 2.0 ** -24 + 2.0 ** -22)[:, None] * (w @ vh.abs())
        for i in range(n):
            bound[i, h] = fine[i] + 2.0 ** -8 * (1 + 2.0 ** -7) * (w[i] @ (vh - out[i, h]).abs())
    return out, bound


@pytest.mark.parametrize("d,nq,nk", [(128, 150, 700), (64, 290, 290), (128, 200, 3000), (64, 140, 9000)])
@pytest.mark.parametrize("peak", [0.0, 7.0, 12.0])
def test_many_rows_divide_by_the_probabilities_that_were_multiplied(d, nq, nk, peak):
    # peak: one key early in the second tile whose score lies that many nats above the first tile's, below the raise of the
    # maximum: nearly all the weight of a row is on it, and the row's result is its value, whatever its probability's rounding
    b = Batch([(nq, nk), (1, 33)], 2, 1, d, "bf16", seed=nq)
    if peak:
        g = torch.Generator().manual_seed(d)
        unit = torch.ones(1, 1, d) / d ** 0.5                # scores in nats: q = a * ones, k = c * ones
        put(b, 0, range(nk), 0.02 * torch.randn(nk, 1, d, generator=g), torch.randn(nk, 1, d, generator=g))
        put(b, 0, [64], d ** 0.5 * unit, 1.5 * torch.sign(torch.randn(1, 1, d, generator=g)))
        b.q[:nq] = (peak / d ** 0.5 * (1 + 0.2 * torch.rand(nq, 2, 1, generator=g))).expand(nq, 2, d).to(b.q.dtype).cuda()
    out, _ = b.run()
    want, bound = one_part_reference(b, 0)
    eps = torch.finfo(torch.bfloat16).eps
    off = (out[:nq].double() - want).abs() - (bound + eps / 2 * (want.abs() + bound))
    assert off.max().item() <= 0, off.max().item()
