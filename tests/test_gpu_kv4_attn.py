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
