"""Per-head norm with rotation on the GPU, beside test_gpu_decode.py: small bases of the frequencies."""
import pytest
import torch

import kv4ref as R
import paper_2606_01751_amd as sx
import workloads as W
from sxgpu import desc_of
from test_gpu_decode import i32, near

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    sx.lib()


@pytest.mark.parametrize("base", [1.0, 2.0 ** -7, 2.0 ** -20])
def test_small_bases(base):
    # angles far beyond the positions.  2^(-2i/d) powers of these bases are exact in float64 every 8th pair or so; the others may
    # be off by half a unit on either side, which moves an angle by pos theta 2^-52: positions keep that below 2^-24
    d, n = 64, 40
    x = torch.randn(n, 3, d, generator=torch.Generator().manual_seed(1))
    pos = torch.arange(n, dtype=torch.int32) * 6                        # 234 * 2^20 * 2^-52 < 2^-24
    qo, ko = torch.empty(n, 2, d, device="cuda"), torch.empty(n, 1, d, device="cuda")
    xd = x.cuda()
    sx.qk_norm_rope(sx.make_desc(2, 1, d, "f32", base), xd[:, :2], xd[:, 2:], pos.cuda(), qo, ko)
    for got, src in ((qo, x[:, :2]), (ko, x[:, 2:])):
        want, bound = R.norm_rope(src, None, 1e-6, pos, base, True)
        near(got, want, bound, "f32")


def test_plan_rows_refuse_bases_below():
    w = W.custom_workload([[(20, False, 0, None)]], n_q_heads=2, n_kv_heads=1, head_dim=64, dtype="f32", rope_base=1e-9, seed=1,
                          name="base")
    plan = sx.Plan(desc_of(w), w.requests, w.n_dst_blocks, w.n_src_blocks)
    q, k = torch.randn(20, 2, 64).cuda(), torch.randn(20, 1, 64).cuda()
    with pytest.raises(sx.SxError, match="rope_base"):
        sx.qk_norm_rope_rows(plan, i32(range(20)), i32([20]), 20, q, k)
    plan.close()
