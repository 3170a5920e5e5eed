"""The 8-bit layer body on the GPU against float64 references (f8ref.py): norms and activations to 8 bits, products.

Tolerances.  A bfloat16 output is off by at most half a step, 2^-8 of its value (with what went before: of the bound too).
Norms are formed in float64 and rounded to float32 once: 2^-23 of the value covers that and the order of the sum.  SwiGLU in
float32: e^-g to 2 units (2^-22), 1 + e^-g, the quotient and the product half a unit each (divisions up to 2.5): 2^-20.
Products: f8ref.product_bound."""
import math

import pytest
import torch

import f8ref as R
import paper_2606_01751_amd as sx
import workloads as W
from sxgpu import desc_of

pytestmark = pytest.mark.gpu
BF16, F8 = torch.bfloat16, torch.float8_e4m3fn


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    sx.lib()


def gen(seed):
    return torch.Generator().manual_seed(seed)


def bits8(t):
    return t.view(torch.uint8).cpu()


def i32(x):
    return torch.as_tensor(x, dtype=torch.int32).cuda()


def make_plan(lengths):
    w = W.custom_workload([[(n, False, 3 * i, None)] for i, n in enumerate(lengths)], n_q_heads=8, n_kv_heads=2, head_dim=128,
                          dtype="bf16", rope_base=1e6, seed=1, plant_per_segment=0, name="f8")
    return sx.Plan(desc_of(w), w.requests, w.n_dst_blocks, w.n_src_blocks)


def row_lists(lengths, counts, seed):
    """(rows, n_rows, [(slot, token)] of every listed row) of a plan's requests."""
    g = gen(seed)
    rows = torch.full((sum(lengths),), -5, dtype=torch.int32)
    where, off = [], 0
    for n, c in zip(lengths, counts):
        t = torch.sort(torch.randperm(n, generator=g)[:c]).values.int()
        rows[off:off + c] = t
        where += [(off + i, off + int(x)) for i, x in enumerate(t)]
        off += n
    return rows.cuda(), i32(counts), where


def hidden(g, n, width, dtype=BF16):
    chan = torch.exp(0.3 * torch.randn(width, generator=g))
    chan[::61] *= 12
    return (torch.randn(n, width, generator=g) * chan * torch.exp(0.4 * torch.randn(n, 1, generator=g))).to(dtype)


def near16(got, want, bound, what):
    got = got.double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN in other places"
    off = (got - want).abs() - (bound + 2.0 ** -8 * (want.abs() + bound) + 1e-38)
    worst = off.nan_to_num(-1.0).max().item() if off.numel() else 0.0
    assert worst <= 0, f"{what}: over the bound by {worst}"


# ---------------------------------------------------------------- 8 bits

def test_every_bfloat16_value_to_8_bits():
    # every finite bfloat16 value among those of its size, beside one of up to 2^9 times it: bit for bit
    v = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(BF16)
    v = v[torch.isfinite(v)].float()
    v = v[torch.sort(v.abs()).indices][:514 * 127].view(514, 127)
    for up in range(10):
        top = (v.abs().amax(1, keepdim=True).double() * 2.0 ** up * 1.3).clamp(max=3.38e38).float()
        x = torch.cat([v, top], 1).to(BF16)
        x = torch.cat([x, x.flip(0)], 1).contiguous()
        y, s = torch.zeros(514, 256, dtype=F8, device="cuda"), torch.full((514, 4), 77, dtype=torch.uint8, device="cuda")
        sx.add_rmsnorm_f8(x.cuda(), y, s)
        c, b = R.quantise(x.double())
        assert torch.equal(s.cpu(), b)
        assert torch.equal(bits8(y), c)


def test_groups_that_are_not_finite_zero_or_tiny():
    x = torch.randn(6, 640, generator=gen(1)).to(BF16)
    x[0, 5], x[1, 130], x[2, 639], x[3, :128] = math.nan, math.inf, -math.inf, 0
    x[4] = 2.0 ** -130                      # below the smallest scale's steps
    x[5, :128], x[5, 128:256] = 3.3e38, 2.0 ** -126
    y, s = torch.ones(6, 640, device="cuda").to(F8), torch.ones(6, 8, dtype=torch.uint8, device="cuda")
    sx.add_rmsnorm_f8(x.cuda(), y, s)
    c, b = R.quantise(x.double())
    assert torch.equal(s.cpu(), b) and torch.equal(bits8(y), c)
    assert (b == 255).sum().item() == 3 and b[3, 0].item() == 1


@pytest.mark.parametrize("n,k", [(128, 128), (256, 1152), (896, 640), (128, 4096)])
def test_pack_weight(n, k):
    w = torch.randn(n, k, generator=gen(n + k)) * torch.exp(2 * torch.randn(n, 1, generator=gen(k)))
    w[3, 7], w[n - 1, k - 1] = 448.0, -1e-30
    if n > 128:
        w[130, 5] = math.inf
    w = w.to(BF16)
    c = torch.zeros(n, k, dtype=F8, device="cuda")
    s = torch.full((n // 128, R.ld(k)), 9, dtype=torch.uint8, device="cuda")
    sx.f8_pack_weight(w.cuda(), c, s)
    want, byte = R.quantise_weight(w.double())
    assert torch.equal(s.cpu(), byte) and torch.equal(bits8(c), want)
    if n == 256:    # stacked, as experts are
        c2, s2 = torch.zeros_like(c), torch.zeros_like(s)
        sx.f8_pack_weight(w.cuda().view(2, 128, k), c2.view(2, 128, k), s2.view(2, 1, -1))
        assert torch.equal(bits8(c2), want) and torch.equal(s2.cpu(), byte)


# ---------------------------------------------------------------- norm

def run_norm(x, delta, gamma, eps, keep16, **kw):
    n, h = x.shape
    o = dict(y8=torch.full((n, h), 7, dtype=torch.uint8, device="cuda").view(F8),
             y_scale=torch.full((n, R.ld(h)), 7, dtype=torch.uint8, device="cuda"))
    o["x_out"] = torch.full((n, h), 7.0, dtype=BF16, device="cuda") if delta is not None else None
    o["y16"] = torch.full((n, h), 7.0, dtype=BF16, device="cuda") if keep16 else None
    up = lambda t: None if t is None else t.cuda()  # noqa: E731
    sx.add_rmsnorm_f8(up(x), gamma=up(gamma), eps=eps, delta=up(delta), **o, **kw)
    return {k: None if v is None else v.cpu() for k, v in o.items()}


def check_norm(o, x, delta, gamma, eps, xrow, yrow, slot):
    """Row i of the call: x row xrow[i], y row yrow[i], slot slot[i]; every other row as it was."""
    s = x[xrow].double()
    if delta is not None:
        s = (s + delta[slot].double()).to(BF16)
        assert torch.equal(o["x_out"][xrow], s)
        s = s.double()
    y = s if gamma is None else R.norm(s, gamma.double(), eps)
    off = 0.0 if gamma is None else 2.0 ** -23
    why = R.held(o["y8"].view(torch.uint8)[yrow], o["y_scale"][yrow], y, off)
    assert why is None, why
    if o["y16"] is not None:
        near16(o["y16"][yrow], y, off * y.abs().nan_to_num(0), "y16")
    for name, rows, is8 in (("x_out", xrow, False), ("y16", yrow, False), ("y8", yrow, True), ("y_scale", yrow, True)):
        if o[name] is not None:
            rest = torch.ones(len(x), dtype=torch.bool)
            rest[rows] = False
            t = o[name].view(torch.uint8) if is8 else o[name]
            assert (t[rest] == 7).all(), f"{name}: a row that is not in the call was written"


@pytest.mark.parametrize("n,h,add,norm,keep16,live", [
    (1, 128, True, True, True, None), (5, 256, True, True, False, 3), (9, 1024, False, True, True, None),
    (3, 1152, True, True, False, 0), (7, 3584, True, True, True, 6), (4, 4096, False, False, False, 3), (6, 4224, True, True, True, None),
    (3, 8192, True, False, False, None), (2, 8320, True, True, True, None), (3, 18944, True, True, False, 2), (64, 640, True, True, False, 99),
    (300, 384, False, True, True, 299),
])
def test_add_rmsnorm_f8(n, h, add, norm, keep16, live):
    g = gen(n * h)
    x, eps = hidden(g, n, h), 1e-5
    delta = hidden(g, n, h) if add else None
    gamma = (1 + 0.2 * torch.randn(h, generator=g)).to(BF16) if norm else None
    o = run_norm(x, delta, gamma, eps, keep16, n_rows=None if live is None else i32([live]))
    rows = torch.arange(n if live is None else min(live, n))
    check_norm(o, x, delta, gamma, eps, rows, rows, rows)


@pytest.mark.parametrize("x_tok,y_tok", [(True, False), (False, False), (False, True), (True, True)])
def test_add_rmsnorm_f8_rows_of_a_plan(x_tok, y_tok):
    lengths, counts = [40, 1, 77, 9], [13, 1, 77, 0]
    plan = make_plan(lengths)
    rows, n_rows, where = row_lists(lengths, counts, 3)
    g = gen(5)
    for h, most in ((896, 77), (4480, 60)):
        x, delta, gamma = hidden(g, 127, h), hidden(g, 127, h), (1 + 0.2 * torch.randn(h, generator=g)).to(BF16)
        o = run_norm(x, delta, gamma, 1e-6, True, plan=plan, rows=rows, n_rows=n_rows, max_rows=most, x_by_token=x_tok, y_by_token=y_tok)
        use = [p for i, p in enumerate(where) if not (i >= 14 + most)]      # request 2's rows beyond max_rows are left out
        slot = torch.tensor([p[0] for p in use])
        tok = torch.tensor([p[1] for p in use])
        check_norm(o, x, delta, gamma, 1e-6, tok if x_tok else slot, tok if y_tok else slot, slot)
    plan.close()


def test_add_rmsnorm_f8_in_place_and_rows_of_extremes():
    g = gen(7)
    for h in (512, 4096, 9216):
        x, delta = hidden(g, 6, h), hidden(g, 6, h)
        gamma = (1 + 0.2 * torch.randn(h, generator=g)).to(BF16)
        x[1, 3], x[2, 100], x[3], x[4], x[5] = math.nan, math.inf, 0, 3e38, 1e-38
        delta[3:] = 0
        xc = x.cuda()
        y8, ys = torch.zeros(6, h, dtype=F8, device="cuda"), torch.zeros(6, R.ld(h), dtype=torch.uint8, device="cuda")
        sx.add_rmsnorm_f8(xc, y8, ys, gamma=gamma.cuda(), eps=1e-6, delta=delta.cuda(), x_out=xc)
        s = (x.double() + delta.double()).to(BF16)
        assert torch.equal(xc.cpu().view(torch.int16)[[0, 2, 3, 4, 5]], s.view(torch.int16)[[0, 2, 3, 4, 5]])
        y = R.norm(s.double(), gamma.double(), 1e-6)
        why = R.held(bits8(y8), ys.cpu(), y, 2.0 ** -23)
        assert why is None, why
        assert (ys[1, :h // 128] == 255).all() and (ys[2, :h // 128] == 255).sum().item() == 1


# ---------------------------------------------------------------- SwiGLU

@pytest.mark.parametrize("n,f,live", [(1, 128, None), (3, 640, 2), (17, 768, None), (5, 14336, None), (130, 1536, 129), (2, 512, 0),
                                     (22001, 1152, None), (70000, 384, 69990)])
def test_silu_mul_f8(n, f, live):
    g = gen(n + f)
    x = (torch.randn(n, 2 * f, generator=g) * torch.exp(torch.randn(2 * f, generator=g))).to(BF16)
    x[0, 0], x[0, 1], x[0, f + 2] = -80.0, 88.0, 0.0
    y, s = torch.full((n, f), 7, dtype=torch.uint8, device="cuda"), torch.full((n, R.ld(f)), 7, dtype=torch.uint8, device="cuda")
    sx.silu_mul_f8(x.cuda(), y.view(F8), s, n_rows=None if live is None else i32([live]))
    m = n if live is None else live
    why = R.held(y.cpu()[:m], s.cpu()[:m], R.silu_mul(x[:m, :f].double(), x[:m, f:].double()), 2.0 ** -20)
    assert why is None, why
    assert (y.cpu()[m:] == 7).all() and (s.cpu()[m:] == 7).all()


def test_silu_mul_f8_of_every_gate():
    # every bfloat16 from 2^-100 to 80 in magnitude, in groups of like magnitude: 2^-20 of the value (as above)
    bits = torch.arange(1 << 15, dtype=torch.int32)
    v = (bits << 16).view(torch.float32)
    v = v[(v >= 2.0 ** -100) & (v <= 80)]
    v = v[:len(v) // 128 * 128]
    x = torch.stack([torch.cat([v, torch.full_like(v, 1.5)]), torch.cat([-v, torch.full_like(v, -0.75)])]).to(BF16)
    f = len(v)
    y, s = torch.empty(2, f, dtype=torch.uint8, device="cuda"), torch.empty(2, R.ld(f), dtype=torch.uint8, device="cuda")
    sx.silu_mul_f8(x.cuda(), y, s)
    why = R.held(y.cpu(), s.cpu(), R.silu_mul(x[:, :f].double(), x[:, f:].double()), 2.0 ** -20)
    assert why is None, why
    # beyond: 0 where e^-g has no float32, the gate itself above
    x = torch.tensor([[-90.0, -1e4, -3e38, 90.0, 1e4, 3e38] + [0.0] * 122 + [1.0] * 128], dtype=BF16)
    y, s = torch.empty(1, 128, dtype=torch.uint8, device="cuda"), torch.empty(1, 4, dtype=torch.uint8, device="cuda")
    sx.silu_mul_f8(x.cuda(), y, s)
    got = R.rows_of(y.cpu(), s.cpu())[0]
    assert (got[:5] == 0).all() and abs(got[5] / 3e38 - 1) < 2.0 ** -3


def test_silu_mul_f8_rows_of_a_plan_and_infinities():
    lengths, counts, f = [30, 4, 50], [11, 4, 50], 640
    plan = make_plan(lengths)
    g = gen(2)
    x = torch.randn(84, 2 * f, generator=g).to(BF16)
    x[1, 0], x[2, 200], x[3, f + 300], x[31, 639] = math.nan, math.inf, math.inf, -math.inf
    y, s = torch.full((84, f), 7, dtype=torch.uint8, device="cuda"), torch.full((84, R.ld(f)), 7, dtype=torch.uint8, device="cuda")
    sx.silu_mul_f8(x.cuda(), y, s, plan=plan, n_rows=i32(counts), max_rows=50)
    rows = torch.cat([torch.arange(0, 11), torch.arange(30, 34), torch.arange(34, 84)])
    # silu(-inf) is -inf / inf: the group stands for NaN, as one of an infinity does
    gate, up = x[rows, :f].double(), x[rows, f:].double()
    want = R.silu_mul(gate, up)
    want[gate == -math.inf] = math.nan
    why = R.held(y.cpu()[rows], s.cpu()[rows], want, 2.0 ** -20)
    assert why is None, why
    rest = torch.ones(84, dtype=torch.bool)
    rest[rows] = False
    assert (y.cpu()[rest] == 7).all()
    plan.close()


# ---------------------------------------------------------------- products

def operands(g, rows, n, k, wide=False):
    """Rows and a weight in 8 bits, on the CPU; wide: scales far apart from group to group."""
    x = hidden(g, rows, k, torch.float64)
    w = torch.randn(n, k, generator=g, dtype=torch.float64) * k ** -0.5
    if wide:
        x = x * 2.0 ** torch.randint(-40, 41, (rows, k // 128), generator=g).repeat_interleave(128, 1)
        w = w * 2.0 ** torch.randint(-40, 41, (n // 128, k // 128), generator=g).repeat_interleave(128, 0).repeat_interleave(128, 1)
    return (*R.quantise(x), *R.quantise_weight(w))


def run_gemm(xc, xs, wc, ws, parts, res=None, **kw):
    ys = [torch.full((len(xc), p), 7.0, dtype=BF16, device="cuda") for p in parts]
    sx.gemm_f8(xc.cuda().view(F8), xs.cuda(), wc.cuda().view(F8), ws.cuda(), ys, residual=None if res is None else res.cuda(), **kw)
    return [y.cpu() for y in ys]


SHAPES = [(1, 128, 128), (2, 256, 384), (15, 640, 512), (16, 128, 4096), (17, 384, 1152), (33, 1024, 640), (64, 512, 768),
          (65, 256, 2048), (96, 1280, 1024), (130, 896, 1664), (200, 384, 256), (257, 640, 896), (513, 1152, 512), (1, 2048, 14336)]


@pytest.mark.parametrize("rows,n,k", SHAPES)
@pytest.mark.parametrize("wide", [False, True])
def test_gemm_f8(rows, n, k, wide):
    g = gen(rows + n + k)
    xc, xs, wc, ws = operands(g, rows, n, k, wide)
    res = hidden(g, rows, n) if not wide else None
    y, = run_gemm(xc, xs, wc, ws, [n], res)
    want, mag = R.product(xc, xs, wc, ws)
    if res is not None:
        want, mag = want + res.double(), mag + res.double().abs()
    near16(y, want, R.product_bound(k, mag), f"{rows} x {n} x {k}")


@pytest.mark.parametrize("rows", [3, 40, 300])
def test_gemm_f8_is_exact_where_float32_is(rows):
    # whole numbers up to 15 in 1024 products of sums below 2^24: the nearest bfloat16 of the exact sum
    g = gen(rows)
    k, n = 1024, 256
    x = torch.randint(-15, 16, (rows, k), generator=g).double()
    w = torch.randint(-15, 16, (n, k), generator=g).double()
    xc, xs = R.quantise(x)
    wc, ws = R.quantise_weight(w)
    assert torch.equal(R.rows_of(xc, xs), x) and torch.equal(R.weight_of(wc, ws), w)
    y, = run_gemm(xc, xs, wc, ws, [n])
    assert torch.equal(y, (x @ w.t()).float().to(BF16))


def codes(g, rows, k, n=None):
    """Random codes and scale bytes on the GPU, of rows or (with n) of a weight."""
    c = (torch.randn(n or rows, k, generator=g) * 20).clamp(-448, 448).to(F8).view(torch.uint8).cuda()
    s = torch.randint(112, 124, ((n or rows) // (128 if n else 1), R.ld(k)), generator=g).to(torch.uint8).cuda()
    return c, s


# launches of every kernel and tile that a call's size can choose, with runs of tiles and weights that end inside one
LARGE = [(16, 6144, 4096), (40, 4096, 4096), (64, 4224, 4096), (180, 4224, 4096), (394, 4224, 4096), (1000, 3968, 4096),
         (2048, 4096, 4096), (2500, 11136, 2048), (8100, 8064, 512), (4100, 4992, 128), (6400, 4992, 128), (1450, 8320, 128),
         (4900, 6528, 896), (700, 12160, 1152), (20, 4224, 16512), (40, 4224, 16512), (200, 2048, 33280), (600, 2048, 16512),
         (1100, 2048, 16512), (200, 8320, 128), (40, 8320, 512), (2000, 8320, 128), (4100, 4224, 15360)]


@pytest.mark.parametrize("rows,n,k", LARGE)
def test_gemm_f8_large_launches(rows, n, k):
    g = gen(rows + n + k)
    x, xs = codes(g, rows, k)
    w, ws = codes(g, 0, k, n)
    res = torch.randn(rows, n, generator=g).to(BF16).cuda()
    parts = [n - 768, 128, 640]                        # the middle one inside a tile of 256
    ys = [torch.full((rows, p), 7.0, dtype=BF16, device="cuda") for p in parts]
    sx.gemm_f8(x, xs, w, ws, ys)
    y, z = torch.cat(ys, 1), torch.empty_like(res)
    sx.gemm_f8(x, xs, w, ws, z, residual=res)
    # the bits that each row has in a call of its own
    some = sorted({0, rows - 1, rows // 2, *torch.randint(rows, (6,), generator=g).tolist()})
    one, two = torch.empty(len(some), n, dtype=BF16, device="cuda"), torch.empty(len(some), n, dtype=BF16, device="cuda")
    sx.gemm_f8(x[some], xs[some], w, ws, one)
    sx.gemm_f8(x[some], xs[some], w, ws, two, residual=res[some])
    assert torch.equal(y[some], one) and torch.equal(z[some], two)
    # and all rows against calls of 100 rows
    for lo in range(0, rows, 100):
        part = torch.empty(min(100, rows - lo), n, dtype=BF16, device="cuda")
        sx.gemm_f8(x[lo:lo + 100], xs[lo:lo + 100], w, ws, part)
        assert torch.equal(part, y[lo:lo + 100]), f"rows from {lo}"
        sx.gemm_f8(x[lo:lo + 100], xs[lo:lo + 100], w, ws, part, residual=res[lo:lo + 100])
        assert torch.equal(part, z[lo:lo + 100]), f"rows from {lo}, residual"
    want, mag = R.product(x[some[:3]].cpu(), xs[some[:3]].cpu(), w.cpu(), ws.cpu())
    near16(one[:3].cpu(), want, R.product_bound(k, mag), "three rows")
    r = res[some[:3]].cpu().double()
    near16(two[:3].cpu(), want + r, R.product_bound(k, mag + r.abs()), "three rows, residual")


@pytest.mark.parametrize("rows,n,k", [(1, 19200, 4224), (4, 17408, 4096), (3, 20480, 3328), (1, 16512, 5248), (2, 18048, 1664)])
def test_gemm_f8_few_rows_of_many_features(rows, n, k):
    # more than 1024 waves that each read 12 blocks ahead, 13 to 41 blocks of k: every place is refilled, most of them twice.
    # The bits are those of the same rows among 60 others, whose tiles go through LDS
    g = gen(n + k)
    x, xs = codes(g, rows + 60, k)
    w, ws = codes(g, 0, k, n)
    res = torch.randn(rows + 60, n, generator=g).to(BF16).cuda()
    parts = [n - 768, 128, 640]
    ys = [torch.full((rows, p), 7.0, dtype=BF16, device="cuda") for p in parts]
    sx.gemm_f8(x[:rows], xs[:rows], w, ws, ys)
    y, z, all_y, all_z = torch.cat(ys, 1), res[:rows].clone(), torch.empty_like(res), torch.empty_like(res)
    sx.gemm_f8(x[:rows], xs[:rows], w, ws, z, residual=z)
    sx.gemm_f8(x, xs, w, ws, all_y)
    sx.gemm_f8(x, xs, w, ws, all_z, residual=res)
    assert torch.equal(y, all_y[:rows]) and torch.equal(z, all_z[:rows])
    want, mag = R.product(x[:rows].cpu(), xs[:rows].cpu(), w.cpu(), ws.cpu())
    near16(y, want, R.product_bound(k, mag), "streamed")
    r = res[:rows].cpu().double()
    near16(z, want + r, R.product_bound(k, mag + r.abs()), "streamed, residual")


@pytest.mark.parametrize("rows,k", [(5, 65536), (300, 65536), (700, 40064)])
def test_gemm_f8_of_long_rows(rows, k):
    g = gen(rows + k)
    xc, xs, wc, ws = operands(g, rows, 128, k)
    y, = run_gemm(xc, xs, wc, ws, [128])
    want, mag = R.product(xc, xs, wc, ws)
    near16(y, want, R.product_bound(k, mag), f"{rows} x {k}")


def test_gemm_f8_parts_and_padded_batches():
    g = gen(4)
    for rows, live in ((37, 30), (70, 64), (200, 1), (5, 0), (20, 25), (300, 290)):
        parts = [512, 128, 256]
        xc, xs, wc, ws = operands(g, rows, 896, 640)
        xc[live:] = 0x7f                   # rows behind the last one may hold anything
        ys = run_gemm(xc, xs, wc, ws, parts, n_rows=i32([live]))
        m = min(rows, live)
        want, mag = R.product(xc[:m], xs[:m], wc, ws)
        near16(torch.cat([y[:m] for y in ys], 1), want, R.product_bound(640, mag), "parts")
        assert all((y[m:] == 7).all() for y in ys)


def test_gemm_f8_rows_that_stand_for_nan_touch_no_other_row():
    g = gen(6)
    for rows in (20, 90, 300):
        xc, xs, wc, ws = operands(g, rows, 256, 768)
        clean, = run_gemm(xc, xs, wc, ws, [256])
        xs[3, 2] = 255
        xc[rows - 1, 700] = 0x7f
        ws2 = ws.clone()
        y, = run_gemm(xc, xs, wc, ws, [256])
        bad = torch.zeros(rows, dtype=torch.bool)
        bad[[3, rows - 1]] = True
        assert torch.isnan(y[bad]).all() and torch.equal(y[~bad], clean[~bad])
        ws2[1, 0] = 255                    # a block of the weight: its 128 columns
        y, = run_gemm(xc, xs, wc, ws2, [256])
        assert torch.isnan(y[:, 128:]).all() and torch.equal(y[~bad, :128], clean[~bad, :128])


@pytest.mark.parametrize("x_tok,y_tok", [(True, False), (False, True), (False, False), (True, True)])
def test_gemm_f8_rows_of_a_plan(x_tok, y_tok):
    lengths, counts = [150, 1, 300, 20], [133, 1, 290, 0]
    plan = make_plan(lengths)
    rows, n_rows, where = row_lists(lengths, counts, 8)
    g = gen(9)
    total, n, k = sum(lengths), 384, 768
    xc, xs, wc, ws = operands(g, total, n, k)
    res = hidden(g, total, n)
    for most in (300, 200, 17):
        y, = run_gemm(xc, xs, wc, ws, [n], res, plan=plan, rows=rows, n_rows=n_rows, max_rows=most, x_by_token=x_tok,
                      y_by_token=y_tok)
        use = [where[i] for lo, c in ((0, 133), (133, 1), (134, 290)) for i in range(lo, lo + min(c, most))]
        slot, tok = torch.tensor([p[0] for p in use]), torch.tensor([p[1] for p in use])
        xr, yr = tok if x_tok else slot, tok if y_tok else slot
        want, mag = R.product(xc[xr], xs[xr], wc, ws)
        near16(y[yr], want + res[yr].double(), R.product_bound(k, mag + res[yr].double().abs()), f"plan {most}")
        rest = torch.ones(total, dtype=torch.bool)
        rest[yr] = False
        assert (y[rest] == 7).all()
    plan.close()


def test_gemm_f8_of_many_short_requests():
    lengths = [3] * 300
    counts = [(7 * i) % 4 for i in range(300)]
    plan = make_plan(lengths)
    rows, n_rows, where = row_lists(lengths, counts, 15)
    g = gen(15)
    xc, xs, wc, ws = operands(g, 900, 256, 384)
    res = hidden(g, 900, 256)
    y, = run_gemm(xc, xs, wc, ws, [256], res, plan=plan, rows=rows, n_rows=n_rows, max_rows=3, x_by_token=True, y_by_token=True)
    tok = torch.tensor([t for _, t in where])
    want, = run_gemm(xc[tok], xs[tok], wc, ws, [256], res[tok])
    assert torch.equal(y[tok], want)
    rest = torch.ones(900, dtype=torch.bool)
    rest[tok] = False
    assert (y[rest] == 7).all()
    plan.close()


def test_products_on_two_streams_at_once():
    g = gen(16)
    sets = []
    for rows, n, k in ((700, 2048, 1152), (300, 1024, 4096)):
        xc, xs = codes(g, rows, k)
        wc, ws = codes(g, 0, k, n)
        want = torch.empty(rows, n, dtype=BF16, device="cuda")
        sx.gemm_f8(xc, xs, wc, ws, want)
        sets.append((xc, xs, wc, ws, want, torch.empty_like(want), torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(20):
        for xc, xs, wc, ws, want, y, s in sets:
            sx.gemm_f8(xc, xs, wc, ws, y, stream=s)
    torch.cuda.synchronize()
    for *_, want, y, _ in sets:
        assert torch.equal(y, want)


def test_gemm_f8_residual_in_place():
    g = gen(12)
    for rows in (9, 150):
        xc, xs, wc, ws = operands(g, rows, 512, 512)
        res = hidden(g, rows, 512)
        y = res.cuda()
        sx.gemm_f8(xc.cuda(), xs.cuda(), wc.cuda(), ws.cuda(), y, residual=y)
        assert torch.equal(y.cpu(), run_gemm(xc, xs, wc, ws, [512], res)[0])


def test_a_rows_product_does_not_depend_on_the_call():
    # the same rows alone, in larger calls, under looser bounds and through a plan: bit for bit
    g = gen(13)
    n, k = 1024, 1664
    xc, xs, wc, ws = operands(g, 1500, n, k)
    want, = run_gemm(xc, xs, wc, ws, [n])
    for lo, m in ((0, 1), (700, 16), (20, 33), (1000, 64), (5, 100), (300, 257), (0, 700)):
        y, = run_gemm(xc[lo:lo + m], xs[lo:lo + m], wc, ws, [n])
        assert torch.equal(y, want[lo:lo + m]), f"{m} rows from {lo}"
    y = run_gemm(xc, xs, wc, ws, [256, 768], n_rows=i32([10]))
    assert torch.equal(torch.cat(y, 1)[:10], want[:10])
    y, = run_gemm(xc[:40], xs[:40], wc[128:256], ws[1:2], [128])
    assert torch.equal(y, want[:40, 128:256])
    plan = make_plan([900, 600])
    y, = run_gemm(xc, xs, wc, ws, [n], plan=plan, n_rows=i32([900, 5]), max_rows=900)
    assert torch.equal(y[:905], want[:905])
    plan.close()


# ---------------------------------------------------------------- streams, graphs, the checked library

def test_a_layer_captured_and_replayed():
    # norm -> gate|up -> SwiGLU -> down + residual, on a stream of its own, replayed with other inputs and row counts
    g = gen(20)
    rows, h, f = 48, 512, 768
    wg, wd = operands(g, 1, 2 * f, h)[2:], operands(g, 1, h, f)[2:]
    wg, wd = [t.cuda() for t in wg], [t.cuda() for t in wd]
    gamma = (1 + 0.2 * torch.randn(h, generator=g)).to(BF16).cuda()
    x, live = torch.zeros(rows, h, dtype=BF16, device="cuda"), i32([rows])
    a8, as_ = torch.zeros(rows, h, dtype=F8, device="cuda"), torch.zeros(rows, R.ld(h), dtype=torch.uint8, device="cuda")
    gu = torch.zeros(rows, 2 * f, dtype=BF16, device="cuda")
    f8, fs = torch.zeros(rows, f, dtype=F8, device="cuda"), torch.zeros(rows, R.ld(f), dtype=torch.uint8, device="cuda")

    def layer(out):
        sx.add_rmsnorm_f8(x, a8, as_, gamma=gamma, eps=1e-6, n_rows=live)
        sx.gemm_f8(a8, as_, *wg, gu, n_rows=live)
        sx.silu_mul_f8(gu, f8, fs, n_rows=live)
        sx.gemm_f8(f8, fs, *wd, out, residual=x, n_rows=live)

    out = torch.zeros(rows, h, dtype=BF16, device="cuda")
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    layer(out)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        layer(out)
    for seed, n in ((1, 48), (2, 7), (3, 0), (4, 33), (5, 48)):
        x.copy_(hidden(gen(seed), rows, h).cuda())
        live.fill_(n)
        out.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        want = torch.full_like(out, 7)
        layer(want)
        torch.cuda.synchronize()
        assert torch.equal(got, want), f"replay {seed}"
        assert (got[n:] == 7).all()
        if n:
            s = x[:n].double().cpu()
            assert R.held(bits8(a8)[:n], as_.cpu()[:n], R.norm(s, gamma.double().cpu(), 1e-6), 2.0 ** -23) is None
            y, mag = R.product(bits8(f8)[:n], fs.cpu()[:n], wd[0].cpu(), wd[1].cpu())
            near16(got[:n], y + s, R.product_bound(f, mag + s.abs()), "layer")


def test_checked_library_refuses_counts_and_lists():
    sx.use_checked(True)
    try:
        g = gen(21)
        xc, xs, wc, ws = operands(g, 10, 128, 128)
        y, = run_gemm(xc, xs, wc, ws, [128], n_rows=i32([10]))
        assert not (y == 7).all()
        for bad in (-1, 11):
            with pytest.raises(sx.SxError) as e:
                run_gemm(xc, xs, wc, ws, [128], n_rows=i32([bad]))
            assert e.value.status == sx.SX_EDEVICE
            with pytest.raises(sx.SxError) as e:
                sx.silu_mul_f8(torch.zeros(10, 256, dtype=BF16, device="cuda"), xc.cuda(), xs.cuda(), n_rows=i32([bad]))
            assert e.value.status == sx.SX_EDEVICE
        plan = make_plan([10])
        for rows in ([0, 3, 3], [0, 1, 10], [-1, 0, 1]):
            with pytest.raises(sx.SxError) as e:
                run_gemm(xc, xs, wc, ws, [128], plan=plan, rows=i32(rows + [0] * 7), n_rows=i32([3]), max_rows=5, x_by_token=True)
            assert e.value.status == sx.SX_EDEVICE
        plan.close()
    finally:
        sx.use_checked(False)


def test_listed_rows_beyond_their_request_are_left_out():
    plan = make_plan([10, 6])
    g = gen(22)
    xc, xs, wc, ws = operands(g, 16, 128, 256)
    rows = i32([2, 10, 5] + [0] * 7 + [-1, 3, 99] + [0] * 3)
    for x_tok, y_tok in ((True, False), (False, True)):
        y, = run_gemm(xc, xs, wc, ws, [128], plan=plan, rows=rows, n_rows=i32([3, 3]), max_rows=10, x_by_token=x_tok, y_by_token=y_tok)
        use = [(0, 2), (2, 5), (11, 13)]
        xr = torch.tensor([p[1 if x_tok else 0] for p in use])
        yr = torch.tensor([p[1 if y_tok else 0] for p in use])
        want, mag = R.product(xc[xr], xs[xr], wc, ws)
        near16(y[yr], want, R.product_bound(256, mag), "left out")
        rest = torch.ones(16, dtype=torch.bool)
        rest[yr] = False
        assert (y[rest] == 7).all()
        o = run_norm(hidden(g, 16, 256), None, None, 1e-6, False, plan=plan, rows=rows, n_rows=i32([3, 3]), max_rows=10,
                     x_by_token=x_tok, y_by_token=y_tok)
        assert ((o["y_scale"] != 7).any(1).nonzero().flatten() == yr).all()
    plan.close()
