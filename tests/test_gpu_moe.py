"""Mixtures of experts on the GPU against float64 references (f8ref.py): routing, products by expert, the weighted sum.

Tolerances.  A weight is one exponential (2 units, 2^-22), a sum of up to n of them in float32 (n + 2^2 half steps) and a
quotient (2.5 units).  Products: f8ref.product_bound; the weighted sum adds top_k + 1 float32 roundings of its terms, and
its inputs y are taken as the products stored them."""
import math

import pytest
import torch

import f8ref as R
import paper_2606_01751_amd as sx
from test_gpu_f8 import BF16, F8, codes, gen, hidden, i32, make_plan, near16, operands, bits8

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    sx.lib()


def run_route(logits, top, renormalise=True, n_req=1, most=None, **kw):
    n, e = logits.shape
    o = dict(ids=torch.full((n, top), -7, dtype=torch.int32, device="cuda"), weights=torch.full((n, top), -7.0, device="cuda"),
             offsets=torch.full((e + 1,), -7, dtype=torch.int32, device="cuda"),
             order=torch.full((n * top,), -7, dtype=torch.int32, device="cuda"))
    ws = torch.full((sx.moe_route_workspace(e, top, n if most is None else most, n_req),), 0xcd, dtype=torch.uint8, device="cuda")
    if most is not None:
        kw["max_rows"] = most
    sx.moe_route(logits.cuda(), o["ids"], o["weights"], o["offsets"], o["order"], ws, renormalise=renormalise, **kw)
    return {k: v.cpu() for k, v in o.items()}


def check_route(o, logits, top, renormalise, slots):
    n, e = logits.shape
    ids, w = R.route(logits[slots], top, renormalise)
    assert torch.equal(o["ids"][slots], ids)
    bound = (2.0 ** -20 + (top if renormalise else e) * R.E) * w + 1e-37
    assert ((o["weights"][slots].double() - w).abs() <= bound).all()
    off, order = R.group(ids, slots.tolist(), e)
    assert torch.equal(o["offsets"], off)
    assert torch.equal(o["order"][:len(order)], order)
    assert (o["order"][len(order):] == -7).all()
    rest = torch.ones(n, dtype=torch.bool)
    rest[slots] = False
    assert (o["ids"][rest] == -7).all() and (o["weights"][rest] == -7).all()


@pytest.mark.parametrize("n,e,top,dtype,renormalise,live", [
    (1, 8, 2, "f32", True, None), (1, 1, 1, "bf16", False, None), (3, 16, 16, "f32", False, None), (64, 128, 8, "f32", True, 61),
    (64, 2, 1, "bf16", True, 0), (65, 64, 6, "bf16", True, None), (255, 160, 8, "f32", True, None), (256, 17, 3, "bf16", False, 256),
    (257, 256, 8, "bf16", True, 250), (1000, 257, 4, "f32", False, None), (700, 512, 16, "bf16", True, 699), (130, 513, 7, "f32", True, None),
    (300, 1024, 16, "bf16", False, 299), (5000, 128, 8, "bf16", True, None), (70000, 12, 2, "f32", True, 69999), (64, 1000, 10, "f32", True, None),
])
def test_moe_route(n, e, top, dtype, renormalise, live):
    g = gen(n + e)
    logits = 1.5 * torch.randn(n, e, generator=g) + torch.randn(e, generator=g)
    logits = logits.to(BF16) if dtype == "bf16" else logits
    o = run_route(logits, top, renormalise, n_rows=None if live is None else i32([live]))
    check_route(o, logits, top, renormalise, torch.arange(n if live is None else min(live, n)))


@pytest.mark.parametrize("e", [5, 100, 200, 700])
def test_moe_route_ties_infinities_and_nan(e):
    g = gen(e)
    top = 5
    logits = torch.randint(-2, 3, (200, e), generator=g).float()      # ties everywhere
    logits[0], logits[1], logits[2] = math.nan, -math.inf, math.inf
    logits[3, ::2], logits[4, 1:] = math.nan, -math.inf
    logits[5, e // 2], logits[6] = math.inf, 0.0
    logits[6, ::3] = -0.0
    logits[7], logits[8, 0] = 3e38, -3e38
    logits[9] = torch.where(torch.arange(e) % 2 == 0, -math.inf, math.nan)
    for ren in (True, False):
        check_route(run_route(logits, top, ren), logits, top, ren, torch.arange(200))
        check_route(run_route(logits.to(BF16), top, ren), logits.to(BF16), top, ren, torch.arange(200))


@pytest.mark.parametrize("lengths,counts,most", [
    ([40, 1, 77, 9], [13, 1, 77, 0], 77), ([300, 1000, 64], [300, 900, 64], 900), ([700, 20], [600, 20], 130),
    ([2] * 300, [i % 3 for i in range(300)], 2), ([64], [40], 64), ([5] * 70, [4] * 70, 3),
])
def test_moe_route_rows_of_a_plan(lengths, counts, most):
    plan = make_plan(lengths)
    e, top, total = 48, 4, sum(lengths)
    logits = torch.randn(total, e, generator=gen(total))
    o = run_route(logits, top, True, len(lengths), most, plan=plan, n_rows=i32(counts))
    slots, off = [], 0
    for n, c in zip(lengths, counts):
        slots += range(off, off + min(c, most))
        off += n
    check_route(o, logits, top, True, torch.tensor(slots, dtype=torch.long))
    plan.close()


# ---------------------------------------------------------------- products by expert

def expert_weights(g, e, n, k):
    made = [operands(g, 1, n, k)[2:] for _ in range(e)]
    return torch.stack([m[0] for m in made]), torch.stack([m[1] for m in made])


def run_experts(xc, xs, wc, ws, off, order, places, **kw):
    y = torch.full((places, wc.shape[1]), 7.0, dtype=BF16, device="cuda")
    sx.gemm_experts_f8(xc.cuda().view(F8), xs.cuda(), wc.cuda().view(F8), ws.cuda(), off.cuda(), None if order is None else order.cuda(),
                       y, **kw)
    return y.cpu()


def want_experts(xc, xs, wc, ws, off, order, places, gather, scatter, n, k):
    want = torch.full((places, n), 7.0, dtype=torch.float64)
    mag = torch.zeros(places, n, dtype=torch.float64)
    for e in range(wc.shape[0]):
        p = torch.arange(int(off[e]), int(off[e + 1]))
        if len(p):
            xr = order[p].long() // gather if gather else p
            yr = order[p].long() if scatter else p
            want[yr], mag[yr] = R.product(xc[xr], xs[xr], wc[e], ws[e])
    return want, R.product_bound(k, mag)


@pytest.mark.parametrize("rows,e,top,n,k,skew", [
    (1, 8, 2, 128, 128, 0), (5, 4, 2, 256, 384, 0), (64, 16, 4, 384, 256, 0), (40, 130, 3, 128, 640, 0), (300, 6, 2, 256, 512, 2),
    (700, 8, 4, 128, 384, 4), (33, 3, 1, 896, 1152, 0), (900, 2, 1, 384, 128, 9), (257, 5, 5, 640, 256, 0),
])
def test_gemm_experts_f8(rows, e, top, n, k, skew):
    g = gen(rows + e + n)
    logits = torch.randn(rows, e, generator=g) - skew * torch.arange(e) / e * 4
    o = run_route(logits, top)
    off, order, places = o["offsets"], o["order"], rows * top
    wc, ws = expert_weights(g, e, n, k)
    for gather, scatter in ((top, False), (0, True), (top, True), (0, False)):
        xc, xs = operands(g, rows if gather else places, 128, k)[:2]
        y = run_experts(xc, xs, wc, ws, off, order if gather or scatter else None, places, gather=gather, scatter=scatter)
        want, bound = want_experts(xc, xs, wc, ws, off, order, places, gather, scatter, n, k)
        near16(y, want, bound, f"gather {gather} scatter {scatter}")


def test_gemm_experts_f8_places_not_in_use_and_bad_entries():
    g = gen(31)
    e, top, rows, n, k = 6, 2, 50, 128, 256
    logits = torch.randn(rows, e, generator=g)
    logits[:, 2] = -50                     # an expert that no row takes
    o = run_route(logits, top, n_rows=i32([41]))
    off, order = o["offsets"], o["order"]
    assert off[2] == off[3] and off[-1] == 82
    wc, ws = expert_weights(g, e, n, k)
    xc, xs = operands(g, rows, 128, k)[:2]
    y = run_experts(xc, xs, wc, ws, off, order, 100, gather=top)
    want, bound = want_experts(xc, xs, wc, ws, off, order, 100, top, False, n, k)
    near16(y, want, bound, "in use")
    assert (y[82:] == 7).all()
    bad = order.clone()
    bad[3], bad[40], bad[81] = -1, 100, 1 << 30    # left out: their places are not written
    for scatter in (False, True):
        y = run_experts(xc, xs, wc, ws, off, bad, 100, gather=top, scatter=scatter)
        out = [int(order[p]) for p in (3, 40, 81)] if scatter else [3, 40, 81]
        want, bound = want_experts(xc, xs, wc, ws, off, order, 100, top, scatter, n, k)
        want[out], bound[out] = 7, 0
        near16(y, want, bound, "left out")
    # fewer rows of x than the order names
    y = run_experts(xc[:20], xs[:20], wc, ws, off, order, 100, gather=top)
    want, bound = want_experts(xc, xs, wc, ws, off, order, 100, top, False, n, k)
    short = torch.tensor([p for p in range(82) if int(order[p]) // top >= 20])
    want[short], bound[short] = 7, 0
    near16(y, want, bound, "short x")
    # offsets cut to n_places
    cut = off.clone()
    cut[-1] = 500
    y = run_experts(xc, xs, wc, ws, cut, order.clamp(0, 99), 100, gather=top)
    assert torch.equal(y[:int(off[-2])], run_experts(xc, xs, wc, ws, off, order, 100, gather=top)[:int(off[-2])])
    sx.use_checked(True)
    try:
        run_experts(xc, xs, wc, ws, off, order, 100, gather=top)
        for a, b in ((off, bad), (cut, order), (off.flip(0), order)):
            with pytest.raises(sx.SxError) as err:
                run_experts(xc, xs, wc, ws, a, b, 100, gather=top)
            assert err.value.status == sx.SX_EDEVICE
        with pytest.raises(sx.SxError) as err:
            run_experts(xc[:20], xs[:20], wc, ws, off, order, 100, gather=top)
        assert err.value.status == sx.SX_EDEVICE
    finally:
        sx.use_checked(False)


@pytest.mark.parametrize("scatter", [False, True])
def test_places_behind_the_rows_of_x(scatter):
    # without gather a place is a row of x itself: the release library leaves those out that x does not have, the checked one refuses
    g = gen(33)
    n, k, sizes, have = 128, 256, [10, 0, 25, 7], 30
    off = torch.tensor([0, 10, 10, 35, 42], dtype=torch.int32)
    order = torch.randperm(50, generator=g).int() if scatter else None
    wc, ws = expert_weights(g, len(sizes), n, k)
    xc, xs = operands(g, 42, 128, k)[:2]
    want = run_experts(xc, xs, wc, ws, off, order, 50, scatter=scatter)
    short = run_experts(xc[:have], xs[:have], wc, ws, off, order, 50, scatter=scatter)
    out = order[have:42].long() if scatter else torch.arange(have, 42)
    want[out] = 7
    assert torch.equal(short, want)
    sx.use_checked(True)
    try:
        run_experts(xc, xs, wc, ws, off, order, 50, scatter=scatter)
        with pytest.raises(sx.SxError) as err:
            run_experts(xc[:have], xs[:have], wc, ws, off, order, 50, scatter=scatter)
        assert err.value.status == sx.SX_EDEVICE
    finally:
        sx.use_checked(False)


def test_an_experts_rows_are_those_of_the_plain_product():
    # the same bits as gemm_f8 with that expert's weight, however many rows the others have
    g = gen(32)
    n, k, sizes = 256, 896, [1, 0, 300, 17, 64, 0, 130, 2]
    off = torch.tensor([sum(sizes[:i]) for i in range(9)], dtype=torch.int32)
    wc, ws = expert_weights(g, 8, n, k)
    xc, xs = operands(g, 514, 128, k)[:2]
    y = run_experts(xc, xs, wc, ws, off, None, 514)
    z = run_experts(xc, xs, wc, ws, off, None, 3000)
    assert torch.equal(y, z[:514]) and (z[514:] == 7).all()
    for e, m in enumerate(sizes):
        if m:
            a = int(off[e])
            one = torch.zeros(m, n, dtype=BF16, device="cuda")
            sx.gemm_f8(xc[a:a + m].cuda(), xs[a:a + m].cuda(), wc[e].cuda(), ws[e].cuda(), one)
            assert torch.equal(one.cpu(), y[a:a + m]), f"expert {e}"


@pytest.mark.parametrize("e,places,n,k,even", [
    (16, 250, 1024, 512, False), (128, 6000, 2176, 768, True), (4, 6800, 1280, 256, False), (32, 7200, 1152, 256, True),
    (4, 1280, 7040, 256, False), (4, 3000, 2176, 1664, False), (8, 160, 7552, 128, False), (64, 6040, 2048, 512, False),
    (8, 8000, 4224, 512, False), (16, 5050, 2048, 256, False), (8, 7100, 5504, 128, False), (1100, 2000, 128, 128, False),
    (6, 4000, 2176, 16512, False), (2, 40, 128, 40064, True), (64, 8000, 1920, 128, True), (8, 128, 7296, 128, True),
    (4, 1200, 1408, 512, False), (4, 70, 384, 1152, False),
])
def test_large_grouped_launches(e, places, n, k, even):
    # the bits of gemm_f8, expert by expert, under a list of places and where each goes
    g = gen(places + n)
    counts = torch.bincount(torch.arange(places) % e if even else (torch.rand(places, generator=g) ** 2 * e).long(), minlength=e)
    off = torch.cat([torch.zeros(1, dtype=torch.long), counts.cumsum(0)]).int()
    made = [codes(g, 0, k, n) for _ in range(min(e, 16))]
    wc, ws = (torch.stack([made[i % 16][j] for i in range(e)]) for j in (0, 1))
    x, xs = codes(g, places, k)
    order = torch.randperm(places, generator=g).int().cuda()
    y = torch.full((places + 3, n), 7.0, dtype=BF16, device="cuda")
    sx.gemm_experts_f8(x, xs, wc, ws, off.cuda(), torch.cat([order, order[:3]]), y, gather=1)
    z = torch.full((places + 3, n), 7.0, dtype=BF16, device="cuda")
    sx.gemm_experts_f8(x, xs, wc, ws, off.cuda(), torch.cat([order, order[:3]]), z, scatter=True)
    assert (y[places:] == 7).all() and (z[places:] == 7).all()
    for i in range(e):
        a, b = int(off[i]), int(off[i + 1])
        if a < b:
            p = order[a:b].long()
            one = torch.empty(b - a, n, dtype=BF16, device="cuda")
            sx.gemm_f8(x[p], xs[p], *made[i % 16], one)
            assert torch.equal(y[a:b], one), f"gather, expert {i}"
            sx.gemm_f8(x[a:b], xs[a:b].clone(), *made[i % 16], one)
            assert torch.equal(z[p], one), f"scatter, expert {i}"


# ---------------------------------------------------------------- the weighted sum

@pytest.mark.parametrize("rows,top,h,live,add", [(1, 1, 8, None, False), (5, 8, 640, 3, True), (33, 3, 2048, None, True),
                                                 (200, 16, 136, 199, False), (7, 2, 4096, 0, True)])
def test_moe_combine(rows, top, h, live, add):
    g = gen(rows + top + h)
    y, w = torch.randn(rows * top, h, generator=g).to(BF16), torch.rand(rows, top, generator=g)
    w[0, 0] = 0
    y[0] = math.nan                        # of weight 0: left out
    res = hidden(g, rows, h) if add else None
    out = torch.full((rows, h), 7.0, dtype=BF16, device="cuda")
    sx.moe_combine(y.cuda(), w.cuda(), out, residual=None if res is None else res.cuda(), n_rows=None if live is None else i32([live]))
    m = rows if live is None else live
    t = torch.where((w == 0)[..., None], 0.0, y.view(rows, top, h).double() * w[..., None].double())
    want, mag = t.sum(1), t.abs().sum(1)
    if add:
        want, mag = want + res.double(), mag + res.double().abs()
    near16(out[:m], want[:m], ((top + 1) * R.E * mag)[:m], "combine")
    assert (out[m:] == 7).all()
    if add:
        r = res.cuda()
        sx.moe_combine(y.cuda(), w.cuda(), r, residual=r)
        full = torch.zeros_like(r)
        sx.moe_combine(y.cuda(), w.cuda(), full, residual=res.cuda())
        assert torch.equal(r, full) and torch.equal(full[:m], out[:m])


def test_moe_combine_rows_of_a_plan():
    lengths, counts, top, h = [20, 3, 40], [11, 3, 40], 2, 256
    plan = make_plan(lengths)
    g = gen(5)
    rows = torch.zeros(63, dtype=torch.int32)
    rows[:11] = torch.tensor([0, 1, 3, 4, 6, 9, 10, 12, 15, 18, 19], dtype=torch.int32)
    rows[20:23], rows[23:63] = torch.arange(3, dtype=torch.int32), torch.arange(40, dtype=torch.int32)
    y, w, res = torch.randn(126, h, generator=g).to(BF16), torch.rand(63, top, generator=g), hidden(g, 63, h)
    out = torch.full((63, h), 7.0, dtype=BF16, device="cuda")
    sx.moe_combine(y.cuda(), w.cuda(), out, residual=res.cuda(), plan=plan, rows=rows.cuda(), n_rows=i32(counts), max_rows=30, out_by_token=True)
    slot = torch.tensor(list(range(11)) + list(range(20, 23)) + list(range(23, 53)))
    tok = torch.tensor([int(rows[i]) for i in range(11)] + list(range(20, 23)) + list(range(23, 53)))
    t = y.view(63, top, h)[slot].double() * w[slot][..., None].double()
    near16(out[tok], t.sum(1) + res[tok].double(), 3 * R.E * (t.abs().sum(1) + res[tok].double().abs()), "plan")
    rest = torch.ones(63, dtype=torch.bool)
    rest[tok] = False
    assert (out[rest] == 7).all()
    plan.close()


def test_a_mixture_captured_and_replayed():
    # norm -> route -> gate|up of the grouped rows -> SwiGLU -> down -> weighted sum, replayed with other inputs and row counts;
    # the eager calls run on a stream of their own with a workspace of their own
    g = gen(40)
    rows, h, f, e, top = 70, 256, 384, 12, 3
    wg, wd = [t.cuda() for t in expert_weights(g, e, 2 * f, h)], [t.cuda() for t in expert_weights(g, e, h, f)]
    gamma = (1 + 0.2 * torch.randn(h, generator=g)).to(BF16).cuda()
    wr = (torch.randn(e, h, generator=g) * h ** -0.5).cuda()
    x, live = torch.zeros(rows, h, dtype=BF16, device="cuda"), i32([rows])

    def buffers():
        z = lambda *s, d=BF16: torch.zeros(*s, dtype=d, device="cuda")  # noqa: E731
        p = rows * top
        return dict(a8=z(rows, h, d=F8), as_=z(rows, R.ld(h), d=torch.uint8), a16=z(rows, h), ids=z(rows, top, d=torch.int32),
                    w=z(rows, top, d=torch.float32), off=z(e + 1, d=torch.int32), order=z(p, d=torch.int32),
                    ws=z(sx.moe_route_workspace(e, top, rows), d=torch.uint8), gu=z(p, 2 * f), f8=z(p, f, d=F8),
                    fs=z(p, R.ld(f), d=torch.uint8), y=z(p, h), out=z(rows, h))

    def layer(b):
        sx.add_rmsnorm_f8(x, b["a8"], b["as_"], gamma=gamma, eps=1e-6, y16=b["a16"], n_rows=live)
        logits = b["a16"].float() @ wr.t()
        sx.moe_route(logits, b["ids"], b["w"], b["off"], b["order"], b["ws"], n_rows=live)
        sx.gemm_experts_f8(b["a8"], b["as_"], *wg, b["off"], b["order"], b["gu"], gather=top)
        sx.silu_mul_f8(b["gu"], b["f8"], b["fs"], n_rows=b["off"][-1:])
        sx.gemm_experts_f8(b["f8"], b["fs"], *wd, b["off"], b["order"], b["y"], scatter=True)
        sx.moe_combine(b["y"], b["w"], b["out"], residual=x, n_rows=live)

    one, two = buffers(), buffers()
    layer(one)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer(one)
    side = torch.cuda.Stream()
    for seed, n in ((1, 70), (2, 9), (3, 0), (4, 64), (5, 70)):
        x.copy_(hidden(gen(seed), rows, h).cuda())
        live.fill_(n)
        one["out"].fill_(7)
        two["out"].fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(side):
            layer(two)
        torch.cuda.synchronize()
        assert torch.equal(one["out"], two["out"]), f"replay {seed}"
        assert (one["out"][n:] == 7).all() and int(one["off"][-1]) == n * top
        if not n:
            continue
        b = {k: v.cpu() for k, v in one.items()}
        ids, w = R.route((b["a16"][:n].float().cuda() @ wr.t()).cpu(), top, True)
        assert torch.equal(b["ids"][:n], ids)
        want = x[:n].double().cpu()
        mag = want.abs()
        # from the stored activations on: products rounded to bfloat16, then the weighted sum
        place = {int(o): p for p, o in enumerate(b["order"][:n * top])}
        for j in range(top):
            for i in range(n):
                p = place[i * top + j]
                ex = int(b["ids"][i, j])
                t, m = R.product(bits8(one["f8"])[p:p + 1], b["fs"][p:p + 1], wd[0][ex].cpu(), wd[1][ex].cpu())
                near16(b["y"][i * top + j][None], t, R.product_bound(f, m), "down")
        t = b["y"].view(rows, top, h)[:n].double() * b["w"][:n, :, None].double()
        near16(b["out"][:n], want + t.sum(1), (top + 1) * R.E * (mag + t.abs().sum(1)), "mixture")


def test_batches_of_no_rows():
    # every call of both chains; a routing of no rows has offsets of 0
    g = gen(41)
    h, f, e, top = 256, 384, 6, 2
    wg, wd = [t.cuda() for t in expert_weights(g, e, 2 * f, h)], [t.cuda() for t in expert_weights(g, e, h, f)]
    gamma = torch.ones(h, dtype=BF16, device="cuda")
    z = lambda *s, d=BF16: torch.zeros(*s, dtype=d, device="cuda")  # noqa: E731
    x, a8, as_ = z(0, h), z(0, h, d=F8), z(0, R.ld(h), d=torch.uint8)
    off = torch.full((e + 1,), -7, dtype=torch.int32, device="cuda")
    ws = z(sx.moe_route_workspace(e, top, 0), d=torch.uint8)
    ids, w, order = z(0, top, d=torch.int32), z(0, top, d=torch.float32), z(0, d=torch.int32)
    sx.add_rmsnorm_f8(x, a8, as_, gamma=gamma, delta=z(0, h), x_out=x, y16=z(0, h))
    sx.add_rmsnorm_f8(x, a8, as_)
    sx.gemm_f8(a8, as_, wg[0][0], wg[1][0], [z(0, f), z(0, f)])
    sx.gemm_f8(z(0, f, d=F8), z(0, R.ld(f), d=torch.uint8), wd[0][0], wd[1][0], x, residual=x)
    for dtype in (torch.float32, BF16):
        for n_rows in (None, i32([3])):     # (whatever a padded batch's count says)
            off.fill_(-7)
            sx.moe_route(z(0, e, d=dtype), ids, w, off, order, ws, n_rows=n_rows)
            assert not off.any()
    gu, f8, fs = z(0, 2 * f), z(0, f, d=F8), z(0, R.ld(f), d=torch.uint8)
    sx.gemm_experts_f8(a8, as_, *wg, off, order, gu, gather=top)
    sx.silu_mul_f8(gu, f8, fs, n_rows=off[-1:])
    sx.gemm_experts_f8(f8, fs, *wd, off, order, z(0, h), scatter=True)
    sx.moe_combine(z(0, h), w, x, residual=x)
    torch.cuda.synchronize()
