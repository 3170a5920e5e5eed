"""The 8-bit layer body without a GPU: refusals of the C entry points and of the binding, and the references' own checks."""
import ctypes
import math
import re

import pytest
import torch

import f8ref as R
import paper_2606_01751_amd as sx
from test_wait_states_cpu import built  # noqa: F401

A = 1 << 30          # an address that no refused call reads
S = 1 << 26          # arguments lie this far apart


def err(status, want, text):
    assert status == want, sx.lib().sx_last_error().decode()
    assert text in sx.lib().sx_last_error().decode()


def at(i, off=0):
    return A + i * S + off


def placed(defaults, kw):
    """The arguments; far=True: at addresses so far apart that no array reaches the next one."""
    kw = dict(kw)
    up = 32 if kw.pop("far", False) else 0
    move = lambda v: v << up if isinstance(v, int) and v >= A else v  # noqa: E731
    a = {n: tuple(map(move, v)) if isinstance(v, tuple) else move(v) for n, v in defaults.items()}
    a.update(kw)
    return a


def call(name, defaults, order, kw):
    a = placed(defaults, kw)
    return getattr(sx.lib(), name)(*[a[k] for k in order], None)


NORM = dict(plan=None, rows=None, n=at(0), m=5, x=at(1), xt=0, delta=at(2), gamma=at(3), eps=1e-6, h=256, xo=at(4), y16=at(5),
            y8=at(6), ys=at(7), yt=0)
GEMM = dict(plan=None, rows=None, n=at(0), m=5, x=at(1), xs=at(2), xt=0, w=at(3), ws=at(4), k=256, parts=2, part_n=(128, 256),
            res=None, y=(at(5), at(6)), yt=0)
SILU = dict(plan=None, n=at(0), m=5, gu=at(1), f=256, y8=at(2), ys=at(3))
ROUTE = dict(plan=None, n=at(0), m=5, logits=at(1), dt=sx.F32, e=64, top=4, re=1, ids=at(2), wt=at(3), off=at(4), order=at(5),
             ws=at(6), wb=1 << 20)
EXPERTS = dict(off=at(0), order=at(1), e=8, places=40, x=at(2), xs=at(3), xr=10, gather=4, w=at(4), ws=at(5), k=256, n=128,
               y=at(6), scatter=0)
COMBINE = dict(plan=None, rows=None, n=at(0), m=5, y=at(1), wt=at(2), top=4, h=256, res=at(3), out=at(4), ot=0)


def norm(**kw):
    return call("sx_add_rmsnorm_f8", NORM, "plan rows n m x xt delta gamma eps h xo y16 y8 ys yt".split(), kw)


def gemm(**kw):
    a = placed(GEMM, kw)
    pn = None if a["part_n"] is None else (ctypes.c_int32 * 8)(*a["part_n"])
    ys = None if a["y"] is None else (ctypes.c_void_p * 8)(*a["y"])
    return sx.lib().sx_gemm_f8(a["plan"], a["rows"], a["n"], a["m"], a["x"], a["xs"], a["xt"], a["w"], a["ws"], a["k"],
                               a["parts"], pn, a["res"], ys, a["yt"], None)


def silu(**kw):
    return call("sx_silu_mul_f8", SILU, "plan n m gu f y8 ys".split(), kw)


def route(**kw):
    return call("sx_moe_route", ROUTE, "plan n m logits dt e top re ids wt off order ws wb".split(), kw)


def experts(**kw):
    return call("sx_gemm_experts_f8", EXPERTS, "off order e places x xs xr gather w ws k n y scatter".split(), kw)


def combine(**kw):
    return call("sx_moe_combine", COMBINE, "plan rows n m y wt top h res out ot".split(), kw)


V, U, H = sx.SX_EINVAL, sx.SX_EUNSUPPORTED, sx.SX_ESHAPE


@pytest.mark.parametrize("kw,want,text", [
    (dict(m=-1), V, "max_rows"), (dict(rows=at(9)), V, "needs a plan"), (dict(h=0), U, "multiple of 128"),
    (dict(h=200), U, "multiple of 128"), (dict(h=(1 << 24) + 128), U, "above"), (dict(x=None), V, "x is NULL"),
    (dict(y8=None), V, "together"), (dict(ys=None), V, "together"), (dict(xo=None, y16=None, y8=None, ys=None), V, "no output"),
    (dict(delta=None), V, "x_out needs delta"), (dict(gamma=None), V, "y16 needs gamma"), (dict(eps=0.0), V, "eps"),
    (dict(eps=math.nan), V, "eps"), (dict(eps=math.inf), V, "eps"), (dict(x=at(1, 8)), V, "x is not 16-byte"),
    (dict(ys=at(7, 4)), V, "y_scale is not 16-byte"), (dict(xo=at(1, 16)), V, "x_out overlaps x"),
    (dict(xo=at(2)), V, "x_out overlaps delta"), (dict(y16=at(1)), V, "y16 overlaps x"), (dict(y8=at(3, 256)), V, "y8 overlaps gamma"),
    (dict(ys=at(0)), V, "y_scale overlaps n_rows"), (dict(ys=at(6, 5 * 256 - 16)), V, "y8 and y_scale overlap"),
    (dict(m=1 << 24, far=True), U, "exceed one launch"),
])
def test_add_rmsnorm_f8_refusals(kw, want, text):
    err(norm(**kw), want, text)


@pytest.mark.parametrize("kw,want,text", [
    (dict(x=None), V, "NULL"), (dict(xs=None), V, "NULL"), (dict(w=None), V, "NULL"), (dict(ws=None), V, "NULL"),
    (dict(part_n=None), V, "NULL"), (dict(y=None), V, "NULL"), (dict(y=(at(5), None)), V, "part 1 is NULL"),
    (dict(parts=0), V, "n_parts"), (dict(parts=5), V, "n_parts"), (dict(res=at(7)), V, "one part"), (dict(k=64), U, "multiple"),
    (dict(k=65536 + 128), U, "above"), (dict(part_n=(128, 130)), U, "multiple"), (dict(part_n=(0, 128)), U, "multiple"),
    (dict(xs=at(2, 4)), V, "x_scale is not 16-byte"), (dict(y=(at(5), at(6, 2))), V, "not 16-byte"),
    (dict(y=(at(5), at(5, 5 * 256 - 16))), V, "overlap"), (dict(y=(at(1, 5 * 256 - 16), at(6))), V, "overlaps x8"),
    (dict(y=(at(5), at(3, 384 * 256 - 16))), V, "overlaps w8"), (dict(y=(at(5), at(0))), V, "overlaps n_rows"),
    (dict(parts=1, res=at(5, 16)), V, "overlaps residual"), (dict(m=(1 << 31) - 1, part_n=(1 << 23, 1 << 24), n=None, far=True), U, "one launch"),
    (dict(rows=at(9)), V, "needs a plan"), (dict(m=-3), V, "max_rows"),
])
def test_gemm_f8_refusals(kw, want, text):
    err(gemm(**kw), want, text)


@pytest.mark.parametrize("kw,want,text", [
    (dict(f=100), U, "multiple"), (dict(gu=None), V, "NULL"), (dict(ys=None), V, "NULL"), (dict(y8=at(1, 16)), V, "overlaps"),
    (dict(gu=at(1, 2)), V, "16-byte"), (dict(m=-1), V, "max_rows"), (dict(ys=at(2)), V, "overlap"),
    (dict(m=(1 << 26), far=True), U, "one launch"),
])
def test_silu_mul_f8_refusals(kw, want, text):
    err(silu(**kw), want, text)


@pytest.mark.parametrize("kw,want,text", [
    (dict(dt=2), U, "dtype"), (dict(e=0), U, "experts"), (dict(e=1025), U, "experts"), (dict(top=0), U, "top_k"),
    (dict(top=17), U, "top_k"), (dict(e=3), U, "top_k"), (dict(ids=None), V, "NULL"), (dict(ws=None), V, "NULL"),
    (dict(wb=15), H, "workspace"), (dict(m=1 << 30, far=True, wb=1 << 40), U, "2^31"), (dict(off=at(2)), V, "overlap"),
    (dict(order=at(3, 64)), V, "overlap"), (dict(ws=at(1)), V, "overlaps logits"), (dict(wt=at(3, 4)), V, "16-byte"),
    (dict(m=-1), V, "max_rows"), (dict(ids=at(0)), V, "overlaps n_rows"),
])
def test_moe_route_refusals(kw, want, text):
    err(route(**kw), want, text)


@pytest.mark.parametrize("kw,want,text", [
    (dict(e=0), U, "experts"), (dict(e=65537), U, "experts"), (dict(places=-1), V, "negative"), (dict(xr=-1), V, "negative"),
    (dict(gather=-1), V, "negative"), (dict(k=100), U, "multiple"), (dict(n=200), U, "multiple"), (dict(xr=0), H, "no rows"),
    (dict(off=None), V, "NULL"), (dict(order=None), V, "NULL"), (dict(order=None, gather=0, scatter=1), V, "NULL"),
    (dict(y=at(2)), V, "overlaps x8"), (dict(y=at(4, 8 * 128 * 256 - 16)), V, "overlaps w8"), (dict(y=at(1)), V, "overlaps order"),
    (dict(w=at(4, 1)), V, "16-byte"), (dict(k=65536 + 128), U, "above"),
])
def test_gemm_experts_f8_refusals(kw, want, text):
    err(experts(**kw), want, text)


def test_products_of_more_workgroups_than_a_launch_has():
    # a launch has fewer than 2^32 threads: 2^28 rows x 2^21 features are 2^33 tiles of 256 x 256
    err(gemm(m=1 << 28, part_n=(1 << 20, 1 << 20), n=None, far=True), U, "one launch")
    err(gemm(m=(1 << 31) - 1, part_n=(1 << 20, 1 << 20), n=None, far=True), U, "one launch")
    err(experts(e=65536, places=1 << 30, xr=1 << 30, n=1 << 22, far=True), U, "one launch")
    err(experts(e=65536, places=1 << 16, xr=1 << 16, n=1 << 24, far=True), U, "one launch")


@pytest.mark.parametrize("kw,want,text", [
    (dict(top=0), U, "top_k"), (dict(top=17), U, "top_k"), (dict(h=12), U, "multiple of 8"), (dict(h=0), U, "multiple of 8"),
    (dict(y=None), V, "NULL"), (dict(wt=None), V, "NULL"), (dict(out=None), V, "NULL"), (dict(out=at(3, 16)), V, "overlaps residual"),
    (dict(out=at(1)), V, "overlaps y"), (dict(res=at(3, 8)), V, "16-byte"), (dict(m=-1), V, "max_rows"),
])
def test_moe_combine_refusals(kw, want, text):
    err(combine(**kw), want, text)


def test_an_output_may_be_one_input_and_no_other():
    # x_out may be x, y the residual, out the residual: not what else lies at that address
    err(norm(delta=at(1), xo=at(1)), V, "x_out overlaps delta")
    err(norm(gamma=at(1), xo=at(1)), V, "x_out overlaps gamma")
    err(norm(x=at(0), xo=at(0)), V, "x_out overlaps n_rows")
    err(gemm(parts=1, x=at(5), res=at(5)), V, "y overlaps x8")
    err(gemm(parts=1, w=at(5), res=at(5)), V, "y overlaps w8")
    err(gemm(parts=1, ws=at(5), res=at(5)), V, "y overlaps w_scale")
    err(combine(y=at(3), out=at(3)), V, "out overlaps y")
    err(combine(wt=at(3), out=at(3)), V, "out overlaps weights")


def test_nothing_to_do_is_fine():
    ok = sx.SX_OK
    assert norm(m=0) == ok and gemm(m=0) == ok and silu(m=0) == ok and combine(m=0) == ok and experts(places=0, off=None) == ok
    assert sx.lib().sx_f8_pack_weight(None, 0, 128, None, None, None) == ok


def test_arrays_of_no_rows_may_be_null():
    # as empty tensors are
    ok = sx.SX_OK
    assert norm(m=0, x=None, delta=None, xo=None, y16=None, y8=None, ys=None) == ok
    assert gemm(m=0, x=None, xs=None, y=(None, None)) == ok and gemm(m=0, x=None, xs=None, parts=1, y=(None,), res=None) == ok
    assert silu(m=0, gu=None, y8=None, ys=None) == ok and combine(m=0, y=None, wt=None, res=None, out=None) == ok
    assert experts(places=0, xr=0, off=None, order=None, x=None, xs=None, y=None) == ok
    # what has no rows of its own may not
    err(gemm(m=0, w=None), V, "NULL")
    err(gemm(m=0, ws=None), V, "NULL")
    err(gemm(m=0, y=None), V, "NULL")
    err(route(m=0, off=None), V, "NULL")
    err(route(m=0, ws=None), V, "NULL")
    # with rows, nor may they
    err(norm(m=1, x=None), V, "x is NULL")
    err(gemm(m=1, y=(at(5), None)), V, "part 1 is NULL")


@pytest.mark.parametrize("args,want,text", [
    ((at(0), 100, 128, at(1), at(2), None), U, "multiple"), ((at(0), 128, 64, at(1), at(2), None), U, "multiple"),
    ((None, 128, 128, at(1), at(2), None), V, "NULL"), ((at(0), 128, 128, at(0), at(2), None), V, "overlaps"),
    ((at(0), 128, 128, at(1), at(1), None), V, "overlap"), ((at(0, 2), 128, 128, at(1), at(2), None), V, "16-byte"),
])
def test_f8_pack_weight_refusals(args, want, text):
    err(sx.lib().sx_f8_pack_weight(*args), want, text)


def test_scale_ld_and_workspace_sizes():
    for k in (128, 384, 512, 640, 4096, 14336, 65536):
        assert sx.f8_scale_ld(k) == R.ld(k) == -(-(k // 128) // 4) * 4
    with pytest.raises(sx.SxError, match="multiple of 128"):
        sx.f8_scale_ld(64)
    with pytest.raises(ValueError, match="32 bits"):
        sx.f8_scale_ld(1 << 32)
    last = 0
    for rows in (0, 1, 64, 65, 256, 257, 70000, 1 << 20, 1 << 26):
        n = sx.moe_route_workspace(160, 8, rows)
        assert last <= n <= 256 * 160 * 4
        last = n
    for req in (2, 255, 256, 257, 70000):
        assert sx.moe_route_workspace(16, 2, 1000, req) <= 257 * 16 * 4
    for bad in ((0, 1, 1), (8, 9, 1), (2000, 2, 1), (8, 2, -1)):
        with pytest.raises(sx.SxError):
            sx.moe_route_workspace(*bad)


def test_binding_refuses_what_is_not_on_the_gpu():
    x = torch.zeros(4, 256, dtype=torch.bfloat16)
    c, s = torch.zeros(4, 256, dtype=torch.uint8), torch.zeros(4, 4, dtype=torch.uint8)
    for f in (lambda: sx.add_rmsnorm_f8(x, c, s), lambda: sx.gemm_f8(c, s, c, s, x), lambda: sx.silu_mul_f8(x, c, s),
              lambda: sx.moe_combine(x, s, x), lambda: sx.f8_pack_weight(x, c, s),
              lambda: sx.gemm_experts_f8(c, s, c[None], s, s, None, x)):
        with pytest.raises(ValueError, match="not on the current GPU"):
            f()


def test_product_kernels_are_those_that_a_call_can_take(built):  # noqa: F811
    # listed rows: every shape; grouped ones: streamed two by two, or tiles from 128 x 64 on
    rows, grouped = 0, 1
    want = {("stream", (1, 1, 12, rows)), ("stream", (1, 1, 16, rows)), ("stream", (2, 2, 4, grouped)),
            ("narrow", (32, 32, 2, 2, 6, rows)), ("narrow", (64, 32, 2, 2, 6, rows)), ("narrow", (64, 64, 2, 2, 4, rows))}
    for g in (rows, grouped):
        want |= {("narrow", (128, 64, 4, 2, 3, g)), ("narrow", (128, 128, 4, 2, 4, g)), ("pair", (128, 128, 4, 2, 2, g)),
                 ("tile", (256, 256, 2, 2, 2, g))}
    got = set()
    for name, _ in built:
        m = re.search(r"f8_(\w+)_kernelI((?:L[ib]\d+E)+)E", name)
        if m and m[1] in ("stream", "narrow", "pair", "tile"):
            got.add((m[1], tuple(int(v) for v in re.findall(r"L[ib](\d+)E", m[2]))))
    assert got == want


# ---- the references ----

def test_binding_takes_no_number_for_a_count_or_an_order():
    # a raw number would be read as an address
    from paper_2606_01751_amd import layer8
    for bad in (5, 5.0, [5], torch.zeros(0, dtype=torch.int32)):
        with pytest.raises(ValueError, match="int32 tensor"):
            layer8._row_args(None, None, bad, None, 8, 0)
    for bad in (9, 1 << 32, 5 - (1 << 32)):        # (which 32 bits would hold as 9, 0 and 5)
        with pytest.raises(ValueError, match="exceeds"):
            layer8._row_args(None, None, None, bad, 8, 0)
    with pytest.raises(ValueError, match="exceeds"):
        layer8._row_args(None, None, None, None, 1 << 31, 0)
    with pytest.raises(ValueError, match="needs a plan"):
        layer8._row_args(None, torch.zeros(8, dtype=torch.int32), None, 8, 8, 0)


def test_e4m3_reference_against_torch():
    codes = torch.arange(256, dtype=torch.int32).to(torch.uint8)
    want = codes.view(torch.float8_e4m3fn).double()
    got = R.values(codes)
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(), want.nan_to_num())
    g = torch.Generator().manual_seed(0)
    z = torch.cat([torch.randn(20000, generator=g, dtype=torch.float64) * 2.0 ** torch.randint(-12, 7, (20000,), generator=g),
                   R.MAGNITUDES, (R.MAGNITUDES[1:] + R.MAGNITUDES[:-1]) / 2]).clamp(-448, 448).float().double()
    z = torch.cat([z, -z])
    assert torch.equal(R.codes_of(z), z.float().to(torch.float8_e4m3fn).view(torch.uint8))


def test_scale_reference_at_its_borders():
    for e in (-126, -125, -10, 0, 5, 119, 120):
        for m, up in ((448.0, 0), (448.0 * (1 + 2 ** -20), 1), (224.0 * (1 + 2.0 ** -20), 0)):
            want = min(max(e + up, -126), 120) + 127
            assert R.scale_byte(torch.tensor([m * 2.0 ** e], dtype=torch.float64)).item() == want
    assert R.scale_byte(torch.tensor([0.0, math.inf, math.nan], dtype=torch.float64)).tolist() == [1, 255, 255]


def test_held_takes_the_reference_and_no_neighbour():
    g = torch.Generator().manual_seed(1)
    y = torch.randn(6, 640, generator=g, dtype=torch.float64) * torch.exp(3 * torch.randn(6, 1, generator=g, dtype=torch.float64))
    c, s = R.quantise(y)
    assert R.held(c, s, y, 0.0) is None
    for i in range(0, 640, 37):
        for step in (1, -1):
            d = c.clone()
            v = int(d[2, i]) & 127
            if 0 <= v + step <= 126:
                d[2, i] = int(d[2, i]) + step
                assert R.held(d, s, y, 1e-6) == "codes"
    for step in (1, -1):
        t = s.clone()
        t[1, 2] = int(t[1, 2]) + step
        assert R.held(c, t, y, 1e-6) == "scale bytes"
    t = s.clone()
    t[0, -1] = 3
    assert R.held(c, t, y, 0.0) == "padding bytes"


def test_route_reference_ties_and_infinities():
    ids, w = R.route(torch.tensor([[1.0, 3.0, 3.0, 2.0], [math.nan, -math.inf, math.nan, -math.inf],
                                   [math.inf, 0.0, math.inf, 5.0], [-0.0, 0.0, -1.0, 0.0]]), 3, True)
    assert ids.tolist() == [[1, 2, 3], [0, 1, 2], [0, 2, 3], [0, 1, 3]]
    assert w[1].tolist() == [0, 0, 0] and w[2].tolist() == [0.5, 0.5, 0.0]
    assert torch.allclose(w[0].sum(), torch.tensor(1.0, dtype=torch.float64))
    off, order = R.group(ids, [0, 1, 5, 6], 4)
    assert off.tolist() == [0, 3, 6, 9, 12] and order.tolist() == [3, 15, 18, 0, 4, 19, 1, 5, 16, 2, 17, 20]
