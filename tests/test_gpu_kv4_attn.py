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


def dense(b, r, table=None):
    """K, V float64 [keys][Hkv][d] of request r on the GPU, as sx_kv4_read gives them, and which keys have a block."""
    t = torch.arange(b.nk[r])
    ids = (b.table if table is None else table)[r, t // 16].long()
    ok = (ids >= 0) & (ids < b.pool.shape[0])
    slots = torch.where(ok, ids * 16 + t % 16, torch.full_like(ids, -1)).int().cuda()
    k, v = (torch.zeros(b.nk[r], b.hkv, b.d, device="cuda") for _ in range(2))
    sx.kv4_read(sx.make_desc(b.hkv, b.hkv, b.d, "f32", 1e4), b.pool, slots, k, v)
    return k.double(), v.double(), ok.cuda()


def attention64(b, r, table=None):
    """(out, lse, their bounds) of request r in float64 on the GPU.  A score of d products and its exponent (2^-24 each), sums of up
    to m terms and the division, twice, as in kv4ref.attention: for the lse as it is, for the result times sum w |v| over the softmax
    weights w, with the parts of a probability (2^-16 for two, 2^-22 for three; 2^-8 and that for the divisor for one) on top."""
    n, m, grp = b.nq[r], b.nk[r], b.hq // b.hkv
    k, v, ok = dense(b, r, table)
    hidden = ~((torch.arange(m, device="cuda")[None] <= torch.arange(m - n, m, device="cuda")[:, None]) & ok[None])
    scale = b.d ** -0.5
    out = torch.zeros(n, b.hq, b.d, dtype=torch.float64, device="cuda")
    lse, bound = torch.zeros(n, b.hq, dtype=torch.float64, device="cuda"), torch.zeros_like(out)
    lse_bound = torch.zeros_like(lse)
    parts = 2.0 ** -22 if b.dtype == "f32" else 2.0 ** -16 if n * grp <= 128 else 2.0 ** -7
    for h in range(b.hq):
        kh, vh, qh = k[:, h // grp].contiguous(), v[:, h // grp].contiguous(), b.q[b.cu[r]:b.cu[r + 1], h].double()
        s = (qh @ kh.t().contiguous() * scale).masked_fill_(hidden, -math.inf)
        lse[:, h] = s.logsumexp(-1)
        mag = (qh.abs() @ kh.abs().t().contiguous()).amax(-1) * scale
        w = s.softmax(-1)
        out[:, h] = w @ vh
        err = 2 * (mag * (b.d + 4) * 2.0 ** -24 + 2.0 ** -22 * (mag + 1) + m * 2.0 ** -24 + 2.0 ** -22)
        bound[:, h] = (err + parts)[:, None] * (w @ vh.abs())
        lse_bound[:, h] = err + 2.0 ** -22 * (1 + lse[:, h].abs())
    return out, lse, bound, lse_bound


def agrees(b, out, lse, r, table=None):
    want, wl, bound, lse_bound = attention64(b, r, table)
    eps = torch.finfo(out.dtype).eps
    got = out[b.cu[r]:b.cu[r + 1]].double()
    off = (got - want).abs() - (bound + eps / 2 * (want.abs() + bound))
    assert off.max().item() <= 0, (r, off.max().item())
    gl = lse[b.cu[r]:b.cu[r + 1]].double()
    assert ((gl - wl).abs() - lse_bound).max().item() <= 0, r


def marked(b, chunk, keys, step):
    """Request 0's values become 0 but in the blocks around the listed keys of every chunk, which have 1 in a column each: a block left
    out, or taken for another, moves a column of few blocks.  Returns a table without every other of these blocks, or with ids
    that are none."""
    n, t, j = b.nk[0], b.table.clone(), 0
    v = torch.zeros(n, 1, b.d)
    bad = (-1, b.pool.shape[0], -5, (1 << 31) - 1)
    last = (n - 1) // 16
    for c in range(-(-n // chunk)):
        for key in keys:
            first = (c * chunk + key) // 16 + c % step
            for blk in (first, first + 1) if key < chunk else ():
                if blk <= last:
                    v[blk * 16:blk * 16 + 16, 0, j % b.d] = 1
                    j += 1
                    if j % 2:
                        t[0, blk] = bad[j // 2 % 4]
    v[last * 16:, 0, 0] = 1
    at = torch.arange(n)
    k, _, _ = dense(b, 0)
    put(b, 0, at, k, v)
    return t


@pytest.mark.parametrize("hq,d,dtype,nq", [(4, 64, "bf16", 1), (1, 64, "bf16", 17), (2, 64, "f32", 1), (1, 64, "f32", 20)])
def test_few_rows_over_chunks_of_more_than_8192_keys(hq, d, dtype, nq):
    # 64 chunks, the most there are, of 66 x 128 keys: a wave loads the ids of its 32 steps at the chunk's keys 0, 4096 and 8192
    b = Batch([(nq, 540000)], hq, 1, d, dtype, seed=nq)
    chunk = 66 * 128
    assert (540000 + chunk - 1) // chunk == 64
    t = marked(b, chunk, (0, 32, 4064, 4096, 4096 + 96, 4224, 8160, 8192, 8192 + 128, 8400), 8)
    agrees(b, *b.run(), 0)
    agrees(b, *b.run(table=t), 0, t)


@pytest.mark.parametrize("hq,d,nq,nk,chunk", [(4, 64, 2048, 20000, 20 * 128), (4, 128, 300, 70000, 11 * 128), (1, 128, 2000, 50000, 13 * 128)])
def test_many_rows_over_chunks_of_more_than_16_tiles(hq, d, nq, nk, chunk):
    # ids come 16 tiles of 64 keys at a time; 70000 keys of 1200 rows make 50 chunks, which the merge takes in two rounds
    b = Batch([(nq, nk)], hq, 1, d, "bf16", seed=nq)
    rows = nq * hq
    most = min(65536 // rows, 64)
    units = -(-nk // 128)
    assert -(-units // most) * 128 == chunk and nk > most * 1024
    t = marked(b, chunk, (0, 48, 63 + 14 * 64, 15 * 64, 16 * 64 - 16, 16 * 64 + 32, 17 * 64, 32 * 64 - 16, 32 * 64 + 16, 33 * 64 + 48), 4)
    agrees(b, *b.run(), 0)
    agrees(b, *b.run(table=t), 0, t)


def test_merge_of_more_than_32_chunks_by_one_wave_a_row():
    # few rows and float32, more than 1024 (token, head) rows a call: 69 chunks' worth of keys in 64
    for hq, dtype, sizes in ((128 // 16, "bf16", [(16, 70000)] * 9), (8, "f32", [(33, 66000)] * 4)):
        b = Batch(sizes[:1], hq, 1, 64, dtype, seed=3)
        b.nq, b.nk = [s[0] for s in sizes], [s[1] for s in sizes]
        b.nk[1] -= 1000
        b.table = b.table.repeat(len(sizes), 1)
        b.cu = [sizes[0][0] * i for i in range(len(sizes) + 1)]
        b.q = torch.randn(b.cu[-1], hq, 64, generator=torch.Generator().manual_seed(1)).to(b.q.dtype).cuda()
        out, lse = b.run()
        for r in (0, 1, len(sizes) - 1):
            agrees(b, out, lse, r)


def test_many_rows_with_missing_blocks_and_nan_in_the_same_tiles():
    # 150 tokens of 2 heads a KV head: the last tiles are seen by some rows only; NaN in values of present blocks, behind the last
    # key, and in a block that is not there
    b = Batch([(150, 410), (70, 80), (1, 20)], 4, 2, 128, "bf16", seed=4)
    nan = torch.full((1, 2, 128), 0.5)
    nan[0, 1, 40] = math.nan
    for r, at in ((0, 300), (0, 345), (0, 391), (0, 415), (1, 33), (1, 70)):
        put(b, r, [at], torch.full((1, 2, 128), 0.25), nan)
    t = b.table.clone()
    t[0, 3], t[0, 16], t[0, 345 // 16], t[0, 24], t[1, 0], t[1, 70 // 16] = -1, b.pool.shape[0], -1, -3, -1, (1 << 31) - 1
    out, _ = b.check(table=t)
    assert out[:150].isnan().any() and not out[0].isnan().any()
    b.check()


@pytest.mark.parametrize("dtype,nq", [("f32", 4), ("bf16", 4), ("bf16", 70), ("f32", 70)])
def test_infinite_queries(dtype, nq):
    # an infinite query element: every score of the row is -inf where the keys' element is positive (an empty row), +inf and with it
    # NaN where one is negative; the other rows keep their bits
    d = 64
    b = Batch([(nq, 100), (2, 50)], 4, 2, d, dtype, seed=nq)
    for r, n in ((0, 100), (1, 50)):
        k = torch.randn(n, 2, d, generator=torch.Generator().manual_seed(r))
        k[:, :, 5] = 1.0
        put(b, r, range(n), k, torch.randn(n, 2, d))
    put(b, 1, [20], -torch.ones(1, 2, d), torch.ones(1, 2, d))
    before, _ = b.run()
    b.q[1, 2, 5] = -math.inf
    b.q[nq + 1, 0, 5] = -math.inf
    out, lse = b.check()
    assert (out[1, 2] == 0).all() and lse[1, 2] == -math.inf and out[nq + 1, 0].isnan().all()
    out[1, 2], out[nq + 1, 0] = before[1, 2], before[nq + 1, 0]
    assert torch.equal(out, before)


def every_code(d):
    """A pool in which K and V rows hold every byte of codes under every scale 2^-126 .. 2^125 and NaN, and their values."""
    import kv4ref as R
    scales = torch.tensor(list(range(1, 253)) + [255])
    bytes_ = torch.arange(256).view(16, 16)
    groups = scales.numel() * 16                                # one of 16 bytes, 32 elements, each
    n = -(-groups // (d // 32))
    at = torch.arange(n * (d // 32)) % groups
    code = bytes_[at % 16]
    el = torch.stack([code & 15, code >> 4], -1).reshape(-1, 32)
    s = scales[at // 16]
    val = R.MAG[el & 7] * torch.where(el >= 8, -1.0, 1.0).double()
    val = torch.where(s[:, None] == 255, torch.full_like(val, math.nan), torch.ldexp(val, (s - 127)[:, None].int()))
    el, val, s = el.view(n, d).to(torch.uint8), val.view(n, d), s.view(n, d // 32).to(torch.uint8)
    pool = torch.zeros(-(-n // 16), 1, R.record(d), dtype=torch.uint8)
    for i in range(n):
        rec = pool[i // 16, 0]
        ko, vo, kso, vso, hi = R.offsets(d, i % 16)
        for o, sc in ((ko, kso), (vo, vso)):
            rec[o[0::2]] = el[i, 0::2] | el[i, 1::2] << 4
            rec[sc[::32]] = s[i]
    return pool, val


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_code_under_every_scale_reads_exactly(d, dtype):
    from test_gpu_decode import DT
    pool, val = every_code(d)
    n, desc = val.shape[0], sx.make_desc(1, 1, d, dtype, 1e4)
    k, v = (torch.zeros(n, 1, d, dtype=DT[dtype], device="cuda") for _ in range(2))
    sx.kv4_read(desc, pool.cuda(), i32(range(n)), k, v)
    for x in (k, v):
        assert torch.equal(x[:, 0].cpu().double().nan_to_num(1e300), val.nan_to_num(1e300))
        assert torch.equal(x[:, 0].cpu().signbit()[~val.isnan()], val.signbit()[~val.isnan()])
    # back to 4 bits: the same values again (the scale may be another where the group has no large element)
    again = torch.zeros_like(pool).cuda()
    sx.kv4_write(desc, k, v, i32(range(n)), again)
    k2, v2 = torch.zeros_like(k), torch.zeros_like(v)
    sx.kv4_read(desc, again, i32(range(n)), k2, v2)
    assert torch.equal(k2.nan_to_num(1e30), k.nan_to_num(1e30)) and torch.equal(v2.nan_to_num(1e30), v.nan_to_num(1e30))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype,nq", [("bf16", 1), ("f32", 1), ("bf16", 130)])
def test_attention_of_one_key_returns_its_value_for_every_code(d, dtype, nq):
    # requests of one key each, K zero: the result is the value, exactly (within what sums hold: 2^72)
    pool, val = every_code(d)
    pick = torch.nonzero((val.abs().amax(-1) <= 2.0 ** 60) & (val.abs().amax(-1) >= 2.0 ** -60)).flatten()
    pick = pick[:: 1 if nq == 1 else 29]
    n = len(pick)
    from test_gpu_decode import DT
    zero_k = torch.zeros(pool.shape[0] * 16, 1, d, device="cuda")
    p, vals = pool.cuda(), torch.zeros(pool.shape[0] * 16, 1, d, device="cuda")
    sx.kv4_read(sx.make_desc(1, 1, d, "f32", 1e4), p, i32(range(pool.shape[0] * 16)), zero_k.clone(), vals)
    # a block for every request: its first token the row, the others (behind the last key) NaN
    one = torch.full((n, 1, pool.shape[2]), 0xFF, dtype=torch.uint8, device="cuda")
    sx.kv4_write(sx.make_desc(1, 1, d, "f32", 1e4), zero_k[pick.cuda()], vals[pick.cuda()], i32(range(n)) * 16, one)
    q = torch.randn(n * nq, 1, d, generator=torch.Generator().manual_seed(1)).to(DT[dtype]).cuda()
    out = torch.empty_like(q)
    desc = sx.make_desc(1, 1, d, dtype, 1e4)
    sx.kv4_attn(desc, q, i32(range(0, (n + 1) * nq, nq)), i32([1] * n), i32(range(n))[:, None].contiguous(), one, out, nq, 1,
                torch.empty(16, dtype=torch.uint8, device="cuda"))
    last = out.view(n, nq, d)[:, -1].cpu().double()             # (the other rows stand before the first key)
    assert torch.equal(last, val[pick]) and (out.view(n, nq, d)[:, :-1] == 0).all()


@pytest.mark.parametrize("hq,hkv,d,sizes", [(8, 2, 64, [(1, 777), (1, 3000)]), (8, 2, 128, [(1, 777), (5, 4000)]), (4, 1, 128, [(60, 1500)]),
                                            (2, 2, 64, [(130, 900)])])
def test_float32_keeps_its_precision(hq, hkv, d, sizes):
    # relative RMS error below 1e-6: three bfloat16 parts of q and of the probabilities leave 2^-24 of each, two would leave 2^-17
    # and about 4e-6 (test_kv4_parts_cpu.py)
    b = Batch(sizes, hq, hkv, d, "f32", seed=d)
    out, _ = b.run()
    for r in range(len(sizes)):
        want = attention64(b, r)[0]
        off = out[b.cu[r]:b.cu[r + 1]].double() - want
        assert (off.square().mean().sqrt() / want.square().mean().sqrt()).item() < 1e-6


@pytest.mark.parametrize("nq", [1, 20])
def test_the_largest_float32_queries(nq):
    # finite values above the largest bfloat16 (255 * 2^120): their first part is that, not infinity, so that a key element of 0
    # takes no part in the score and one of 2^-120 a finite one
    d = 64
    b = Batch([(nq, 90)], 4, 2, d, "f32", seed=nq)
    k = torch.randn(90, 2, d, generator=torch.Generator().manual_seed(1))
    k[:, :, 32:] = 0
    put(b, 0, range(90), k, torch.randn(90, 2, d))
    b.q[:, :, 40] = 0
    want, want_lse = b.run()
    for big in (torch.finfo(torch.float32).max, -255.5 * 2.0 ** 120, 255.0 * 2.0 ** 120):
        b.q[:, :, 40] = big
        out, lse = b.run()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
    k[:, :, 40] = 2.0 ** -120 * torch.randint(-6, 7, (90, 2), generator=torch.Generator().manual_seed(2))
    put(b, 0, range(90), k, torch.randn(90, 2, d))
    b.q[:, :, 40] = 255.75 * 2.0 ** 120
    b.check()
