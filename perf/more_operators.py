"""Measured cases of the 8-bit layer body: the row-sparse layer body's norm, activation and products with operands in
8-bit floating point, and the feed-forward module as a mixture of experts.

A layer calls them in this order, and every case is one of the calls (`kind`):

  norm     residual addition and RMSNorm of rows, rounded to 8 bits for the next product (without gamma: rounded only)
  gemm     product of 8-bit rows with an 8-bit weight of one or more stacked parts, with a residual or without
  silu     SwiGLU activation of a gate|up product, rounded to 8 bits
  route    the top-k experts of every row, their weights, and the rows grouped by expert
  experts  products of the grouped rows with their expert's 8-bit weight; of the down projection also the weighted sum
           of a row's experts

With `own` false each runs in its plain form: elementary torch operations in 32 bits, rounded once at the end.  With `own`
true it makes the library's calls.

The 8-bit format: 128 consecutive elements of a row share a power of two 2^e, the smallest with amax <= 448 * 2^e and
-126 <= e <= 120, held as the byte e + 127 (255 where the group holds a NaN or an infinity: it stands for NaN); an
element is the nearest e4m3 number (4 bits of exponent, 3 of mantissa, largest 448) times 2^e, ties to even.  A weight
[n][k] shares them over blocks of 128 x 128.  The scale bytes of a row are padded to a multiple of four.
"""
import math

import torch

own = False

GROUP = 128     # elements that share a scale
EPS = 1e-6


def _case(name, kind, **more):
    return {"name": name, "kind": kind, **more}


def listed():
    return [
        # one step of a small decoding batch in a captured graph, a few of its slots empty: launches and latency only
        _case("norm_decode_48", "norm", rows=48, padded=5, width=4096, add=True, norm=True, keep16=False),
        # the long prompt of an agent, 28 heads of 128; a mixture's router reads the norm in 16 bits beside it
        _case("norm_prompt_20k", "norm", rows=19997, padded=0, width=3584, add=True, norm=True, keep16=True),
        # the feed-forward rows of a decoding batch
        _case("silu_decode_17", "silu", rows=17, padded=0, width=14336),
        # 15 % of a 32768-token prompt and its new tokens
        _case("silu_rows_6712", "silu", rows=6712, padded=0, width=14336),
        # queries, keys and values of one decoding step: the weights' bytes bound it
        _case("gemm_qkv_decode_17", "gemm", rows=17, padded=2, k=4096, parts="4096,1024,1024", residual=False),
        # a larger batch through the long down projection
        _case("gemm_down_decode_96", "gemm", rows=96, padded=0, k=14336, parts="4096", residual=True),
        # output projection of the recomputed rows of an 8192-token prompt's last layers
        _case("gemm_out_rows_394", "gemm", rows=394, padded=0, k=4096, parts="4096", residual=True),
        # gate and up projections of the recomputed rows of a 32768-token prompt
        _case("gemm_gate_up_6712", "gemm", rows=6712, padded=0, k=4096, parts="28672", residual=False),
        # routing of one decoding step
        _case("route_decode_64", "route", rows=64, padded=3, experts=128, top=8, dtype="f32", renormalise=True),
        # routing of a long prompt, logits straight from a 16-bit product
        _case("route_prompt_32k", "route", rows=32767, padded=0, experts=128, top=8, dtype="bf16", renormalise=True),
        # gate and up projections of a decoding batch: nearly every expert's weight is read for a few rows
        _case("experts_up_decode_64", "experts", rows=64, padded=0, experts=128, top=8, hidden=2048, ffn=768, part="up"),
        # down projections of a prompt chunk, summed into the residual stream
        _case("experts_down_8k", "experts", rows=8192, padded=0, experts=128, top=8, hidden=2048, ffn=768, part="down"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: any kind, from one row up to the listed work."""
    kind = rng.choice(["norm", "silu", "gemm", "gemm", "gemm", "route", "experts", "experts"])
    if kind == "norm":
        width = GROUP * _log(rng, 1, 64)
        rows = _log(rng, 1, min(32768, 19997 * 3584 // width))
        norm = rng.random() < 0.8
        more = dict(width=width, add=norm and rng.random() < 0.7, norm=norm, keep16=norm and rng.random() < 0.3)
    elif kind == "silu":
        width = GROUP * _log(rng, 1, 148)
        rows = _log(rng, 1, min(32768, 6712 * 14336 // width))
        more = dict(width=width)
    elif kind == "gemm":
        parts = [GROUP * _log(rng, 1, 64) for _ in range(rng.choice([1, 1, 2, 3]))]
        if len(parts) == 1 and rng.random() < 0.5:
            parts[0] = GROUP * _log(rng, 8, 224)
        n = sum(parts)
        k = GROUP * _log(rng, 1, min(112, 28672 * 4096 // (GROUP * n)))
        rows = _log(rng, 1, min(8192, 6712 * 28672 * 4096 // (n * k)))
        more = dict(k=k, parts=",".join(map(str, parts)), residual=len(parts) == 1 and rng.random() < 0.6)
    elif kind == "route":
        experts = rng.choice([8, 16, 64, 128, 160, 256, rng.randint(2, 512)])
        top = min(experts, rng.choice([1, 2, 4, 6, 8]))
        rows = _log(rng, 1, min(32767, 32767 * 128 // experts))
        more = dict(experts=experts, top=top, dtype=rng.choice(["f32", "bf16"]), renormalise=rng.random() < 0.7)
    else:
        experts = rng.choice([4, 8, 16, 64, 128, rng.randint(2, 160)])
        top = min(experts, rng.choice([1, 2, 4, 8]))
        hidden = GROUP * _log(rng, 2, 32)
        ffn = GROUP * _log(rng, 1, max(1, min(56, 128 * 1536 * 2048 // (experts * 2 * hidden * GROUP))))
        rows = _log(rng, 1, max(1, min(8192, 8192 * 8 * 768 * 2048 // (top * 2 * hidden * ffn))))
        more = dict(experts=experts, top=top, hidden=hidden, ffn=ffn, part=rng.choice(["up", "down"]))
    padded = rng.choice([0, 0, 1, 6])
    c = _case(None, kind, rows=rows, padded=padded if rows > padded else 0, **more)
    del c["name"]
    return c


def _parts(case):
    return [int(p) for p in case["parts"].split(",")]


# ---- the 8-bit format in torch ----

def _ld(k):
    """Bytes between the scale rows of rows of k elements."""
    return -(-k // (4 * GROUP)) * 4


def _byte(amax, bad):
    """Scale bytes of groups with these largest magnitudes."""
    bits = amax.view(torch.int32)
    byte = ((bits >> 23) - 8 + ((bits & 0x7fffff) > 0x600000).int()).clamp(1, 247)
    return torch.where(bad, torch.full_like(byte, 255), byte)


def _codes(g, byte):
    """e4m3 codes of elements g whose groups have these scale bytes."""
    inv = ((254 - byte.clamp(max=253)) << 23).view(torch.float32)
    return torch.where(byte == 255, torch.zeros_like(g), g * inv).to(torch.float8_e4m3fn)


def _quantise(x):
    """Rows x [n][k] float32 -> codes [n][k], scale bytes [n][ld], the bytes of the padding 0."""
    n, k = x.shape
    g = x.view(n, k // GROUP, GROUP)
    byte = _byte(g.abs().amax(-1), ~torch.isfinite(g).all(-1))
    scale = torch.zeros(n, _ld(k), dtype=torch.uint8, device=x.device)
    scale[:, :k // GROUP] = byte.to(torch.uint8)
    return _codes(g, byte[..., None]).view(n, k), scale


def _quantise_weight(w):
    """A weight [..., n, k] float32 -> codes and scale bytes [..., n / 128, ld]."""
    *lead, n, k = w.shape
    g = w.view(*lead, n // GROUP, GROUP, k // GROUP, GROUP)
    byte = _byte(g.abs().amax((-3, -1)), torch.zeros((), dtype=torch.bool, device=w.device))
    scale = torch.zeros(*lead, n // GROUP, _ld(k), dtype=torch.uint8, device=w.device)
    scale[..., :k // GROUP] = byte.to(torch.uint8)
    return _codes(g, byte[..., None, :, None]).view(w.shape), scale


def _power(byte):
    return torch.where(byte == 255, math.nan, (byte.int() << 23).view(torch.float32))


def _rows_of(codes, scale):
    """What rows of codes [n][k] stand for, in float32."""
    n, k = codes.shape
    return (codes.float().view(n, -1, GROUP) * _power(scale[:, :k // GROUP])[..., None]).view(n, k)


def _weight_of(codes, scale):
    *lead, n, k = codes.shape
    g = codes.float().view(*lead, n // GROUP, GROUP, k // GROUP, GROUP)
    return (g * _power(scale[..., :k // GROUP])[..., None, :, None]).view(codes.shape)


# ---- inputs ----

def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _hidden(g, n, width):
    """Rows of a residual stream: a few channels far larger than the rest, rows of different sizes."""
    chan = torch.exp(0.3 * _normal(g, width))
    chan[::97] *= 12.0
    return _normal(g, n, width) * chan * torch.exp(0.4 * _normal(g, n, 1))


def _weight(g, n, k):
    return _quantise_weight(_normal(g, n, k) * (k ** -0.5))


def _expert_weights(g, e, n, k):
    """Weights [e][n][k], drawn for a few experts at a time to keep the float32 values small."""
    step = max(1, (1 << 27) // (n * k))
    made = [_quantise_weight(_normal(g, min(step, e - i), n, k) * (k ** -0.5)) for i in range(0, e, step)]
    return torch.cat([m[0].view(torch.uint8) for m in made]).view(torch.float8_e4m3fn), torch.cat([m[1] for m in made])


def _logits(g, rows, experts):
    """Router logits: some experts are taken far more often than others."""
    return 1.5 * _normal(g, rows, experts) + 0.8 * _normal(g, experts)


def _top(logits, top, renormalise):
    """(ids, weights) of the top experts of every row, the lower index first among equals."""
    x = logits.float()
    ids = torch.sort(x, dim=-1, descending=True, stable=True).indices[:, :top]
    p = torch.exp(x - x.amax(-1, keepdim=True))
    w = torch.gather(p, 1, ids)
    return ids.int(), w / (w.sum(-1, keepdim=True) if renormalise else p.sum(-1, keepdim=True))


def _group(ids, experts):
    """(offsets, order): the places of ids [rows][top], taken in order, grouped by expert."""
    flat = ids.flatten().long()
    order = torch.sort(flat, stable=True).indices.int()
    count = torch.zeros(experts + 1, dtype=torch.int64, device=ids.device).index_add(0, flat + 1, torch.ones_like(flat))
    return torch.cumsum(count, 0).int(), order


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 2 + 1)
    kind, rows = case["kind"], case["rows"]
    live = rows - case["padded"]
    # `count`: how many rows of the batch's arrays are in use, known on the device only; None: all of them
    s = {"case": case, "kind": kind, "keep": {}, "live": live,
         "count": torch.tensor([live], dtype=torch.int32, device="cuda") if case["padded"] else None}
    zeros8 = lambda n, k: torch.zeros(n, k, dtype=torch.float8_e4m3fn, device="cuda")  # noqa: E731
    bytes_ = lambda n, k: torch.zeros(n, _ld(k), dtype=torch.uint8, device="cuda")  # noqa: E731
    zeros16 = lambda *shape: torch.zeros(*shape, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    if kind == "norm":
        h = case["width"]
        s["x"] = _hidden(g, rows, h).bfloat16()
        s["delta"] = (0.5 * _normal(g, rows, h)).bfloat16() if case["add"] else None
        s["gamma"] = (1 + 0.2 * _normal(g, h)).bfloat16() if case["norm"] else None
        s["x_out"] = zeros16(rows, h) if case["add"] else None
        s["y16"] = zeros16(rows, h) if case["keep16"] else None
        s["y"], s["scale"] = zeros8(rows, h), bytes_(rows, h)
    elif kind == "silu":
        f = case["width"]
        s["x"] = (_normal(g, rows, 2 * f) * torch.exp(0.3 * _normal(g, 2 * f))).bfloat16()
        s["y"], s["scale"] = zeros8(rows, f), bytes_(rows, f)
    elif kind == "gemm":
        k, parts = case["k"], _parts(case)
        s["x"], s["xs"] = _quantise(_hidden(g, rows, k))
        s["w"], s["ws"] = _weight(g, sum(parts), k)
        s["res"] = _hidden(g, rows, parts[0]).bfloat16() if case["residual"] else None
        s["y"] = [zeros16(rows, p) for p in parts]
    else:
        e, top = case["experts"], case["top"]
        logits = _logits(g, rows, e)
        if kind == "route":
            s["logits"] = logits if case["dtype"] == "f32" else logits.bfloat16()
            s["ids"] = torch.zeros(rows, top, dtype=torch.int32, device="cuda")
            s["weights"] = torch.zeros(rows, top, device="cuda")
            s["offsets"] = torch.zeros(e + 1, dtype=torch.int32, device="cuda")
            s["order"] = torch.zeros(rows * top, dtype=torch.int32, device="cuda")
        else:
            h, f, up = case["hidden"], case["ffn"], case["part"] == "up"
            n, k = (2 * f, h) if up else (h, f)
            ids, s["weights"] = _top(logits, top, True)
            s["offsets"], order = _group(ids[:live], e)
            s["order"] = torch.cat([order, torch.zeros(case["padded"] * top, dtype=torch.int32, device="cuda")])
            s["most"] = int((s["offsets"][1:] - s["offsets"][:-1]).max())
            s["x"], s["xs"] = _quantise(_hidden(g, rows if up else rows * top, k))
            s["w"], s["ws"] = _expert_weights(g, e, n, k)
            s["y"] = zeros16(rows * top, n)
            if not up:
                s["res"], s["out"] = _hidden(g, rows, h).bfloat16(), zeros16(rows, h)
    return s


# ---- one pass ----

def run(s):
    return (_own if own else _plain)[s["kind"]](s)


def _powers(scale):
    """The scale bytes as the powers of two that they stand for."""
    return scale.view(torch.float8_e8m0fnu)


def _own_norm(s):
    import paper_2606_01751_amd as sx
    sx.add_rmsnorm_f8(s["x"], s["y"], s["scale"], gamma=s["gamma"], eps=EPS, delta=s["delta"], x_out=s["x_out"],
                      y16=s["y16"], n_rows=s["count"])
    return {"x": s["x_out"], "y16": s["y16"], "y": s["y"], "scale": _powers(s["scale"])}


def _own_silu(s):
    import paper_2606_01751_amd as sx
    sx.silu_mul_f8(s["x"], s["y"], s["scale"], n_rows=s["count"])
    return {"y": s["y"], "scale": _powers(s["scale"])}


def _own_gemm(s):
    import paper_2606_01751_amd as sx
    sx.gemm_f8(s["x"], s["xs"], s["w"], s["ws"], s["y"], residual=s["res"], n_rows=s["count"])
    return s["y"]


def _own_route(s):
    import paper_2606_01751_amd as sx
    c, keep = s["case"], s["keep"]
    if "workspace" not in keep:     # kept by the program from step to step
        size = sx.moe_route_workspace(c["experts"], c["top"], c["rows"])
        keep["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    sx.moe_route(s["logits"], s["ids"], s["weights"], s["offsets"], s["order"], keep["workspace"],
                 renormalise=c["renormalise"], n_rows=s["count"])
    return {n: s[n] for n in ("ids", "weights", "offsets", "order")}


def _own_experts(s):
    import paper_2606_01751_amd as sx
    top = s["case"]["top"]
    if s["case"]["part"] == "up":
        sx.gemm_experts_f8(s["x"], s["xs"], s["w"], s["ws"], s["offsets"], s["order"], s["y"], gather=top)
        return s["y"]
    sx.gemm_experts_f8(s["x"], s["xs"], s["w"], s["ws"], s["offsets"], s["order"], s["y"], scatter=True)
    sx.moe_combine(s["y"], s["weights"], s["out"], residual=s["res"], n_rows=s["count"])
    return s["out"]


def _kept(s, new, old):
    """The rows in use from `new`, the others as `old` has them."""
    if s["live"] == old.shape[0]:
        return new
    if old.dtype is torch.float8_e4m3fn:
        return torch.cat([new[:s["live"]].view(torch.uint8), old[s["live"]:].view(torch.uint8)]).view(old.dtype)
    return torch.cat([new[:s["live"]], old[s["live"]:]])


def _plain_norm(s):
    x, x_out, y16 = s["x"], None, None
    if s["delta"] is not None:
        x = (x.float() + s["delta"].float()).bfloat16()
        x_out = _kept(s, x, s["x_out"])
    y = x.float()
    if s["gamma"] is not None:
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * s["gamma"].float()
    if s["y16"] is not None:
        y16 = _kept(s, y.bfloat16(), s["y16"])
    codes, scale = _quantise(y)
    return {"x": x_out, "y16": y16, "y": _kept(s, codes, s["y"]), "scale": _powers(_kept(s, scale, s["scale"]))}


def _plain_silu(s):
    f = s["case"]["width"]
    gate, up = s["x"][:, :f].float(), s["x"][:, f:].float()
    codes, scale = _quantise(gate / (1 + torch.exp(-gate)) * up)
    return {"y": _kept(s, codes, s["y"]), "scale": _powers(_kept(s, scale, s["scale"]))}


def _plain_gemm(s):
    y = torch.matmul(_rows_of(s["x"], s["xs"]), _weight_of(s["w"], s["ws"]).t())
    if s["res"] is not None:
        y += s["res"].float()
    return [_kept(s, p.bfloat16(), o) for p, o in zip(y.split(_parts(s["case"]), 1), s["y"])]


def _plain_route(s):
    c, live = s["case"], s["live"]
    ids, weights = _top(s["logits"], c["top"], c["renormalise"])
    offsets, order = _group(ids[:live], c["experts"])
    return {"ids": _kept(s, ids, s["ids"]), "weights": _kept(s, weights, s["weights"]), "offsets": offsets,
            "order": torch.cat([order, s["order"][live * c["top"]:]])}


def _plain_experts(s):
    c = s["case"]
    top, e, up, places = c["top"], c["experts"], c["part"] == "up", s["live"] * c["top"]
    # every expert's rows, padded to the busiest expert's
    at = s["offsets"][:-1, None].long() + torch.arange(s["most"], device="cuda")
    mine = at < s["offsets"][1:, None]
    at = at.clamp(max=max(0, places - 1))
    order = s["order"].long()
    x = _rows_of(s["x"], s["xs"])[order[at] // top if up else at]                   # [e][most][k]
    y = torch.bmm(x, _weight_of(s["w"], s["ws"]).transpose(1, 2).contiguous())[mine]   # in the order of the places
    if up:
        return _kept({"live": places}, y.bfloat16(), s["y"])
    y = torch.zeros_like(y).index_copy_(0, order[:places], y).view(s["live"], top, -1)
    out = (y * s["weights"][:s["live"], :, None]).sum(1) + s["res"][:s["live"]].float()
    return _kept(s, out.bfloat16(), s["out"])


_own = {"norm": _own_norm, "silu": _own_silu, "gemm": _own_gemm, "route": _own_route, "experts": _own_experts}
_plain = {"norm": _plain_norm, "silu": _plain_silu, "gemm": _plain_gemm, "route": _plain_route,
          "experts": _plain_experts}


# ---- what a pass cannot do without ----

def work(case):
    kind, rows = case["kind"], case["rows"] - case["padded"]
    if kind == "norm":
        h = case["width"]
        row = h * (2 + 4 * case["add"] + 1 + 2 * case["keep16"]) + h // GROUP
        return {"bytes": rows * row + 2 * h * case["norm"], "flops": rows * h * (1 + case["add"] + 4 * case["norm"])}
    if kind == "silu":
        f = case["width"]
        return {"bytes": rows * (5 * f + f // GROUP), "flops": rows * f * 6}
    if kind == "gemm":
        k, n = case["k"], sum(_parts(case))
        held = k + k // GROUP
        return {"bytes": rows * held + n * k + (n // GROUP) * (k // GROUP) + rows * n * (4 if case["residual"] else 2),
                "flops": 2 * rows * n * k}
    e, top = case["experts"], case["top"]
    if kind == "route":
        return {"bytes": rows * (e * (4 if case["dtype"] == "f32" else 2) + 12 * top) + 4 * (e + 1),
                "flops": rows * e * 3}
    h, f, up = case["hidden"], case["ffn"], case["part"] == "up"
    n, k = (2 * f, h) if up else (h, f)
    # an expert's weight is read when a row takes it: expected for rows that take `top` of the experts at random
    taken = e * (1 - (1 - top / e) ** rows)
    x_rows = rows if up else rows * top
    more = rows * top * n * 2 if up else rows * (4 * h + 4 * top)
    return {"bytes": int(taken * (n * k + (n // GROUP) * (k // GROUP))) + x_rows * (k + k // GROUP) + 4 * rows * top + more,
            "flops": 2 * rows * top * n * k}


# ---- the definitions in 64 bits ----

def _exact_scale(y):
    """The power of two of every group of rows y [n][k] (float64): tried from the logarithm, one up and one down."""
    amax = y.abs().view(y.shape[0], -1, GROUP).amax(-1)
    e = torch.ceil(torch.log2(amax / 448)).clamp(-126, 120)
    e = torch.where(torch.ldexp(torch.full_like(e, 448.0), e.int()) < amax, e + 1, e)
    return torch.where((torch.ldexp(torch.full_like(e, 448.0), (e - 1).int()) >= amax) & (e > -126), e - 1, e)


def _exact_held(y, live):
    """Rows of y in units of their groups' powers of two: what the codes round; 0 behind the rows in use."""
    e = _exact_scale(y).repeat_interleave(GROUP, 1)
    z = torch.ldexp(y, -e.int())
    z[live:] = 0
    return z


_MAGNITUDES = [(m / 8 if not x else 1 + m / 8) * 2.0 ** (max(x, 1) - 7) for x in range(16) for m in range(8)]


def _exact_codes(codes):
    """e4m3 numbers from their bits: sign, 4 bits of exponent (bias 7, 0 for subnormals), 3 of mantissa."""
    t = torch.tensor(_MAGNITUDES, dtype=torch.float64, device=codes.device)
    b = codes.contiguous().view(torch.uint8).int()
    return torch.where(b >= 128, -1.0, 1.0).double() * t[(b & 127).long()]


def _exact_spread(byte, n):
    """Powers of two of the first n groups' bytes, once for every element."""
    return torch.ldexp(torch.ones((), dtype=torch.float64, device=byte.device), byte[:, :n].int() - 127).repeat_interleave(GROUP, 1)


def _exact_rows(codes, scale):
    return _exact_codes(codes) * _exact_spread(scale, codes.shape[1] // GROUP)


def _exact_weight(codes, scale):
    return _exact_codes(codes) * _exact_spread(scale, codes.shape[1] // GROUP).repeat_interleave(GROUP, 0)


def exact(case, seed):
    s = prepare(case, seed)
    kind, live = case["kind"], s["live"]
    if kind == "norm":
        h = s["x"].double() if s["delta"] is None else s["x"].double() + s["delta"].double()
        y = h.bfloat16().double()               # the norm is of the residual stream as it is kept
        if s["gamma"] is not None:
            y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / case["width"] + EPS) * s["gamma"].double()
        y16 = None if s["y16"] is None else y.clone()
        for t in (h, y16):
            if t is not None:
                t[live:] = 0
        return {"x": None if s["delta"] is None else h, "y16": y16, "y": _exact_held(y, live), "scale": None}
    if kind == "silu":
        gate, up = s["x"].double().chunk(2, 1)
        return {"y": _exact_held(gate * torch.sigmoid(gate) * up, live), "scale": None}
    if kind == "gemm":
        y = _exact_rows(s["x"], s["xs"]) @ _exact_weight(s["w"], s["ws"]).t()
        if s["res"] is not None:
            y += s["res"].double()
        y[live:] = 0
        return list(torch.split(y, _parts(case), 1))
    top = case["top"]
    if kind == "route":
        x = s["logits"].double()
        ids = _top(s["logits"], top, False)[0].long()
        p = torch.softmax(x, -1).gather(1, ids)
        if case["renormalise"]:
            p = p / p.sum(-1, keepdim=True)
        p[live:] = 0
        return {"ids": None, "weights": p, "offsets": None, "order": None}
    up, order, offsets = case["part"] == "up", s["order"].long(), s["offsets"].tolist()
    x = _exact_rows(s["x"], s["xs"])
    y = torch.zeros(s["y"].shape, dtype=torch.float64, device="cuda")
    for i, (a, b) in enumerate(zip(offsets, offsets[1:])):
        if b > a:
            w = _exact_weight(s["w"][i], s["ws"][i]).t()
            if up:
                y[a:b] = x[order[a:b] // top] @ w
            else:
                y[order[a:b]] = x[a:b] @ w
    if up:
        return y
    out = (y.view(case["rows"], top, -1) * s["weights"].double()[..., None]).sum(1) + s["res"].double()
    out[live:] = 0
    return out
