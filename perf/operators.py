"""Measured cases of the decoding operators: appending to, and attending over, a KV cache held in 4 bits.

A serving loop calls them in this order, and every case is one of the calls (`kind`):

  slots   block tables and slot maps of a batch of requests that each append tokens
  qk      per-head RMSNorm of queries and keys, and their rotation to the tokens' positions
  rows    token rows written into 4-bit cache blocks by slot, and read back by slot
  blocks  whole blocks of the 16- or 32-bit paged cache packed into 4-bit blocks, and unpacked again
  attn    attention of every request's last tokens over its 4-bit blocks

With `own` false each runs in its plain form: elementary torch operations in 32 bits (angles in 64), rounded once at the
end.  With `own` true it makes the library's calls.

The 4-bit cache (16 tokens a block): 32 consecutive elements of a head's row share a power of two 2^e, the smallest with
amax <= 7 * 2^e and -126 <= e <= 125, held as the byte e + 127 (255 where the group holds a NaN or an infinity: it reads
as NaN); an element is the sign and the nearest of {0, .5, 1, 1.5, 2, 3, 4, 6} times 2^e, ties to the even code.  The
order of a block's bytes is at `_lay`.
"""
import math
import random

import torch

own = False

BLOCK = 16      # tokens of a cache block
GROUP = 32      # elements that share a scale
EPS = 1e-6
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _case(name, kind, heads, dtype="bf16", **more):
    hq, hkv, d = heads
    return {"name": name, "kind": kind, "q_heads": hq, "kv_heads": hkv, "head_dim": d, "dtype": dtype, **more}


def listed():
    small, llama, agent, narrow = (8, 2, 64), (32, 8, 128), (28, 4, 128), (16, 4, 64)
    return [
        # one step of a small decoding batch: launches and latency only
        _case("slots_decode_64", "slots", llama, requests=64, tokens=64, most=4096),
        # prompts and running requests mixed in one step, 131072 new tokens
        _case("slots_mixed_128k", "slots", llama, requests=300, tokens=131072, most=8192),
        # a few rows of an accuracy-first float32 model, far positions, padded to the captured batch size
        _case("qk_f32_decode_19", "qk", small, "f32", tokens=19, padded=5, rope="gptj", norm=True, far=True),
        # one step of a large decoding batch
        _case("qk_decode_256", "qk", llama, tokens=256, padded=0, rope="neox", norm=True, far=True),
        # the prompt chunk of a long request, 28 query heads
        _case("qk_prompt_32k", "qk", agent, tokens=32768, padded=0, rope="neox", norm=True, far=False),
        # one step's new rows of a batch, slots all over the pool
        _case("rows_decode_96", "rows", llama, tokens=96, padded=7, pool=4096),
        # the prefilled cache of a long chat goes into 4-bit blocks and comes back for the next prompt
        _case("blocks_chat_32k", "blocks", llama, count=2048),
        # one request's first answer tokens, float32
        _case("attn_f32_one_777", "attn", small, "f32", requests=1, queries=1, keys=777, empty=False),
        # one long conversation alone on the card: few rows, a long axis
        _case("attn_one_128k", "attn", llama, requests=1, queries=1, keys=131072, empty=False),
        # a serving batch of ragged lengths, 7 query heads per KV head, one slot of the batch idle
        _case("attn_batch_64", "attn", agent, requests=64, queries=1, keys=8192, empty=True),
        # drafted tokens of a batch checked in one pass, narrow heads
        _case("attn_drafts_24", "attn", narrow, requests=24, queries=5, keys=6000, empty=False),
        # a prompt chunk over its long 4-bit history
        _case("attn_chunk_2k", "attn", llama, requests=1, queries=2048, keys=32768, empty=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: any kind, one token up to the listed sizes, any listed data type and head shape."""
    kind = rng.choice(["slots", "qk", "rows", "blocks", "attn", "attn", "attn"])
    heads = rng.choice([(32, 8, 128), (28, 4, 128), (8, 2, 64), (16, 4, 64), (8, 1, 128), (8, 8, 64), (32, 2, 128)])
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    if kind == "slots":
        n = _log(rng, 1, 512)
        tokens = n if rng.random() < 0.4 else n + _log(rng, 1, 130000)
        c = _case(None, kind, heads, requests=n, tokens=tokens, most=rng.choice([512, 4096, 8192]))
    elif kind == "qk":
        n = _log(rng, 1, 32768 if dtype == "bf16" else 8192)
        c = _case(None, kind, heads, dtype, tokens=n, padded=rng.choice([0, 0, 1, 9]) if n > 9 else 0,
                  rope=rng.choice(["neox", "neox", "gptj"]), norm=rng.random() < 0.8, far=n <= 512)
    elif kind == "rows":
        n = _log(rng, 1, 4096)
        c = _case(None, kind, heads, dtype, tokens=n, padded=rng.choice([0, 0, 3]) if n > 3 else 0, pool=4096)
    elif kind == "blocks":
        c = _case(None, kind, heads, dtype, count=_log(rng, 1, 2048 if dtype == "bf16" else 1024))
    else:
        queries = rng.choice([1, 1, 1, 2, 4, 7, _log(rng, 9, 600)])
        keys = max(queries, _log(rng, 1, 131072))
        most = max(1, min(64, 262144 // keys, (1 << 25) // (keys * queries)))
        requests = _log(rng, 1, most)
        c = _case(None, kind, heads, dtype, requests=requests, queries=queries, keys=keys,
                  empty=requests > 1 and rng.random() < 0.3)
        if keys * queries > 1 << 25:
            c["keys"] = max(queries, (1 << 25) // queries)
    del c["name"]
    return c


# ---- lengths: a function of the case alone ----

def _rng(case):
    return random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))


def _slot_lengths(case):
    """(held, appended) tokens of each request; the first request's appended tokens bring the sum to `tokens`."""
    rng = _rng(case)
    n, total = case["requests"], case["tokens"]
    held = [0 if rng.random() < 0.1 else rng.randint(1, case["most"]) for _ in range(n)]
    if total <= n:
        return held, [1] * total + [0] * (n - total)
    w = [rng.random() ** 4 for _ in range(n)]
    new = [int((total - n) * x / sum(w)) + 1 for x in w]
    new[0] += total - sum(new)
    return held, new


def _attn_lengths(case):
    """(queries, keys) of each request: the first has the most of both, the others fewer; `empty`: the last has one
    query and no key."""
    rng = _rng(case)
    more = range(case["requests"] - 1)
    nq = [case["queries"]] + [rng.randint(max(1, case["queries"] // 2), case["queries"]) for _ in more]
    low = [min(case["keys"], max(q, case["keys"] // 8)) for q in nq[1:]]
    nk = [case["keys"]] + [rng.randint(x, case["keys"]) for x in low]
    if case["empty"]:
        nq[-1], nk[-1] = 1, 0
    return nq, nk


def _pairs(case):
    nq, nk = _attn_lengths(case)
    return sum(q * k - q * (q - 1) // 2 if k >= q else k * (k + 1) // 2 for q, k in zip(nq, nk))


# ---- the 4-bit format in torch ----

def _groups(x):
    return x.float().reshape(*x.shape[:-1], -1, GROUP)


def _quantise(x):
    """x [..., d] -> codes uint8 [..., d] (sign * 8 + magnitude index) and scale bytes uint8 [..., d / 32]."""
    g = _groups(x)
    amax = g.abs().amax(-1)
    bits = amax.view(torch.int32)
    byte = ((bits >> 23) - 2 + ((bits & 0x7fffff) > 0x600000).int()).clamp(1, 252)
    bad = ~torch.isfinite(g).all(-1)
    a = (g * ((254 - byte) << 23).view(torch.float32)[..., None]).abs()
    half = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    m = ((a / half).round() * half).clamp(max=6.0)
    code = torch.where(m < 2, 2 * m, torch.where(m < 4, m + 2, m / 2 + 4))
    code = torch.where(bad[..., None], torch.zeros_like(code), code + 8 * torch.signbit(g))
    byte = torch.where(bad, torch.full_like(byte, 255), byte)
    return code.to(torch.uint8).reshape(x.shape), byte.to(torch.uint8)


def _values(code, byte):
    """What codes [..., d] with scale bytes [..., d / 32] stand for, in float32."""
    table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device=code.device)
    scale = (byte.int() << 23).view(torch.float32)
    scale = torch.where(byte == 255, torch.full_like(scale, math.nan), scale)
    return (_groups(table[code.int()]) * scale[..., None]).reshape(code.shape)


def _lay(k, v):
    """A block's bytes of each head [n][heads][record] from K and V [n][16 tokens][heads][d]: K codes as [d / (d/4)]
    [token][d/8 bytes], V codes as [token / 4][16 column groups][token % 4][d/32 bytes], then K's and V's scale bytes as
    [d/32][token].  Two elements a byte, the even one low."""
    n, _, h, d = k.shape
    (kc, ks), (vc, vs) = _quantise(k), _quantise(v)
    kb = (kc[..., 0::2] | (kc[..., 1::2] << 4)).view(n, BLOCK, h, 4, d // 8).permute(0, 2, 3, 1, 4)
    vb = (vc[..., 0::2] | (vc[..., 1::2] << 4)).view(n, 4, 4, h, 16, d // 32).permute(0, 3, 1, 4, 2, 5)
    return torch.cat([x.reshape(n, h, -1) for x in (kb, vb, ks.permute(0, 2, 3, 1), vs.permute(0, 2, 3, 1))], -1)


def _unlay(rec, d):
    """K and V float32 [...][heads][16 tokens][d] of blocks [...][heads][record]."""
    lead, c = rec.shape[:-1], BLOCK * d // 2
    n = len(lead)
    kb = rec[..., :c].reshape(*lead, 4, BLOCK, d // 8).movedim(n, n + 1).reshape(*lead, BLOCK, d // 2)
    vb = rec[..., c:2 * c].reshape(*lead, 4, 16, 4, d // 32).movedim(n + 1, n + 2).reshape(*lead, BLOCK, d // 2)
    s = rec[..., 2 * c:].reshape(*lead, 2, d // GROUP, BLOCK).transpose(-1, -2)
    both = [torch.stack([b & 15, b >> 4], -1).reshape(*lead, BLOCK, d) for b in (kb, vb)]
    return _values(both[0], s[..., 0, :, :]), _values(both[1], s[..., 1, :, :])


# ---- inputs ----

def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _kv(g, n, h, d):
    """Key and value rows [n][h][d]: keys with a few channels far larger than the rest, as models have them."""
    chan = torch.exp(0.4 * _normal(g, h, d))
    chan[:, ::29] *= 5.0
    return _normal(g, n, h, d) * chan, 0.5 * _normal(g, n, h, d)


def _blocks_of(g, counts, pool):
    """Distinct blocks of the pool for each request: a table [requests][most], -1 behind a request's last block."""
    most = max(1, max(counts))
    perm = torch.randperm(pool, generator=g, device="cuda").int()
    n = torch.tensor(counts, device="cuda")
    first = torch.cumsum(n, 0) - n
    at = first[:, None] + torch.arange(most, device="cuda")[None]
    return torch.where(torch.arange(most, device="cuda")[None] < n[:, None], perm[at.clamp(max=pool - 1)],
                       torch.full_like(at, -1, dtype=torch.int32)).contiguous()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 2 + 1)
    hq, hkv, d, dt = case["q_heads"], case["kv_heads"], case["head_dim"], DT[case["dtype"]]
    kind = case["kind"]
    s = {"case": case, "kind": kind, "keep": {}}
    if kind == "slots":
        held, new = _slot_lengths(case)
        n = case["requests"]
        have = [-(-c // BLOCK) for c in held]
        need = sum(-(-(c + m) // BLOCK) for c, m in zip(held, new)) - sum(have)
        width = max(1, max(-(-(c + m) // BLOCK) for c, m in zip(held, new)))
        s["ctx"] = torch.tensor(held, dtype=torch.int32, device="cuda")
        s["new"] = torch.tensor(new, dtype=torch.int32, device="cuda")
        pool = sum(have) + need + 64
        table = _blocks_of(g, have, pool)
        s["table"] = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
        s["table"][:, :min(width, table.shape[1])] = table[:, :width]
        used = torch.zeros(pool, dtype=torch.bool, device="cuda")
        used[table[table >= 0].long()] = True
        free = torch.nonzero(~used).flatten().int()
        s["free"] = free[torch.randperm(free.numel(), generator=g, device="cuda")].contiguous()
        s["head"] = torch.full((1,), 3, dtype=torch.int32, device="cuda")
        room = case["tokens"] + case["tokens"] % 7          # the step's arrays are a little longer than its tokens
        for name, size in (("seq", n), ("cu", n + 1), ("pos", room), ("slot", room), ("state", 2)):
            s[name] = torch.zeros(size, dtype=torch.int32, device="cuda")
    elif kind == "qk":
        n = case["tokens"]
        qkv = (_normal(g, n, hq + 2 * hkv, d) * torch.exp(0.3 * _normal(g, hq + 2 * hkv, 1))).to(dt)
        s["q"], s["k"] = qkv[:, :hq], qkv[:, hq:hq + hkv]        # parts of one projection's rows
        s["gq"], s["gk"] = ((1 + 0.2 * _normal(g, d)).to(dt) if case["norm"] else None for _ in range(2))
        if case["far"]:
            pos = torch.randint(0, 131072, (n,), generator=g, device="cuda")
        else:
            pos = torch.arange(n, device="cuda") + torch.randint(0, 65536, (1,), generator=g, device="cuda")
        if case["padded"]:
            pos[n - case["padded"]:] = -1
        s["pos"] = pos.int()
        s["q_out"] = torch.zeros(n, hq, d, dtype=dt, device="cuda")
        s["k_out"] = torch.zeros(n, hkv, d, dtype=dt, device="cuda")
    elif kind == "rows":
        n, pool = case["tokens"], case["pool"]
        k, v = _kv(g, n, hkv, d)
        s["k"], s["v"] = k.to(dt), v.to(dt)
        slot = torch.randperm(pool * BLOCK, generator=g, device="cuda")[:n].int()
        if case["padded"]:
            slot[n - case["padded"]:] = -1
        s["slot"] = slot.contiguous()
        s["pool"] = torch.zeros(pool, hkv, BLOCK * (d + d // 16), dtype=torch.uint8, device="cuda")
        s["k_out"], s["v_out"] = torch.zeros_like(s["k"]), torch.zeros_like(s["v"])
    elif kind == "blocks":
        n = case["count"]
        k, v = _kv(g, (n + 8) * BLOCK, hkv, d)
        s["k"], s["v"] = (x.view(n + 8, BLOCK, hkv, d).transpose(1, 2).to(dt).contiguous() for x in (k, v))
        for name, size in (("src", n + 8), ("mid", n + 5), ("dst", n + 3)):
            s[name] = torch.randperm(size, generator=g, device="cuda")[:n].int().contiguous()
        s["pool"] = torch.zeros(n + 5, hkv, BLOCK * (d + d // 16), dtype=torch.uint8, device="cuda")
        s["k_out"], s["v_out"] = (torch.zeros(n + 3, hkv, BLOCK, d, dtype=dt, device="cuda") for _ in range(2))
    else:
        nq, nk = _attn_lengths(case)
        counts = [-(-c // BLOCK) for c in nk]
        pool = sum(counts) + 16
        k, v = _kv(g, pool * BLOCK, hkv, d)
        s["pool"] = _lay(k.view(pool, BLOCK, hkv, d), v.view(pool, BLOCK, hkv, d)).contiguous()
        s["table"] = _blocks_of(g, counts, pool)
        s["q"] = (_normal(g, sum(nq), hq, d) * 0.7).to(dt)
        s["cu"] = torch.tensor([sum(nq[:i]) for i in range(len(nq) + 1)], dtype=torch.int32, device="cuda")
        s["len"] = torch.tensor(nk, dtype=torch.int32, device="cuda")
        s["out"] = torch.zeros(sum(nq), hq, d, dtype=dt, device="cuda")
        s["lse"] = torch.zeros(sum(nq), hq, dtype=torch.float32, device="cuda")
    return s


# ---- one pass ----

def run(s):
    return (_own if own else _plain)[s["kind"]](s)


def _desc(s, sx):
    """The layer descriptor that a program keeps for its model."""
    c, keep = s["case"], s["keep"]
    if "desc" not in keep:
        keep["desc"] = sx.make_desc(c["q_heads"], c["kv_heads"], c["head_dim"], c["dtype"], 1e6, c.get("rope", "neox"))
    return keep["desc"]


def _own_slots(s):
    import paper_2606_01751_amd as sx
    sx.append_slots(s["ctx"], s["new"], s["free"], s["table"], s["seq"], s["cu"], s["pos"], s["slot"], s["state"],
                    free_head=s["head"])
    return {n: s[n] for n in ("table", "seq", "cu", "pos", "slot", "state")}


def _own_qk(s):
    import paper_2606_01751_amd as sx
    sx.qk_norm_rope(_desc(s, sx), s["q"], s["k"], s["pos"], s["q_out"], s["k_out"], gamma_q=s["gq"], gamma_k=s["gk"],
                    eps=EPS)
    return {"q": s["q_out"], "k": s["k_out"]}


def _own_rows(s):
    import paper_2606_01751_amd as sx
    desc = _desc(s, sx)
    sx.kv4_write(desc, s["k"], s["v"], s["slot"], s["pool"])
    sx.kv4_read(desc, s["pool"], s["slot"], s["k_out"], s["v_out"])
    return {"k": s["k_out"], "v": s["v_out"]}


def _own_blocks(s):
    import paper_2606_01751_amd as sx
    desc = _desc(s, sx)
    sx.kv4_pack(desc, s["k"], s["v"], s["src"], s["pool"], s["mid"])
    sx.kv4_unpack(desc, s["pool"], s["mid"], s["k_out"], s["v_out"], s["dst"])
    return {"k": s["k_out"], "v": s["v_out"]}


def _own_attn(s):
    import paper_2606_01751_amd as sx
    c, keep, desc = s["case"], s["keep"], _desc(s, sx)
    if "workspace" not in keep:     # kept by the program from step to step
        size = sx.kv4_attn_workspace(desc, c["requests"], c["queries"], c["keys"])
        keep["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    sx.kv4_attn(desc, s["q"], s["cu"], s["len"], s["table"], s["pool"], s["out"], c["queries"], c["keys"],
                keep["workspace"], lse=s["lse"])
    return {"out": s["out"], "lse": s["lse"]}


def _plain_slots(s):
    ctx, new, free, head, table = s["ctx"], s["new"], s["free"], s["head"], s["table"]
    width, room = table.shape[1], s["pos"].numel()
    cu = torch.cat([torch.zeros(1, dtype=torch.int32, device="cuda"), torch.cumsum(new, 0, dtype=torch.int32)])
    seq = ctx + new
    have = (ctx + BLOCK - 1) // BLOCK
    need = ((seq + BLOCK - 1) // BLOCK).clamp(max=width) - have
    first = torch.cumsum(need, 0, dtype=torch.int32) - need
    i = torch.arange(room, dtype=torch.int32, device="cuda")
    r = torch.searchsorted(cu[1:], i, right=True).clamp(max=new.numel() - 1)
    listed_ = i < cu[-1]
    p = ctx[r] + i - cu[r]
    bi = p // BLOCK
    fi = head + first[r] + bi - have[r]
    old = table[r, bi.clamp(0, width - 1).long()]
    none = torch.full_like(old, -1)
    fresh = torch.where((fi < free.numel()) & (bi < width), free[fi.clamp(0, free.numel() - 1).long()], none)
    block = torch.where(bi < have[r], old, fresh)
    slot = torch.where(listed_ & (block >= 0), block * BLOCK + p % BLOCK, none)
    opens = listed_ & (bi >= have[r]) & (bi < width) & (p % BLOCK == 0)
    wide = torch.cat([table.flatten(), none[:1]])
    wide[torch.where(opens, r * width + bi, table.numel())] = block
    state = torch.stack([(head[0] + need.sum()).clamp(max=free.numel()), (listed_ & (slot < 0)).sum()]).int()
    return {"table": wide[:-1].view_as(table), "seq": seq, "cu": cu, "pos": torch.where(listed_, p, none), "slot": slot,
            "state": state}


def _turn(x, gamma, pos, style, out):
    """x [n][h][d] normalised per head (gamma not None) and rotated to pos; rows at negative positions as `out` has
    them."""
    d = x.shape[-1]
    y = x.float()
    if gamma is not None:
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * gamma.float()
    theta = 1e6 ** (-torch.arange(0, d, 2, dtype=torch.float64, device="cuda") / d)
    phi = pos.double()[:, None, None] * theta
    c, t = phi.cos().float(), phi.sin().float()
    if style == "neox":
        a, b = y[..., :d // 2], y[..., d // 2:]
        y = torch.cat([a * c - b * t, b * c + a * t], -1)
    else:
        a, b = y[..., 0::2], y[..., 1::2]
        y = torch.stack([a * c - b * t, b * c + a * t], -1).flatten(-2)
    return torch.where((pos >= 0)[:, None, None], y.to(x.dtype), out)


def _plain_qk(s):
    return {n: _turn(s[n], s["g" + n], s["pos"], s["case"]["rope"], s[n + "_out"]) for n in ("q", "k")}


def _plain_rows(s):
    keep = (s["slot"] >= 0)[:, None, None]
    return {n: torch.where(keep, _values(*_quantise(s[n])).to(s[n].dtype), s[n + "_out"]) for n in ("k", "v")}


def _plain_blocks(s):
    src, dst = s["src"].long(), s["dst"].long()
    return {n: s[n + "_out"].index_copy(0, dst, _values(*_quantise(s[n][src])).to(s[n].dtype)) for n in ("k", "v")}


def _plain_attn(s):
    c = s["case"]
    hq, hkv, d = c["q_heads"], c["kv_heads"], c["head_dim"]
    grp, cu, lens, table = hq // hkv, s["cu"].long(), s["len"].long(), s["table"]
    nr, most, keys = lens.numel(), c["queries"], table.shape[1] * BLOCK
    k, v = _unlay(s["pool"][table.clamp(min=0).long()], d)                    # [r][pages][hkv][16][d]
    k, v = (x.transpose(1, 2).reshape(nr * hkv, keys, d) for x in (k, v))
    i = torch.arange(most, device="cuda")
    at = cu[:-1, None] + i                                                    # rows of q, padded to `most` a request
    live = i < (cu[1:] - cu[:-1])[:, None]
    q = s["q"][at.clamp(max=s["q"].shape[0] - 1)].float()                     # [r][most][hq][d]
    q = q.view(nr, most, hkv, grp, d).permute(0, 2, 1, 3, 4).reshape(nr * hkv, most * grp, d)
    x = torch.bmm(q, k.transpose(1, 2).contiguous()).view(nr, hkv, most, grp, keys)
    x *= 1.0 / math.sqrt(d)
    last = (lens - (cu[1:] - cu[:-1]))[:, None] + i                           # the row's own position
    hidden = torch.arange(keys, device="cuda") > last[..., None]
    x.masked_fill_(hidden[:, None, :, None, :], -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    x -= top
    x.exp_()
    den = x.sum(-1, keepdim=True)
    o = torch.bmm(x.view(nr * hkv, most * grp, keys), v).view(nr, hkv, most, grp, d) / torch.where(den == 0, 1.0, den)
    lse = (den.log() + top)[..., 0].permute(0, 2, 1, 3).reshape(nr, most, hq)
    o = o.permute(0, 2, 1, 3, 4).reshape(nr, most, hq, d).to(s["q"].dtype)
    return {"out": s["out"].index_copy(0, at[live], o[live]), "lse": s["lse"].index_copy(0, at[live], lse[live])}


_own = {"slots": _own_slots, "qk": _own_qk, "rows": _own_rows, "blocks": _own_blocks, "attn": _own_attn}
_plain = {"slots": _plain_slots, "qk": _plain_qk, "rows": _plain_rows, "blocks": _plain_blocks, "attn": _plain_attn}


# ---- what a pass cannot do without ----

def work(case):
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    esz = 4 if case["dtype"] == "f32" else 2
    kind = case["kind"]
    held = 2 * hkv * (d // 2 + d // GROUP)          # a token's K and V in 4 bits
    if kind == "slots":
        h, new = _slot_lengths(case)
        need = sum(-(-(c + m) // BLOCK) + c // -BLOCK for c, m in zip(h, new))
        return {"bytes": 16 * case["requests"] + 8 * case["tokens"] + 8 * need, "flops": 0}
    if kind == "qk":
        n = case["tokens"] - case["padded"]
        return {"bytes": 2 * n * (hq + hkv) * d * esz + 4 * n, "flops": n * (hq + hkv) * d * (7 if case["norm"] else 3)}
    if kind in ("rows", "blocks"):
        n = case["tokens"] - case["padded"] if kind == "rows" else case["count"] * BLOCK
        return {"bytes": n * (4 * hkv * d * esz + held + 4), "flops": 0}
    nq, nk = _attn_lengths(case)
    rows, pages = sum(nq) * hq, sum(-(-c // BLOCK) for c in nk)
    return {"bytes": sum(nk) * held + 2 * rows * d * esz + 4 * rows + 4 * pages,
            "flops": 4 * d * hq * _pairs(case)}


# ---- the definitions in 64 bits ----

_MAGNITUDE = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_held(x):
    """What the 4-bit cache holds for rows x [..., d]: the nearest of every magnitude tried, the even code on a tie."""
    g = x.double().reshape(-1, GROUP)
    amax = g.abs().amax(-1)
    e = torch.ceil(torch.log2(amax / 7)).clamp(-126, 125)
    for step in (1.0, -1.0):        # (the logarithm may be off by one unit next to a border)
        up = torch.ldexp(torch.full_like(e, 7.0), e.int()) < amax if step > 0 else \
            torch.ldexp(torch.full_like(e, 7.0), (e - 1).int()) >= amax
        e = torch.where(up, (e + step).clamp(-126, 125), e)
    s = torch.ldexp(torch.ones_like(e), e.int())[:, None]
    a = g.abs() / s
    best, off = torch.zeros_like(a), a.clone()
    for i, m in enumerate(_MAGNITUDE[1:], 1):
        o = (a - m).abs()
        take = (o < off) | ((o == off) & (i % 2 == 0))
        best, off = torch.where(take, torch.full_like(a, m), best), torch.where(take, o, off)
    return (torch.copysign(best, g) * s).reshape(x.shape)


def _exact_pool(rec, d):
    """K and V in float64 [blocks][heads][16][d]: element by element from the byte that holds it."""
    t = torch.arange(BLOCK, device=rec.device)[:, None]
    c = torch.arange(d, device=rec.device)[None]
    size = BLOCK * d // 2
    k_at = (c // (d // 4)) * (BLOCK * d // 8) + t * (d // 8) + c % (d // 4) // 2
    col = d // 16
    v_at = size + ((t // 4 * 16 + c // col) * 4 + t % 4) * (d // 32) + c % col // 2
    s_at = 2 * size + c // GROUP * BLOCK + t
    m = torch.tensor(_MAGNITUDE, dtype=torch.float64, device=rec.device)
    out = []
    for at, sc in ((k_at, s_at), (v_at, s_at + BLOCK * d // GROUP)):
        code = rec[..., at].int() >> (4 * (c % 2)) & 15
        val = m[(code & 7).long()] * torch.where(code >= 8, -1.0, 1.0).double()
        out.append(torch.ldexp(val, rec[..., sc].int() - 127))
    return out


def exact(case, seed):
    s = prepare(case, seed)
    hq, hkv, d = case["q_heads"], case["kv_heads"], case["head_dim"]
    kind = case["kind"]
    if kind == "slots":
        return None
    if kind == "qk":
        pos = s["pos"].double()
        pair = torch.arange(d // 2, dtype=torch.float64, device="cuda")
        ang = pos[:, None] * torch.exp(-math.log(1e6) * 2 * pair / d)
        z = torch.polar(torch.ones_like(ang), ang)[:, None]
        out = {}
        for name, x, gamma in (("q", s["q"], s["gq"]), ("k", s["k"], s["gk"])):
            y = x.double()
            if gamma is not None:
                y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / d + EPS) * gamma.double()
            pair = (y[..., :d // 2], y[..., d // 2:]) if case["rope"] == "neox" else (y[..., ::2], y[..., 1::2])
            w = torch.complex(*(p.contiguous() for p in pair)) * z
            y = torch.cat([w.real, w.imag], -1) if case["rope"] == "neox" else torch.view_as_real(w).flatten(-2)
            out[name] = y * (pos >= 0)[:, None, None]
        return out
    if kind == "rows":
        live = (s["slot"] >= 0)[:, None, None]
        return {n: _exact_held(s[n]) * live for n in ("k", "v")}
    if kind == "blocks":
        out = {}
        for n in ("k", "v"):
            y = torch.zeros(s[n + "_out"].shape, dtype=torch.float64, device="cuda")
            y[s["dst"].long()] = _exact_held(s[n][s["src"].long()])
            out[n] = y
        return out
    nq, nk = _attn_lengths(case)
    grp, scale = hq // hkv, d ** -0.5
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["lse"].shape, -math.inf, dtype=torch.float64, device="cuda")
    first = 0
    for r, (n, m) in enumerate(zip(nq, nk)):
        pages = s["table"][r, :-(-m // BLOCK)].long()
        for h in range(hkv if m else 0):
            k, v = (x.reshape(-1, d)[:m] for x in _exact_pool(s["pool"][pages, h], d))
            q = s["q"][first:first + n, h * grp:(h + 1) * grp].double().reshape(n * grp, d)
            x = (q @ k.t()) * scale
            row = torch.arange(n, device="cuda").repeat_interleave(grp) + (m - n)
            x.masked_fill_(torch.arange(m, device="cuda")[None] > row[:, None], -math.inf)
            z = torch.logsumexp(x, -1, keepdim=True)
            x.sub_(torch.where(z == -math.inf, torch.zeros_like(z), z)).exp_()
            out[first:first + n, h * grp:(h + 1) * grp] = (x @ v).view(n, grp, d)
            lse[first:first + n, h * grp:(h + 1) * grp] = z.view(n, grp)
        first += n
    return {"out": out, "lse": lse}
