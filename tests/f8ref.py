"""Float64 references of the 8-bit layer body, on the CPU, from their definitions (include/sx_f8.h).

e4m3 numbers and the groups' powers of two are built from their definitions, without torch's 8-bit types.  What float32
arithmetic may add to a result is derived where it is used."""
import math

import torch

GROUP = 128
E = 2.0 ** -24      # half a step of float32, relative

# e4m3 by code: sign, 4 bits of exponent (bias 7; 0: subnormal), 3 of mantissa; 0x7f is NaN
MAGNITUDES = torch.tensor([(m / 8 if not x else 1 + m / 8) * 2.0 ** (max(x, 1) - 7) for x in range(16) for m in range(8)][:127],
                          dtype=torch.float64)


def ld(k):
    return (k // GROUP + 3) // 4 * 4


def values(codes):
    """What e4m3 codes (uint8) are, in float64."""
    t = torch.cat([MAGNITUDES, torch.tensor([math.nan], dtype=torch.float64)])
    c = codes.long()
    return t[c & 127] * torch.where(c >= 128, -1.0, 1.0).double()


def powers(byte):
    """2^(byte - 127), NaN for 255."""
    p = torch.ldexp(torch.ones(byte.shape, dtype=torch.float64), byte.int() - 127)
    return torch.where(byte == 255, math.nan, p)


def scale_byte(amax):
    """Byte of the smallest 2^e with amax <= 448 * 2^e, -126 <= e <= 120; 255 where amax is not finite."""
    fine = torch.isfinite(amax)
    e = torch.ceil(torch.log2(torch.where(fine, amax, 1.0) / 448)).clamp(-126, 120)
    for _ in range(2):   # (the logarithm may be off by one next to a border)
        e = torch.where(448 * 2.0 ** e < amax, e + 1, e).clamp(-126, 120)
        e = torch.where(448 * 2.0 ** (e - 1) >= amax, e - 1, e).clamp(-126, 120)
    return torch.where(fine, e + 127, 255.0).to(torch.uint8)


def codes_of(z):
    """Nearest e4m3 codes of values z with |z| <= 448, the even code on a tie."""
    a = z.abs()
    hi = torch.searchsorted(MAGNITUDES, a).clamp(max=126)      # first magnitude >= a
    lo = (hi - 1).clamp(min=0)
    dh, dl = MAGNITUDES[hi] - a, a - MAGNITUDES[lo]
    up = (dh < dl) | ((dh == dl) & (hi % 2 == 0))
    return (torch.where(up, hi, lo) + 128 * torch.signbit(z)).to(torch.uint8)


def quantise(y):
    """Rows y [n][k] in float64 -> (codes, scale bytes [n][ld])."""
    n, k = y.shape
    g = y.view(n, k // GROUP, GROUP)
    byte = scale_byte(torch.where(torch.isfinite(g).all(-1), g.abs().amax(-1), math.inf))
    s = torch.zeros(n, ld(k), dtype=torch.uint8)
    s[:, :k // GROUP] = byte
    z = torch.where((byte == 255)[..., None], 0.0, g * 2.0 ** (127.0 - byte.double())[..., None])
    c = codes_of(z)
    return torch.where((byte == 255)[..., None], torch.zeros_like(c), c).view(n, k), s


def quantise_weight(w):
    """A weight [n][k] in float64 -> (codes, scale bytes [n / 128][ld])."""
    n, k = w.shape
    g = w.view(n // GROUP, GROUP, k // GROUP, GROUP)
    byte = scale_byte(torch.where(torch.isfinite(g).all(-1).all(1), g.abs().amax((1, 3)), math.inf))
    s = torch.zeros(n // GROUP, ld(k), dtype=torch.uint8)
    s[:, :k // GROUP] = byte
    bad = (byte == 255)[:, None, :, None]
    c = codes_of(torch.where(bad, 0.0, g * 2.0 ** (127.0 - byte.double())[:, None, :, None]))
    return torch.where(bad, torch.zeros_like(c), c).view(n, k), s


def rows_of(codes, scale):
    n, k = codes.shape
    return (values(codes).view(n, k // GROUP, GROUP) * powers(scale[:, :k // GROUP])[..., None]).view(n, k)


def weight_of(codes, scale):
    n, k = codes.shape
    g = values(codes).view(n // GROUP, GROUP, k // GROUP, GROUP)
    return (g * powers(scale[:, :k // GROUP])[:, None, :, None]).view(n, k)


def held(codes, scale, y, off):
    """Whether codes and scale bytes hold rows y (float64), of which the library may have computed values up to `off`
    (relative) away: each group's byte is that of some amax so near, each element the nearest code of some value so near.
    The name of the first thing that is not, or None."""
    n, k = codes.shape
    g = y.view(n, k // GROUP, GROUP)
    byte = scale[:, :k // GROUP]
    if scale[:, k // GROUP:].any():
        return "padding bytes"
    amax = torch.where(torch.isfinite(g).all(-1), g.abs().amax(-1), math.inf)
    if ((byte < scale_byte(amax * (1 - off))) | (byte > scale_byte(amax * (1 + off)))).any():
        return "scale bytes"
    bad = byte == 255
    if codes.view(n, k // GROUP, GROUP)[bad].any():
        return "codes of a group that stands for NaN"
    z = torch.where(bad[..., None], 0.0, g * 2.0 ** (127.0 - byte.double())[..., None])
    a = z.abs().clamp(max=448)
    # half of the step around each element: 2^-10 below 2^-6, else 2^-4 of its binade
    half = torch.where(a < 2.0 ** -6, 2.0 ** -10, 2.0 ** (torch.floor(torch.log2(a.clamp(min=2.0 ** -6))) - 4))
    v = values(codes).view(n, k // GROUP, GROUP)
    if not ((v - z).abs() <= half * (1 + 1e-12) + z.abs() * off).all():
        return "codes"
    if (torch.signbit(v) != torch.signbit(z)).logical_and(z != 0).any():
        return "signs"
    return None


def norm(s, gamma, eps):
    y = s / torch.sqrt((s * s).mean(-1, keepdim=True) + eps)
    return y * gamma


def silu_mul(gate, up):
    return gate * torch.sigmoid(gate) * up


def product(xc, xs, wc, ws):
    """(x w^T, sum of the magnitudes of its terms)."""
    x, w = rows_of(xc, xs), weight_of(wc, ws)
    return x @ w.t(), x.abs() @ w.abs().t()


def product_bound(k, mag):
    """What the matrix cores may be off by over k products whose magnitudes add up to mag.  The 8-bit instruction aligns the
    products of eight consecutive elements to the largest one's exponent and cuts each off 13 bits below it: seven of them
    lose less than 2^-13 of the largest, that is 7 * 2^-13 of the eight's magnitudes.  (Measured: beside a product of 1 those
    of 2^-13 in its eight are added, those of 2^-14 are not; in other eights all are.)  The sums of the eights and of the
    steps are float32 ones: a whole step for each of up to k / 8 + k / 128 additions."""
    return (7 * 2.0 ** -13 + (k / 8 + k / 128 + 8) * 2 * E) * mag


def route(logits, top, renormalise):
    """ids, weights (float64), rows [n][experts] of logits: a Python loop a row."""
    ids, ws = [], []
    for row in logits.double().tolist():
        v = [-math.inf if math.isnan(x) else x for x in row]
        best = sorted(range(len(v)), key=lambda e: (-v[e], e))[:top]
        m = v[best[0]]
        p = [0.0 if m == -math.inf else 1.0 if x == m else math.exp(x - m) for x in v]
        tot = sum(p[e] for e in best) if renormalise else sum(p)
        ids.append(best)
        ws.append([p[e] / tot if tot else 0.0 for e in best])
    return torch.tensor(ids, dtype=torch.int32).view(-1, top), torch.tensor(ws, dtype=torch.float64).view(-1, top)


def group(ids, slots, experts):
    """(offsets, order) of ids [n][top] of rows at these slots, in ascending places."""
    top = ids.shape[1]
    at = [[] for _ in range(experts)]
    for row, s in zip(ids.tolist(), slots):
        for j, e in enumerate(row):
            at[e].append(s * top + j)
    off = [0]
    for a in at:
        off.append(off[-1] + len(a))
    return torch.tensor(off, dtype=torch.int32), torch.tensor([p for a in at for p in a], dtype=torch.int32)
