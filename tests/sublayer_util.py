"""Plain implementations in 64 bits of the operators of a feed-forward sublayer, and how far a call in fp32 may be from them.

U is half a unit of fp32.  Errors are first order: every rounding that a call makes, with the sizes of what it rounds, and twice that where a bound is a sum of many
such terms is not needed: none of them is at its largest everywhere."""
import math

U = 2.0 ** -24
HALF = {"float32": 2.0 ** -24, "bfloat16": 2.0 ** -8}      # of a result's size: its own rounding
ACTS = ("none", "relu", "gelu", "silu")
# Beside the relative errors: numbers below 2^-126 may count as 0.
TINY = 2.0 ** -120


def number(cdl, act):
    return {"none": cdl.ACT_NONE, "relu": cdl.ACT_RELU, "gelu": cdl.ACT_GELU, "silu": cdl.ACT_SILU}[act]


def up(n):
    return (n + 127) // 128 * 128


def empty8(torch, rows, cols):
    """(q, scale) of rows in eight bits, filled with what nobody writes"""
    return (torch.full((rows, up(cols)), 77, dtype=torch.uint8, device="cuda"), torch.full((up(cols) // 128, up(rows)), 77, dtype=torch.uint8, device="cuda"))


def quantize(torch, cdl, x, fmt="e4m3", tiles=False):
    rows, cols = x.shape
    q, scale = empty8(torch, rows, cols)
    cdl.cdl_block8_quantize(x, rows, cols, q, scale, tiles=tiles, format=cdl.E4M3 if fmt == "e4m3" else cdl.E5M2)
    return q, scale


def values(torch, q, scale, fmt="e4m3", cols=None):
    """what they stand for, in 64 bits"""
    s = scale[:, : q.shape[0]].t().repeat_interleave(128, dim=1).int() - 127
    v = torch.ldexp(q.view(torch.float8_e4m3fn if fmt == "e4m3" else torch.float8_e5m2).double(), s)
    return v if cols is None else v[:, :cols]


def outside(got, want, bound):
    """entries that are further off than they may be (NaN: never inside, but where NaN is wanted)"""
    bad = ~((got.double() - want).abs() <= bound)
    return int((bad & ~((got != got) & (want != want)) & ~(got.double() == want)).sum())


# ---- activations ----------------------------------------------------------------------------------------------------

def act(torch, name, z):
    """value, derivative, and their errors, for z in 64 bits that the call has in fp32"""
    a = z.abs()
    if name == "none":
        return z, torch.ones_like(z), torch.zeros_like(z), torch.zeros_like(z)
    if name == "relu":
        return z.clamp(min=0), (z > 0).double(), torch.zeros_like(z), torch.zeros_like(z)
    if name == "gelu":
        # The tail Phi(-|z|) is a polynomial (2.2e-7 of itself off; nine products and sums, whose coefficients alternate: 7 U more), in a reciprocal (2 U) and times an
        # exponential (2 U, and z^2 U for its argument's two roundings): 1.4e-6 + z^2 U of itself.  Phi above zero is one subtraction more.
        tail = 0.5 * torch.erfc(a / math.sqrt(2.0))
        bell = torch.exp(-z * z / 2)
        off = (1.4e-6 + z * z * U) * tail + torch.where(z < 0, 0.0, U)
        phi = torch.where(z < 0, tail, 1 - tail)
        near = (z * z + 4) * U * a * bell / math.sqrt(2 * math.pi)      # of z times the density
        slope = phi + z * bell / math.sqrt(2 * math.pi)
        return z * phi, slope, a * off + U * (z * phi).abs() + TINY, off + near + U * slope.abs() + TINY
    # exp(-z): its argument's rounding, |z| U, and its own, 2 U; the sum and the reciprocal 3 U
    s = torch.sigmoid(z)
    off = ((1 - s) * (a + 3) + 3) * U * s
    slope = s * (1 + z * torch.sigmoid(-z))
    return z * s, slope, a * off + U * (z * s).abs() + TINY, off * (1 + a * torch.sigmoid(-z)) + a * s * (off + U) + 3 * U * s * (1 + a * torch.sigmoid(-z)) + TINY


def act_back(torch, name, g, z, kind):
    """[(gradient, error)], (y, error) of a layer's activation: z is [z] or [gate, up]"""
    h = HALF[kind]
    value, slope, off_v, off_s = act(torch, name, z[0])
    if len(z) == 1:
        d = [(g * slope, g.abs() * off_s)]
        y = (value, off_v)
    else:
        d = [(g * z[1] * slope, (g * z[1]).abs() * off_s), (g * value, g.abs() * off_v)]
        y = (value * z[1], off_v * z[1].abs())
    return [(v, e + 3 * U * v.abs() + TINY) for v, e in d], (y[0], y[1] + (h + U) * y[0].abs() + TINY)


def column_sum(torch, d, off):
    """sum over the rows, and its error: a thread has at most 1 / 16 of the rows and 16 more in a row (never more than 256 + 1 / 2048 of them), then up to 8 + 16 + 64 sums"""
    rows = d.shape[0]
    chain = min(rows, 300 + rows // 256) + 96
    return d.sum(dim=0), off.sum(dim=0) + chain * U * d.abs().sum(dim=0)


# ---- layer norm -----------------------------------------------------------------------------------------------------

def norm(torch, x, weight, bias, eps, kind):
    """(y, error), (mean, error), (rstd, error); a lane adds up at most 32 entries, a row's lanes 4 + 2 + 16 sums: 64 U with what stands beside them"""
    cols = x.shape[1]
    mean = x.mean(dim=1, keepdim=True)
    size = x.abs().mean(dim=1, keepdim=True)
    off_m = 64 * U * size
    c = x - mean
    var = (c * c).mean(dim=1, keepdim=True)
    rstd = 1 / torch.sqrt(var + eps)
    # the squares about a mean that is off: each by 2 |c| (off + U |c|), the sum of c being zero up to its rounding; half of it and two roundings in rstd
    off_r = rstd * (0.5 * (64 * U + 2 * U + (off_m ** 2 + 2 * off_m * 64 * U * size) / (var + eps).clamp(min=1e-300)) + 3 * U)
    w = torch.ones(cols, dtype=torch.float64, device=x.device) if weight is None else weight.double()
    b = torch.zeros(cols, dtype=torch.float64, device=x.device) if bias is None else bias.double()
    y = c * rstd * w + b
    off_y = w.abs() * ((off_m + U * c.abs()) * rstd + c.abs() * off_r + 2 * U * c.abs() * rstd) + U * y.abs() + HALF[kind] * y.abs() + TINY
    return (y, off_y), (mean[:, 0], off_m[:, 0] + U * mean[:, 0].abs()), (rstd[:, 0], off_r[:, 0])


def norm_back(torch, g, x, weight, mean, rstd, add, kind):
    """(d_x, error), (d_weight, error), (d_bias, error) for the mean and rstd of the call"""
    rows, cols = g.shape
    m, r = mean.double()[:, None], rstd.double()[:, None]
    n = (x - m) * r
    h = g if weight is None else g * weight.double()
    one, two = h.mean(dim=1, keepdim=True), (h * n).mean(dim=1, keepdim=True)
    d = r * (h - one - n * two)
    # n two roundings, h one, the means 66 with their products; then a product, two differences, the factor
    inner = 6 * U * (h.abs() + one.abs() + (n * two).abs()) + 68 * U * h.abs().mean(dim=1, keepdim=True) + 72 * U * n.abs() * (h * n).abs().mean(dim=1, keepdim=True)
    if add is not None:
        d = d + add
    off = r * inner + (2 * U + HALF[kind]) * d.abs() + TINY
    gn = g * n
    return (d, off), column_sum(torch, gn, 3 * U * gn.abs()), column_sum(torch, g, torch.zeros_like(g))


# ---- products -------------------------------------------------------------------------------------------------------

def product(torch, va, vb, bias, kind):
    """(z, error) before any rounding of z: K exact products summed in fp32, in bf16 what the instructions leave out of them (at most 16 * 2^-14 of the sum of their sizes)"""
    ref, size = va @ vb.t(), va.abs() @ vb.abs().t()
    off = max(va.shape[1], 2) * U * size
    if kind == "bfloat16":
        off = off + 2.0 ** -10 * size
    if bias is not None:
        ref = ref + bias.double()
        off = off + U * (ref.abs() + off)
    return ref, off


def forward(torch, name, z, add, kind):
    """(y, error) from [(z, error)]: steepest at 1.13 (gelu, silu)"""
    h = HALF[kind]
    value, _, off, _ = act(torch, name, z[0][0])
    off = off + 1.13 * z[0][1]
    y = value
    if len(z) == 2:
        y, off = value * z[1][0], off * z[1][0].abs() + (value.abs() + off) * z[1][1]
    if add is not None:
        y = y + add
    return y, off + (h + 2 * U) * (y.abs() + off) + TINY
