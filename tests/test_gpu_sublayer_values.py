"""What the operators of a feed-forward sublayer promise of their values beyond bounds of their roundings: the same bits whatever else is asked for, rows without spread and far from zero,
what is not finite, products with nothing left out."""
import pytest

import gpu_util as gu
import sublayer_util as su

pytestmark = pytest.mark.gpu
KINDS = ("float32", "bfloat16")


@pytest.fixture(scope="module")
def env():
    import paper_2501_09849_amd as cdl
    return gu.torch_mod(), cdl


def finished(torch, cdl, a, b, size, kind, name, bias, kept):
    """y of a product (one matrix b) or a gated one (two), and its z where `kept` asks for them"""
    M, N, K = size
    new = lambda: torch.full((M, N), float("nan"), dtype=getattr(torch, kind), device="cuda")      # noqa: E731
    y, z = new(), [new() if k else None for k in kept]
    query = cdl.block8_gemm_act_workspace_bytes if len(b) == 1 else cdl.block8_gemm_gated_workspace_bytes
    ws = torch.full((max(256, query(M, N, K)),), 0xff, dtype=torch.uint8, device="cuda")
    more = dict(act=su.number(cdl, name), ws=ws)
    if len(b) == 1:
        cdl.cdl_block8_gemm_act(*a, *b[0], M, N, K, y, z=z[0], bias=bias[0], **more)
    else:
        cdl.cdl_block8_gemm_gated(*a, *b[0], *b[1], M, N, K, y, z_gate=z[0], z_up=z[1], bias_gate=bias[0], bias_up=bias[1], **more)
    torch.cuda.synchronize()
    return y, z


# few rows, few tiles, many; at each of them storing z as well changes which tiles are estimated to be the quickest, or would change whether tiles are
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("sides", [1, 2])
@pytest.mark.parametrize("size", [(1, 8192, 4096), (40, 8192, 128), (64, 4096, 4096), (96, 4096, 512), (200, 8192, 4096), (300, 1024, 2048), (300, 8192, 512), (1000, 8192, 512), (2048, 2048, 768),
                                  (4096, 4096, 768), (9000, 512, 768)])
def test_a_forward_pass_formed_again_with_z(env, size, sides, kind):
    torch, cdl = env
    M, N, K = size
    gen = torch.Generator(device="cuda").manual_seed(M + N + K)
    a = su.quantize(torch, cdl, torch.randn((M, K), device="cuda", generator=gen))
    b = [su.quantize(torch, cdl, torch.randn((N, K), device="cuda", generator=gen) * K ** -0.5, tiles=True) for _ in range(sides)]
    bias = [torch.randn(N, device="cuda", generator=gen) for _ in range(sides)]
    for name in ("none", "gelu", "silu"):
        want, _ = finished(torch, cdl, a, b, size, kind, name, bias, [False] * sides)
        assert torch.isfinite(want).all()
        all_z = None
        for kept in ([True],) if sides == 1 else ([True, True], [True, False], [False, True]):
            got, z = finished(torch, cdl, a, b, size, kind, name, bias, kept)
            assert torch.equal(got, want), (name, kept)
            all_z = all_z or z
            assert all(torch.equal(p, q) for p, q, k in zip(z, all_z, kept) if k)


# ---- layer norm: rows whose mean is large beside their spread ----------------------------------------------------------

WIDTHS = [1, 7, 100, 128, 300, 513, 768, 1000, 1021, 1025, 2047, 3001, 4096, 8200, 16376, 16384]      # every number of lanes and chunks, whole and ragged


def norm_fwd(torch, cdl, x, w=None, b=None, eps=1e-5, keep=False):
    rows, cols = x.shape
    y, mean, rstd = torch.full_like(x, float("nan")), torch.full((rows,), float("nan"), device="cuda"), torch.full((rows,), float("nan"), device="cuda")
    q, scale = su.empty8(torch, rows, cols) if keep else (None, None)
    cdl.cdl_layer_norm_fwd(x, rows, cols, y, mean, rstd, weight=w, bias=b, eps=eps, q=q, scale=scale)
    torch.cuda.synchronize()
    return y, mean, rstd


def norm_bounds(torch, x, w, b, eps, kind):
    """[(result, error)] of y, mean and rstd.  A sum of a row is 32 entries in a lane and 4 + 2 + 8 joins, less than 64 roundings.  The mean first formed is off by its own rounding and by that
    of the sum of differences from the first entry; what is subtracted in the end is the mean of differences from it, so that is all that is left of either."""
    U = su.U
    mean = x.mean(dim=1, keepdim=True)
    c = x - mean
    var, size = (c * c).mean(dim=1, keepdim=True), c.abs().mean(dim=1, keepdim=True)
    first = U * mean.abs() + 68 * U * (x - x[:, :1]).abs().mean(dim=1, keepdim=True)
    off_c = 2 * U * c.abs() + U * first + 66 * U * (size + first)
    rstd = 1 / torch.sqrt(var + eps)
    off_var = 68 * U * (var + 2 * first * first) + 2 * first * 66 * U * (size + first)
    off_r = rstd * (0.5 * off_var / (var + eps) + 4 * U)
    y = c * rstd * w + b
    off_y = w.abs() * (off_c * rstd + c.abs() * off_r + 2 * U * c.abs() * rstd) + U * y.abs() + su.HALF[kind] * y.abs() + su.TINY
    return (y, off_y), (mean[:, 0], (U * mean.abs() + 66 * U * (size + first))[:, 0]), (rstd[:, 0], off_r[:, 0])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("cols", WIDTHS)
def test_rows_of_one_value_are_the_bias(env, cols, kind):
    """No difference from the first entry has a rounding: the mean is the value, y the bias; with eps 0 there is no norm."""
    torch, cdl = env
    gen = torch.Generator(device="cuda").manual_seed(cols)
    values = [1000.1, 0.1, 100.0, 1000.0, 3.0, -30000.3, 0.0, 1e-20]
    x = torch.tensor(values, device="cuda")[:, None].expand(-1, cols).contiguous().to(getattr(torch, kind))
    w, b = torch.randn(cols, device="cuda", generator=gen), torch.randn(cols, device="cuda", generator=gen)
    for keep in (False, True):
        y, mean, rstd = norm_fwd(torch, cdl, x, w, b, keep=keep)
        assert torch.equal(mean, x[:, 0].float()) and torch.equal(y, b.to(x.dtype).expand_as(y))
        assert float((rstd.double() * 1e-5 ** 0.5 - 1).abs().max()) <= 4 * su.U
        y, mean, rstd = norm_fwd(torch, cdl, x, w, b, eps=0.0, keep=keep)
        assert torch.equal(mean, x[:, 0].float()) and torch.isnan(y).all() and torch.isinf(rstd).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("cols", WIDTHS[1:])
def test_the_mean_adds_nothing_to_the_rows(env, cols, kind):
    """Rows whose mean is up to 10^5 times their spread, rows with a spread of a few units of their last place, rows whose first entry is far from all others."""
    torch, cdl = env
    gen = torch.Generator(device="cuda").manual_seed(cols)
    r = lambda *s: torch.randn(s, device="cuda", generator=gen)      # noqa: E731
    x = r(64, cols)
    x[:16] += 1000.1
    x[16:24] = x[16:24] * 1e-2 + 1000.1
    x[24:32] = 1000.1 + 6.104e-5 * torch.randint(0, 3, (8, cols), device="cuda", generator=gen)
    x[32:40, 0] = 1e4
    x[40:48] = x[40:48] * 1e-3 - 0.1
    x[48:52, 0] += 1e6
    x = x.to(getattr(torch, kind))
    w, b = 1 + 0.2 * r(cols), 0.2 * r(cols)
    for eps in (1e-5, 1e-12):
        for got, want in zip(norm_fwd(torch, cdl, x, w, b, eps), norm_bounds(torch, x.double(), w.double(), b.double(), eps, kind)):
            assert su.outside(got, *want) == 0, eps


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,cols", [(1, 16384), (4, 16384), (3, 8001), (16, 1024), (15, 769), (64, 128), (61, 100), (700, 300)])
def test_a_gradient_alone_is_that_of_a_call_with_sums(env, rows, cols, kind):
    """(few rows of a call with sums are one block's, of one without they are not)"""
    torch, cdl = env
    gen = torch.Generator(device="cuda").manual_seed(rows + cols)
    x, g, add = (torch.randn((rows, cols), device="cuda", generator=gen).to(getattr(torch, kind)) for _ in range(3))
    w = torch.randn(cols, device="cuda", generator=gen)
    _, mean, rstd = norm_fwd(torch, cdl, x)
    got = [torch.full_like(x, float("nan")) for _ in range(2)]
    sums = [torch.full((cols,), float("nan"), device="cuda") for _ in range(2)]
    ws = torch.empty(max(256, cdl.layer_norm_bwd_workspace_bytes(rows, cols)), dtype=torch.uint8, device="cuda")
    for given in (dict(x=x), dict(zip(("q", "scale"), su.quantize(torch, cdl, x)))):
        cdl.cdl_layer_norm_bwd(g, rows, cols, mean, rstd, d_x=got[0], weight=w, add=add, **given)
        cdl.cdl_layer_norm_bwd(g, rows, cols, mean, rstd, d_x=got[1], d_weight=sums[0], d_bias=sums[1], weight=w, add=add, ws=ws, **given)
        at = su.values(torch, given["q"], given["scale"], cols=cols) if "q" in given else x.double()
        wants = su.norm_back(torch, g.double(), at, w, mean, rstd, add.double(), kind)
        assert torch.equal(*got) and [su.outside(v, *want) for v, want in zip([got[0]] + sums, wants)] == [0, 0, 0]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("cols", [40, 1021, 9000])
def test_rows_whose_squares_overflow(env, cols, kind):
    """Squares beyond the largest number of fp32: rstd 0; differences beyond it: not finite; no other row knows of either."""
    torch, cdl = env
    gen = torch.Generator(device="cuda").manual_seed(cols)
    x = torch.randn((9, cols), device="cuda", generator=gen).to(getattr(torch, kind))
    w, b = torch.randn(cols, device="cuda", generator=gen), torch.randn(cols, device="cuda", generator=gen)
    clean = norm_fwd(torch, cdl, x, w, b)
    x[2] *= 1e25
    x[5, ::2], x[5, 1::2] = 3e38, -3e38
    y, mean, rstd = norm_fwd(torch, cdl, x, w, b)
    assert float(rstd[2]) == 0 and torch.isfinite(mean[2]) and torch.equal(y[2], b.to(y.dtype)) and not torch.isfinite(y[5]).any()
    rest = [0, 1, 3, 4, 6, 7, 8]
    assert all(torch.equal(p[rest], q[rest]) for p, q in zip((y, mean, rstd), clean))


# ---- what is not finite ----------------------------------------------------------------------------------------------

INF, NAN = float("inf"), float("nan")
# value and derivative at minus infinity, infinity and no number
VALUES = {"none": [-INF, INF, NAN], "relu": [0.0, INF, NAN], "gelu": [NAN, INF, NAN], "silu": [NAN, INF, NAN]}
SLOPES = {"none": [1.0, 1.0, 1.0], "relu": [0.0, 1.0, NAN], "gelu": [NAN, NAN, NAN], "silu": [NAN, NAN, NAN]}


def same(torch, got, wants):
    """each of `got` against one number"""
    return all((torch.isnan(v) if want != want else v.double() == want).all() for v, want in zip(got, wants))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("name", su.ACTS)
def test_gradients_where_z_is_not_finite(env, name, kind):
    """z as it is: its own entry; as kept in eight bits: no number for the 128 entries of its block"""
    torch, cdl = env
    t, at = getattr(torch, kind), [5, 130, 299]
    for rows, cols in ((3, 300), (50, 301), (500, 300)):
        gen = torch.Generator(device="cuda").manual_seed(rows)
        g, z, up = ((torch.rand((rows, cols), device="cuda", generator=gen) + 0.5).to(t) for _ in range(3))
        z[1, at] = torch.tensor([-INF, INF, NAN], device="cuda", dtype=t)
        d, y, bias = torch.empty_like(g), torch.empty_like(g), torch.empty(cols, device="cuda")
        ws = torch.empty(max(256, cdl.gated_bwd_workspace_bytes(rows, cols)), dtype=torch.uint8, device="cuda")
        act = su.number(cdl, name)
        cdl.cdl_act_bwd(g, rows, cols, act, d_z=d, d_bias=bias, y=y, z=z, ws=ws)
        slopes, values = SLOPES[name], VALUES[name]
        assert same(torch, d[1, at], [s * float(v) for s, v in zip(slopes, g[1, at])]) and same(torch, y[1, at], values)
        rest = torch.ones_like(z, dtype=torch.bool)
        rest[1, at] = False
        assert torch.isfinite(d[rest]).all() and torch.isfinite(y[rest]).all()
        assert [bool(torch.isfinite(v)) for v in bias[at]] == [s == s for s in slopes] and int(torch.isfinite(bias).sum()) == cols - sum(s != s for s in slopes)
        d_up = torch.empty_like(g)
        cdl.cdl_gated_bwd(g, rows, cols, act, d_gate=d, d_up=d_up, y=y, z_gate=z, z_up=up)
        assert same(torch, d_up[1, at], [v * float(f) for v, f in zip(values, g[1, at])]) and same(torch, y[1, at], [v * float(f) for v, f in zip(values, up[1, at])])
        assert [bool(torch.isfinite(v)) for v in d[1, at]] == [s == s for s in slopes]
        assert torch.isfinite(d[rest]).all() and torch.isfinite(d_up[rest]).all() and torch.isfinite(y[rest]).all()
        q, scale = su.quantize(torch, cdl, z)
        cdl.cdl_act_bwd(g, rows, cols, act, d_z=d, y=y, q=q, scale=scale)
        hit = torch.zeros_like(rest)
        hit[1] = True      # (each block of the row has one)
        assert torch.isnan(y[hit]).all() and torch.isfinite(y[~hit]).all() and torch.isfinite(d[~hit]).all()
        assert torch.equal(d, g) if name == "none" else torch.isnan(d[hit]).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("name", su.ACTS)
@pytest.mark.parametrize("size", [(2, 300, 0), (2, 300, 200), (300, 401, 9000), (1021, 1000, 520), (2000, 1999, 520), (3000, 2900, 384)])
def test_products_where_z_is_not_finite(env, size, name, kind):
    torch, cdl = env
    M, N, K = size
    gen = torch.Generator(device="cuda").manual_seed(M)
    a, w = (su.quantize(torch, cdl, torch.randn((n, max(K, 1)), device="cuda", generator=gen) * max(K, 1) ** -0.5) for n in (M, N))
    bias, at = torch.rand(N, device="cuda", generator=gen) + 0.5, [0, N // 2, N - 1]
    bias[at] = torch.tensor([-INF, INF, NAN], device="cuda")
    rest = torch.ones(N, dtype=torch.bool, device="cuda")
    rest[at] = False
    for kept in (False, True):
        y, (z,) = finished(torch, cdl, a, [w], size, kind, name, [bias], [kept])
        assert same(torch, y.t()[at], VALUES[name]) and torch.isfinite(y[:, rest]).all()
        assert not kept or (same(torch, z.t()[at], VALUES["none"]) and torch.isfinite(z[:, rest]).all())
        y, _ = finished(torch, cdl, a, [w, w], size, kind, name, [bias, torch.ones(N, device="cuda") * 1000], [kept, kept])      # (z of the other projection: positive)
        assert same(torch, y.t()[at], VALUES[name]) and torch.isfinite(y[:, rest]).all()


# ---- exact products --------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("sides", [1, 2])
@pytest.mark.parametrize("fa,fb", [("e4m3", "e4m3"), ("e5m2", "e4m3")])
@pytest.mark.parametrize("size", [(1, 48, 300), (3, 1000, 2048), (40, 333, 1300), (64, 4096, 4096), (96, 4096, 512), (300, 401, 9000), (129, 250, 9000), (256, 256, 30000), (1021, 1000, 520), (2000, 1999, 520), (3000, 3001, 200),
                                  (9000, 4000, 256)])
def test_results_in_fp32_leave_nothing_out(env, size, fa, fb, sides):
    """Products of 2^-8 beside one of 2^8 in every 128: each sum and partial sum is a multiple of 2^-8 below 2^16, a number of fp32 whatever the order, so the results are exact.  The instructions
    for eight bits keep of eight products or more at a time what lies above 2^-14 of the largest: they lose those of 2^-8 beside the large one, which leaves four entries of five off."""
    torch, cdl = env
    M, N, K = size
    gen = torch.Generator(device="cuda").manual_seed(M + N + K)

    def matrix(rows, fmt, sign):
        x = (torch.randint(0, 2, (rows, K), device="cuda", generator=gen) * 2 - 1).float() * 2.0 ** -4
        x[:, 37::128] = 16.0
        x[:, 36::128] = 2.0 ** -4 * sign
        return su.quantize(torch, cdl, x, fmt), x.double()
    a, va = matrix(M, fa, 1)
    b = [matrix(N, fb, 1 - 2 * i) for i in range(sides)]
    wants = [va @ v.t() for _, v in b]
    assert all(float(w.abs().max()) < 2.0 ** 16 for w in wants)
    new = lambda: torch.full((M, N), float("nan"), device="cuda")      # noqa: E731
    query = cdl.block8_gemm_act_workspace_bytes if sides == 1 else cdl.block8_gemm_gated_workspace_bytes
    y, z, ws = new(), [new() for _ in b], torch.full((max(256, query(M, N, K)),), 0xff, dtype=torch.uint8, device="cuda")
    fmt = {"e4m3": cdl.E4M3, "e5m2": cdl.E5M2}
    more = dict(act=cdl.ACT_RELU, ws=ws, a_format=fmt[fa], b_format=fmt[fb])
    for keep in (True, False):
        y.fill_(float("nan"))
        if sides == 1:
            cdl.cdl_block8_gemm_act(*a, *b[0][0], M, N, K, y, z=z[0] if keep else None, **more)
            want = wants[0].clamp(min=0)
        else:
            cdl.cdl_block8_gemm_gated(*a, *b[0][0], *b[1][0], M, N, K, y, z_gate=z[0] if keep else None, z_up=z[1] if keep else None, **more)
            want = (wants[0].clamp(min=0) * wants[1]).float().double()      # (one rounding)
        assert all(torch.equal(p.double(), w) for p, w in zip(z, wants)) and torch.equal(y.double(), want)


# ---- sums over the rows of tensors whose offsets pass 32 bits ----------------------------------------------------------

ROWS, COLS = 1050000, 4101      # more than 2^32 entries


def large(torch, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.empty((ROWS, COLS), dtype=torch.bfloat16, device="cuda")
    for first in range(0, ROWS, 1 << 17):
        x[first:first + (1 << 17)] = torch.randn((min(1 << 17, ROWS - first), COLS), device="cuda", generator=gen)
    return x


@pytest.mark.parametrize("kept", [False, True])
@pytest.mark.parametrize("sides", [1, 2])
def test_sums_of_large_activations(env, sides, kept):
    """The gradients of slices are those of calls on the slices, the sums those of all rows in 64 bits."""
    torch, cdl = env
    g, z = large(torch, 1), [large(torch, 2 + i) for i in range(sides)]
    if kept:
        z = [su.quantize(torch, cdl, z.pop()) for _ in range(sides)]
    bias = [torch.full((COLS,), float("nan"), device="cuda") for _ in range(sides)]
    query = cdl.act_bwd_workspace_bytes if sides == 1 else cdl.gated_bwd_workspace_bytes
    ws = torch.empty(query(ROWS, COLS), dtype=torch.uint8, device="cuda")

    def call(g, z, rows, **out):
        names = [""] if sides == 1 else ["_gate", "_up"]
        given = {k + n: t for n, v in zip(names, z) for k, t in zip(("q", "scale") if kept else ("z",), v if kept else (v,))}
        out = {("d_z" if sides == 1 else "d") + n if k == "d" else k + n: t for k, v in out.items() if k != "ws" for n, t in zip(names, v)}
        (cdl.cdl_act_bwd if sides == 1 else cdl.cdl_gated_bwd)(g, rows, COLS, cdl.ACT_SILU, ws=ws, **given, **out)
    d = [torch.empty_like(g) for _ in range(sides)]
    call(g, z, ROWS, d=d, d_bias=bias)
    part = lambda v, at: (v[0][at], v[1][:, at].contiguous()) if kept else v[at]      # noqa: E731
    for first in (0, 523904, 1047168, 1049856):      # around 2^31 and 2^32 entries, and the last rows
        n = min(256, ROWS - first)
        of = [torch.empty((n, COLS), dtype=g.dtype, device="cuda") for _ in d]
        at = slice(first, first + n)
        some = [part(v, at) for v in z]
        if kept and n % 128:
            some = [(q, torch.nn.functional.pad(s, (0, -n % 128))) for q, s in some]
        call(g[at], some, n, d=of)
        assert all(torch.equal(t[at], p) for t, p in zip(d, of)), first
    del d
    sums, sizes = ([torch.zeros(COLS, dtype=torch.float64, device="cuda") for _ in range(sides)] for _ in range(2))
    for first in range(0, ROWS, 1 << 16):
        at = slice(first, min(first + (1 << 16), ROWS))
        values = [su.values(torch, *part(v, at), cols=COLS) if kept else v[at].double() for v in z]
        for i, (v, off) in enumerate(su.act_back(torch, "silu", g[at].double(), values, "float32")[0]):
            sums[i] += v.sum(dim=0)
            sizes[i] += off.sum(dim=0) + (ROWS / 121 / 8 + 40) * su.U * v.abs().sum(dim=0)      # 121 stretches of rows, an eighth of each one behind the other, then 8 + 2 + 18 sums
    for got, want, off in zip(bias, sums, sizes):
        assert su.outside(got, want, off) == 0
