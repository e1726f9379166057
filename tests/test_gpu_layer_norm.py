"""Layer norm and its gradients against sums in 64 bits, its rows in eight bits byte for byte against the block quantizer."""
import pytest

import gpu_util as gu
import sublayer_util as su

pytestmark = pytest.mark.gpu
KINDS = ("float32", "bfloat16")


@pytest.fixture(scope="module")
def env():
    import paper_2501_09849_amd as cdl
    return gu.torch_mod(), cdl


def states(torch, rows, cols, kind, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed + 31 * rows + cols)
    x = torch.randn((rows, cols), device="cuda", generator=gen)
    x = torch.where(torch.rand((rows, cols), device="cuda", generator=gen) < 0.01, x * 8, x)
    x = x * torch.exp2(torch.randn((rows, 1), device="cuda", generator=gen)) + torch.randn((rows, 1), device="cuda", generator=gen)
    w, b = 1 + 0.2 * torch.randn(cols, device="cuda", generator=gen), 0.2 * torch.randn(cols, device="cuda", generator=gen)
    return x.to(getattr(torch, kind)), w, b, gen


def forward(torch, cdl, x, w, b, eps=1e-5, fmt=None):
    rows, cols = x.shape
    y = torch.full_like(x, float("nan"))
    mean, rstd = torch.full((rows,), float("nan"), device="cuda"), torch.full((rows,), float("nan"), device="cuda")
    q, scale = su.empty8(torch, rows, cols) if fmt else (None, None)
    cdl.cdl_layer_norm_fwd(x, rows, cols, y, mean, rstd, weight=w, bias=b, eps=eps, q=q, scale=scale, format=cdl.E5M2 if fmt == "e5m2" else cdl.E4M3)
    torch.cuda.synchronize()
    return y, mean, rstd, q, scale


def backward(torch, cdl, g, mean, rstd, want="xwb", fmt="e4m3", **given):
    rows, cols = g.shape
    out = dict(d_x=torch.full_like(g, float("nan")) if "x" in want else None, d_weight=torch.full((cols,), float("nan"), device="cuda") if "w" in want else None,
               d_bias=torch.full((cols,), float("nan"), device="cuda") if "b" in want else None)
    ws = torch.full((max(256, cdl.layer_norm_bwd_workspace_bytes(rows, cols)),), 0xff, dtype=torch.uint8, device="cuda")
    cdl.cdl_layer_norm_bwd(g, rows, cols, mean, rstd, ws=ws, format=cdl.E5M2 if fmt == "e5m2" else cdl.E4M3, **out, **given)
    torch.cuda.synchronize()
    return out["d_x"], out["d_weight"], out["d_bias"]


# every number of lanes and chunks of a row, whole and ragged, one row to many
SIZES = [(1, 1), (3, 7), (5, 8), (33, 64), (130, 127), (129, 128), (257, 129), (64, 200), (300, 256), (17, 257), (40, 512), (1000, 513), (7, 768), (4100, 1021), (515, 1024), (9, 1025),
         (33, 2047), (21, 2048), (6, 3001), (12, 4096), (5, 4097), (4, 8192), (3, 8200), (2, 16384), (3, 15001), (300, 16376), (1, 16383), (2600, 1536), (20000, 40)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_forward(env, rows, cols, kind):
    torch, cdl = env
    x, w, b, _ = states(torch, rows, cols, kind, 1)
    for weight, bias in ((w, b), (None, None), (w, None)):
        (y, off_y), (mean, off_m), (rstd, off_r) = su.norm(torch, x.double(), weight, bias, 1e-5, kind)
        got = forward(torch, cdl, x, weight, bias)
        assert su.outside(got[1], mean, off_m) == 0 and su.outside(got[2], rstd, off_r) == 0
        assert su.outside(got[0], y, off_y) == 0
    assert all(torch.equal(p, q) for p, q in zip(got[:3], forward(torch, cdl, x, w, None)[:3]))      # same inputs, same bits


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_the_copy_in_eight_bits_is_the_quantizers(env, rows, cols, kind):
    torch, cdl = env
    x, w, b, _ = states(torch, rows, cols, kind, 2)
    for fmt in ("e4m3", "e5m2"):
        y, mean, rstd, q, scale = forward(torch, cdl, x, w, b, fmt=fmt)
        rq, rs = su.quantize(torch, cdl, x, fmt)
        assert torch.equal(q, rq) and torch.equal(scale, rs)
        assert all(torch.equal(p, r) for p, r in zip((y, mean, rstd), forward(torch, cdl, x, w, b)[:3]))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_backward(env, rows, cols, kind):
    torch, cdl = env
    x, w, b, gen = states(torch, rows, cols, kind, 3)
    g, add = (torch.randn((rows, cols), device="cuda", generator=gen).to(x.dtype) for _ in range(2))
    _, mean, rstd, q, scale = forward(torch, cdl, x, w, b, fmt="e4m3")
    for given, at in ((dict(x=x), x.double()), (dict(q=q, scale=scale), su.values(torch, q, scale, "e4m3", cols))):
        for weight, along in ((w, add), (None, None)):
            wants = su.norm_back(torch, g.double(), at, weight, mean, rstd, None if along is None else along.double(), kind)
            got = backward(torch, cdl, g, mean, rstd, weight=weight, add=along, **given)
            assert [su.outside(v, *want) for v, want in zip(got, wants)] == [0, 0, 0]
        some = backward(torch, cdl, g, mean, rstd, want="w", weight=None, **given)
        assert torch.equal(some[1], got[1])
        some = backward(torch, cdl, g, mean, rstd, want="xb", weight=None, **given)
        assert torch.equal(some[0], got[0]) and torch.equal(some[2], got[2])
        assert torch.equal(backward(torch, cdl, g, mean, rstd, want="x", weight=None, **given)[0], got[0])


def test_backward_from_the_wider_format(env):
    torch, cdl = env
    x, w, b, gen = states(torch, 77, 300, "bfloat16", 4)
    g = torch.randn((77, 300), device="cuda", generator=gen).to(x.dtype)
    _, mean, rstd, q, scale = forward(torch, cdl, x, w, b, fmt="e5m2")
    wants = su.norm_back(torch, g.double(), su.values(torch, q, scale, "e5m2", 300), w, mean, rstd, None, "bfloat16")
    got = backward(torch, cdl, g, mean, rstd, weight=w, q=q, scale=scale, fmt="e5m2")
    assert [su.outside(v, *want) for v, want in zip(got, wants)] == [0, 0, 0]


@pytest.mark.parametrize("cols", [100, 768])
def test_gradients_are_those_of_differences(env, cols):
    """Along a direction: (f(x + e) - f(x - e)) / 2 of the sum of g y, in 64 bits, is off by the third derivative's share, and the call by its roundings."""
    torch, cdl = env
    x, w, b, gen = states(torch, 5, cols, "float32", 5)
    g, to = (torch.randn((5, cols), device="cuda", generator=gen) for _ in range(2))
    dw, db = torch.randn(cols, device="cuda", generator=gen), torch.randn(cols, device="cuda", generator=gen)
    _, mean, rstd, _, _ = forward(torch, cdl, x, w, b)
    d_x, d_w, d_b = backward(torch, cdl, g, mean, rstd, x=x, weight=w)

    def f(e):
        y = su.norm(torch, x.double() + e * to.double(), w.double() + e * dw.double(), b.double() + e * db.double(), 1e-5, "float32")[0][0]
        return float((y * g.double()).sum())
    h = 1e-4
    steps = [(f(h) - f(-h)) / (2 * h), (f(2 * h) - f(-2 * h)) / (4 * h)]
    want = (4 * steps[0] - steps[1]) / 3                      # (the third derivative's share cancels)
    got = float((d_x.double() * to).sum() + (d_w.double() * dw).sum() + (d_b.double() * db).sum())
    size = float((d_x.double() * to).abs().sum() + (d_w.double() * dw).abs().sum() + (d_b.double() * db).abs().sum())
    assert abs(got - want) <= 1e-5 * size and abs(want) > 1e-3 * size


@pytest.mark.parametrize("kind", KINDS)
def test_rows_without_spread(env, kind):
    """All entries equal: the rows are the bias; with eps 0 they have no norm, and no other row knows of it."""
    torch, cdl = env
    x, w, b, _ = states(torch, 9, 300, kind, 6)
    x[4] = 3.0
    y, mean, rstd, _, _ = forward(torch, cdl, x, w, b)
    assert float(mean[4]) == 3.0 and abs(float(rstd[4]) * 1e-5 ** 0.5 - 1) < 1e-6 and torch.equal(y[4], b.to(y.dtype))
    one, _, two, _, _ = forward(torch, cdl, x, w, b, eps=0.0)
    assert torch.isnan(one[4]).all() and torch.isinf(two[4])
    keep = torch.arange(9, device="cuda") != 4
    assert torch.isfinite(one[keep]).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("cols", [100, 700, 3000])
def test_what_is_not_finite_stays_in_its_row(env, kind, cols):
    torch, cdl = env
    x, w, b, gen = states(torch, 11, cols, kind, 7)
    clean = forward(torch, cdl, x, w, b, fmt="e4m3")
    bad = x.clone()
    bad[2, 5], bad[7, cols - 1] = float("nan"), float("inf")
    got = forward(torch, cdl, bad, w, b, fmt="e4m3")
    rest = [i for i in range(11) if i not in (2, 7)]
    assert torch.isnan(got[0][[2, 7]]).all() and torch.equal(got[0][rest], clean[0][rest]) and torch.equal(got[3][rest], clean[3][rest])
    assert int(got[4][0, 2]) == 255 and int(got[4][(cols - 1) // 128, 7]) == 255
    g = torch.randn((11, cols), device="cuda", generator=gen).to(x.dtype)
    d = backward(torch, cdl, g, got[1], got[2], want="x", x=bad, weight=w)[0]
    assert torch.isnan(d[[2, 7]]).all() and torch.equal(d[rest], backward(torch, cdl, g, clean[1], clean[2], want="x", x=x, weight=w)[0][rest])


@pytest.mark.parametrize("kind", KINDS)
def test_a_mean_far_from_zero(env, kind):
    """The squares are taken about the mean: rows at 1000 with a spread of one keep their digits."""
    torch, cdl = env
    gen = torch.Generator(device="cuda").manual_seed(8)
    x = (1000 + torch.randn((20, 1000), device="cuda", generator=gen)).to(getattr(torch, kind))
    (y, off), _, (rstd, off_r) = su.norm(torch, x.double(), None, None, 1e-5, kind)
    got = forward(torch, cdl, x, None, None)
    assert su.outside(got[0], y, off) == 0 and su.outside(got[2], rstd, off_r) == 0
    assert float(off_r.max()) < 1e-4 * float(rstd.max())


def test_in_place(env):
    torch, cdl = env
    for cols in (777, 2048):
        x, w, b, gen = states(torch, 50, cols, "bfloat16", 9)
        y, mean, rstd, _, _ = forward(torch, cdl, x, w, b)
        g, add = (torch.randn((50, cols), device="cuda", generator=gen).to(x.dtype) for _ in range(2))
        d_x, _, _ = backward(torch, cdl, g, mean, rstd, x=x, weight=w, add=add)
        own = x.clone()
        cdl.cdl_layer_norm_fwd(own, 50, cols, own, weight=w, bias=b)
        assert torch.equal(own, y)
        for name in ("g", "add"):
            t = dict(g=g.clone(), add=add.clone())
            cdl.cdl_layer_norm_bwd(t["g"], 50, cols, mean, rstd, d_x=t[name], x=x, weight=w, add=t["add"])
            assert torch.equal(t[name], d_x)


def test_no_rows(env):
    torch, cdl = env
    cdl.cdl_layer_norm_fwd(None, 0, 5, None, type=cdl.BF16)
    d = torch.full((2, 5), 7.0, device="cuda")
    cdl.cdl_layer_norm_bwd(None, 0, 5, None, None, d_weight=d[0].clone(), d_bias=None, type=cdl.F32)
    w, b = torch.full((5,), 7.0, device="cuda"), torch.full((5,), 7.0, device="cuda")
    cdl.cdl_layer_norm_bwd(None, 0, 5, None, None, d_weight=w, d_bias=b, type=cdl.F32)
    assert (w == 0).all() and (b == 0).all()
