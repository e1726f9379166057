"""Block-scaled products with bias, activation and residual, and gated ones, against sums in 64 bits of the values that the bytes stand for."""
import pytest

import gpu_util as gu
import sublayer_util as su

pytestmark = pytest.mark.gpu
KINDS = ("float32", "bfloat16")


@pytest.fixture(scope="module")
def env():
    import paper_2501_09849_amd as cdl
    return gu.torch_mod(), cdl


class Case:
    def __init__(self, torch, cdl, M, N, K, kind, sides, fa="e4m3", fb="e4m3", seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed + M + 7 * N + 31 * K)
        self.torch, self.cdl, self.M, self.N, self.K, self.kind, self.sides = torch, cdl, M, N, K, kind, sides
        self.fa, self.fb = fa, fb
        x = torch.randn((M, K), device="cuda", generator=gen) * torch.exp2(torch.randint(-3, 4, (M, (K + 127) // 128), device="cuda", generator=gen).float()).repeat_interleave(128, dim=1)[:, :K]
        self.a = su.quantize(torch, cdl, x, fa)
        self.b = [su.quantize(torch, cdl, torch.randn((N, K), device="cuda", generator=gen) * max(K, 1) ** -0.5, fb, True) for _ in range(sides)]
        self.bias = [torch.randn(N, device="cuda", generator=gen) for _ in range(sides)]
        self.add = torch.randn((M, N), device="cuda", generator=gen).to(getattr(torch, kind))
        va = su.values(torch, *self.a, fa)
        self.z = {with_bias: [su.product(torch, va, su.values(torch, *b, fb), bias if with_bias else None, kind) for b, bias in zip(self.b, self.bias)] for with_bias in (False, True)}

    def call(self, name, with_bias=True, add=False, keep=True, y=None):
        torch, cdl = self.torch, self.cdl
        new = lambda: torch.full((self.M, self.N), float("nan"), dtype=getattr(torch, self.kind), device="cuda")      # noqa: E731
        y, z = new() if y is None else y, [new() if keep else None for _ in range(self.sides)]
        bias = self.bias if with_bias else [None] * self.sides
        query = cdl.block8_gemm_act_workspace_bytes if self.sides == 1 else cdl.block8_gemm_gated_workspace_bytes
        ws = torch.full((max(256, query(self.M, self.N, self.K)),), 0xff, dtype=torch.uint8, device="cuda")
        fmt = {"e4m3": cdl.E4M3, "e5m2": cdl.E5M2}
        more = dict(act=su.number(cdl, name), ws=ws, a_format=fmt[self.fa], b_format=fmt[self.fb])
        if self.sides == 1:
            cdl.cdl_block8_gemm_act(*self.a, *self.b[0], self.M, self.N, self.K, y, z=z[0], bias=bias[0], add=self.add if add else None, **more)
        else:
            cdl.cdl_block8_gemm_gated(*self.a, *self.b[0], *self.b[1], self.M, self.N, self.K, y, z_gate=z[0], z_up=z[1], bias_gate=bias[0], bias_up=bias[1], **more)
        torch.cuda.synchronize()
        return y, z

    def check(self, name, with_bias=True, add=False):
        torch = self.torch
        y, z = self.call(name, with_bias, add)
        wants = self.z[with_bias]
        for got, (want, off) in zip(z, wants):
            assert su.outside(got, want, off + su.HALF[self.kind] * (want.abs() + off)) == 0
        assert su.outside(y, *su.forward(torch, name, wants, self.add.double() if add else None, self.kind)) == 0
        assert torch.equal(y, self.call(name, with_bias, add, keep=False)[0])      # same inputs, same bits, with z and without


# single tokens, few rows, ragged tiles of every form, contractions of one block and split ones
SIZES = [(1, 1, 1), (1, 128, 128), (1, 2048, 768), (4, 1000, 130), (16, 333, 2048), (17, 48, 300), (33, 129, 640), (64, 64, 64), (64, 260, 4096), (65, 127, 129), (70, 31, 100), (128, 128, 1024),
         (200, 72, 8000), (129, 1001, 384), (255, 257, 256), (512, 512, 512), (1021, 1000, 520), (1024, 770, 4096), (300, 401, 9000), (2000, 1999, 520), (3000, 3001, 200), (3900, 4090, 900),
         (4096, 4098, 128), (2048, 2048, 640), (129, 250, 30001), (256, 256, 32768)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("M,N,K", SIZES)
def test_a_layer(env, M, N, K, kind):
    case = Case(*env, M, N, K, kind, 1)
    case.check("gelu")
    case.check("none", add=True)
    case.check("silu", with_bias=False)
    case.check("relu", add=True)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("M,N,K", SIZES)
def test_a_gated_block(env, M, N, K, kind):
    case = Case(*env, M, N, K, kind, 2)
    case.check("silu")
    case.check("gelu", with_bias=False)


@pytest.mark.parametrize("name", su.ACTS)
@pytest.mark.parametrize("sides", [1, 2])
@pytest.mark.parametrize("M,N,K", [(5, 200, 300), (300, 200, 700), (3000, 2900, 384)])
def test_every_activation(env, M, N, K, sides, name):
    for kind in KINDS:
        Case(*env, M, N, K, kind, sides).check(name, add=sides == 1)


@pytest.mark.parametrize("fa,fb", [("e4m3", "e5m2"), ("e5m2", "e4m3"), ("e5m2", "e5m2")])
@pytest.mark.parametrize("sides", [1, 2])
@pytest.mark.parametrize("M,N,K", [(3, 200, 300), (30, 200, 300), (200, 300, 700), (3000, 2900, 384)])
def test_other_formats(env, M, N, K, sides, fa, fb):
    for kind in KINDS:
        Case(*env, M, N, K, kind, sides, fa, fb).check("silu")


@pytest.mark.parametrize("M,N", [(5, 100), (300, 129), (3000, 2900)])
def test_the_product_is_the_products(env, M, N):
    """Without bias, activation and residual: cdl_block8_gemm's sums, to their roundings."""
    torch, cdl = env
    case = Case(torch, cdl, M, N, 300, "float32", 1)
    y, (z,) = case.call("none", with_bias=False)
    assert torch.equal(y, z)
    ref = torch.empty_like(y)
    ws = torch.empty(max(256, cdl.block8_gemm_workspace_bytes(M, N, 300)), dtype=torch.uint8, device="cuda")
    cdl.cdl_block8_gemm(*case.a, *case.b[0], M, N, 300, ref, ws)
    want, off = case.z[False][0]
    assert su.outside(ref, want, off) == 0 and su.outside(y, ref.double(), 2 * off) == 0


@pytest.mark.parametrize("M,N", [(5, 100), (40, 99), (300, 129), (3000, 2900)])
def test_onto_the_residual(env, M, N):
    torch, cdl = env
    for kind in KINDS:
        case = Case(torch, cdl, M, N, 300, kind, 1)
        want, _ = case.call("gelu", add=True)
        own = case.add.clone()
        keep, case.add = case.add, own
        got, _ = case.call("gelu", add=True, keep=False, y=own)
        assert torch.equal(got, want)
        case.add = keep


@pytest.mark.parametrize("sides", [1, 2])
@pytest.mark.parametrize("M", [3, 300, 3000])
def test_what_is_not_finite_stays_where_it_is(env, sides, M):
    """NaN in an entry of a: in that row; in one of the weights: in that column."""
    torch, cdl = env
    N, K = 400, 300
    gen = torch.Generator(device="cuda").manual_seed(M)
    x, w = torch.randn((M, K), device="cuda", generator=gen), torch.randn((N, K), device="cuda", generator=gen)
    for kind in KINDS:
        case = Case(torch, cdl, M, N, K, kind, sides)
        for at, lines in (("a", M), ("b", N)):
            clean_x, clean_w = su.quantize(torch, cdl, x), su.quantize(torch, cdl, w)
            bad = (x if at == "a" else w).clone()
            bad[2, 200] = float("nan") if kind == "float32" else float("inf")
            case.a, case.b = clean_x, [clean_w] * sides
            clean, clean_z = case.call("silu")
            if at == "a":
                case.a = su.quantize(torch, cdl, bad)
            else:
                case.b = [clean_w] * (sides - 1) + [su.quantize(torch, cdl, bad)]
            got, z = case.call("silu")
            rest = [i for i in range(lines) if i != 2]
            for p, q in ((got, clean), (z[-1], clean_z[-1])):
                p, q = (p, q) if at == "a" else (p.t(), q.t())
                assert torch.isnan(p[2]).all() and torch.equal(p[rest], q[rest])


def test_empty_sizes(env):
    torch, cdl = env
    bias = torch.tensor([1.0, -2.0, 3.0], device="cuda")
    y, z = torch.full((2, 3), 7.0, device="cuda"), torch.full((2, 3), 7.0, device="cuda")
    cdl.cdl_block8_gemm_act(None, None, None, None, 2, 3, 0, y, z=z, bias=bias, act=cdl.ACT_RELU)
    assert y.tolist() == [[1.0, 0.0, 3.0]] * 2 and z.tolist() == [[1.0, -2.0, 3.0]] * 2
    cdl.cdl_block8_gemm_gated(None, None, None, None, None, None, 2, 3, 0, y, bias_gate=bias, bias_up=bias, act=cdl.ACT_RELU)
    assert y.tolist() == [[1.0, 0.0, 9.0]] * 2
    cdl.cdl_block8_gemm_act(None, None, None, None, 0, 3, 128, None, y_type=cdl.F32)
    cdl.cdl_block8_gemm_gated(None, None, None, None, None, None, 3, 0, 128, None, y_type=cdl.BF16)
