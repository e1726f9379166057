"""What the operators of a feed-forward sublayer promise of their values beyond the roundings' bounds: the same bits whatever else is asked for."""
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
