"""The operators in eight bits over tensors whose offsets pass 32 bits, in entries and in bytes: their ends against calls on the ends alone, or against sums in 64 bits."""
import pytest

import gpu_util as gu
from test_gpu_block8 import values
from test_gpu_head_loss import U

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import paper_2501_09849_amd as cdl
    torch = gu.torch_mod()
    yield torch, cdl
    torch.cuda.empty_cache()


@pytest.mark.parametrize("n", [2 ** 32 + 11, 2 ** 34 + 2 ** 12 + 3])      # (the second one takes two launches)
def test_dropout(env, n):
    torch, cdl = env
    x = torch.empty(n, dtype=torch.bfloat16, device="cuda").fill_(3.0)
    cdl.cdl_dropout(x, n, 0.25, 77, 5, x)
    for first in (0, 2 ** 31 - 8, 2 ** 32 - 1024, 2 ** 34 - 1024, n // 8 * 8 - 4096):
        if first < n:
            count = min(4096, n - first)
            part = torch.full((count,), 3.0, dtype=torch.bfloat16, device="cuda")
            cdl.cdl_dropout(part, count, 0.25, 77, 5 + first // 8, part)
            assert torch.equal(x[first:first + count], part), first
    last = n - n % 8
    part = torch.full((n - last,), 3.0, dtype=torch.bfloat16, device="cuda")
    cdl.cdl_dropout(part, n - last, 0.25, 77, 5 + last // 8, part)
    assert torch.equal(x[last:], part)


@pytest.mark.parametrize("tiles", [False, True])
def test_quantizer(env, tiles):
    torch, cdl = env
    rows, cols = 1050000, 4097
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    for first in range(0, rows, 1 << 17):
        x[first:first + (1 << 17)] = torch.randn((min(1 << 17, rows - first), cols), device="cuda", generator=gen)
    across, down = cdl.block8_pitch(cols), cdl.block8_pitch(rows)
    q, s = torch.empty((rows, across), dtype=torch.uint8, device="cuda"), torch.empty((across // 128, down), dtype=torch.uint8, device="cuda")
    qt, st = torch.empty((cols, down), dtype=torch.uint8, device="cuda"), torch.empty((down // 128, across), dtype=torch.uint8, device="cuda")
    cdl.cdl_block8_quantize(x, rows, cols, q, s, qt, st, tiles=tiles)
    for first in (0, 524160, 1048448):      # (the rows around 2^31 and 2^32 entries, and the last ones; multiples of 128)
        count = min(256, rows - first)
        pitch = cdl.block8_pitch(count)
        part = x[first:first + count].contiguous()
        pq, ps = torch.empty((count, across), dtype=torch.uint8, device="cuda"), torch.empty((across // 128, pitch), dtype=torch.uint8, device="cuda")
        pqt, pst = torch.empty((cols, pitch), dtype=torch.uint8, device="cuda"), torch.empty((pitch // 128, across), dtype=torch.uint8, device="cuda")
        cdl.cdl_block8_quantize(part, count, cols, pq, ps, pqt, pst, tiles=tiles)
        assert torch.equal(q[first:first + count], pq) and torch.equal(s[:, first:first + pitch], ps)
        assert torch.equal(qt[:, first:first + pitch], pqt) and torch.equal(st[first // 128:first // 128 + pitch // 128], pst)


@pytest.mark.parametrize("out", ["bfloat16", "float32"])
def test_product(env, out):
    torch, cdl = env
    M, N, K = 1050000, 4099, 100
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, w = torch.randn((M, K), device="cuda", generator=gen), torch.randn((N, K), device="cuda", generator=gen)
    a, sa = torch.empty((M, 128), dtype=torch.uint8, device="cuda"), torch.empty((1, cdl.block8_pitch(M)), dtype=torch.uint8, device="cuda")
    b, sb = torch.empty((N, 128), dtype=torch.uint8, device="cuda"), torch.empty((1, cdl.block8_pitch(N)), dtype=torch.uint8, device="cuda")
    cdl.cdl_block8_quantize(x, M, K, a, sa)
    cdl.cdl_block8_quantize(w, N, K, b, sb)
    y = torch.empty((M, N), dtype=getattr(torch, out), device="cuda")
    ws = torch.empty(max(256, cdl.block8_gemm_workspace_bytes(M, N, K)), dtype=torch.uint8, device="cuda")
    cdl.cdl_block8_gemm(a, sa, b, sb, M, N, K, y, ws)
    vb = values(torch, b, sb, "e4m3")
    for first in (0, 261900, 523900, 1047700, M - 300):      # (around 2^30, 2^31 and 2^32 entries, and the last)
        va = values(torch, a[first:first + 300], sa[:, first:first + 300], "e4m3")
        ref, size = va @ vb.t(), va.abs() @ vb.abs().t()
        # as for the small products: K exact products summed in fp32; bf16: what the instructions leave out, and a rounding
        bound = K * 2.0 ** -24 * size
        if out == "bfloat16":
            bound = bound + 2.0 ** -10 * size + 2.0 ** -8 * (ref.abs() + 2.0 ** -10 * size)
        assert ((y[first:first + 300].double() - ref).abs() <= bound).all(), first


@pytest.mark.parametrize("D", [2048, 2044])      # (operands as they are, and copied)
def test_loss(env, D):
    torch, cdl = env
    T, V = 20, 1050007
    gen = torch.Generator(device="cuda").manual_seed(5)
    h = torch.randn((T, D), device="cuda", generator=gen).bfloat16()
    w = torch.empty((V, D), dtype=torch.bfloat16, device="cuda")
    step = 1 << 17
    for first in range(0, V, step):
        w[first:first + step] = torch.randn((min(step, V - first), D), device="cuda", generator=gen) * (1.5 / D ** 0.5)
    target = torch.randint(0, V, (T,), device="cuda", generator=gen)
    target[:3] = torch.tensor([0, V - 1, -1])
    ok = target >= 0
    loss, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    d_h, d_w = torch.empty_like(h), torch.empty_like(w)
    ws = torch.empty(cdl.head_loss_workspace_bytes(T, V, D, cdl.BF16, True), dtype=torch.uint8, device="cuda")
    cdl.cdl_head_loss_fwd(h, w, target, T, V, D, loss, lse, ws)
    cdl.cdl_head_loss_bwd(h, w, target, lse, T, V, D, d_h, d_w, ws)
    z = torch.cat([h.double() @ w[first:first + step].double().t() for first in range(0, V, step)], dim=1)
    ref = torch.logsumexp(z, dim=1)
    at = torch.where(ok, target, 0)
    # D products, an exponential's argument, 32 terms in a row and the sums of V / 32 stretches, 1024 / 4 threads' worth of them in a row at most
    error = (D + 2) * U * D * 6.0 * 1.5 / D ** 0.5 + (512 + 16 * z.abs().amax(dim=1)) * U
    assert ((lse.double() - ref).abs() <= error).all()
    assert ((loss.double() - torch.where(ok, ref - z.gather(1, at[:, None])[:, 0], 0.0)).abs() <= error).all()
    g = torch.exp(z - ref[:, None]) * ok[:, None]
    g.scatter_add_(1, at[:, None], -ok.double()[:, None])
    want = sum(g[:, first:first + step] @ w[first:first + step].double() for first in range(0, V, step))
    assert float((d_h.double() - want).norm()) <= 2.0 ** -8 * float(want.norm())
    for first in (0, 524200, 1048500, V - 300):      # (words around 2^30, 2^31 entries, and the last)
        part = g[:, first:first + 300].t() @ h.double()
        assert float((d_w[first:first + 300].double() - part).norm()) <= 2.0 ** -8 * float(part.norm()), first
