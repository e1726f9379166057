"""Every form of tiles of the block-scaled product and of the loss's products: whole and ragged, one tile a block and several, split contractions, rows of the result on 16, 4 and 2 bytes,
against sums in 64 bits.  (That these sizes take these forms is checked on the CPU.)"""
import pytest

import eight_bit_cases as cases
import gpu_util as gu
from test_gpu_block8 import check_product, product, quantize, values
from test_gpu_head_loss import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import paper_2501_09849_amd as cdl
    return gu.torch_mod(), cdl


@pytest.mark.parametrize("out", ["float32", "bfloat16"])
@pytest.mark.parametrize("M,N,K", list(cases.PRODUCTS))
def test_product(env, M, N, K, out):
    check_product(*env, M, N, K, out, "e4m3", "e4m3", True)


@pytest.mark.parametrize("out", ["float32", "bfloat16"])
@pytest.mark.parametrize("fa,fb", [("e4m3", "e5m2"), ("e5m2", "e4m3"), ("e5m2", "e5m2")])
@pytest.mark.parametrize("M,N,K", cases.ALL_FORMATS)
def test_product_of_other_formats(env, M, N, K, fa, fb, out):
    check_product(*env, M, N, K, out, fa, fb, False)


@pytest.mark.parametrize("M,N,K", [(4096, 4096, 1024), (2048, 2048, 640), (64, 2048, 640)])
def test_results_in_bf16_are_the_nearest_but_for_few(env, M, N, K):
    """Over random operands the 8-bit instructions are off by about 1.5e-5 of a result's typical size s, which changes its rounding to bf16 only where the result lies that close to the middle between
    two neighbours: they are 2^-8 to 2^-7 |y| apart, so of results of size |y| at most 2 * 1.5e-5 s / (2^-8 |y|) = 0.008 s / |y| are.  Over a normal distribution of y / s that is
    0.008 * 0.8 * ln(1 / 0.008) = 3 % and the 0.6 % of entries below 0.008 s: 4 % at most.  What differs may differ by one unit: 2^-7 of the larger of |y| and 1.5e-5 s times a few."""
    torch, cdl = env
    gen = torch.Generator(device="cuda").manual_seed(M + K)
    x, w = torch.randn((M, K), device="cuda", generator=gen), torch.randn((N, K), device="cuda", generator=gen)
    a, sa, _, _ = quantize(torch, cdl, x, cols=False)
    b, sb, _, _ = quantize(torch, cdl, w, tiles=True, cols=False)
    ref = (values(torch, a, sa, "e4m3") @ values(torch, b, sb, "e4m3").t())
    y = product(torch, cdl, a, sa, b, sb, M, N, K, "bfloat16")
    off = y != ref.float().to(torch.bfloat16)
    assert float(off.double().mean()) < 0.04
    # the sum of 1.5e-5 s (ten times it: the tail) and one unit
    assert ((y.double() - ref).abs() <= 2.0 ** -7 * ref.abs() + 1.5e-4 * float(ref.std())).all()


@pytest.mark.parametrize("T,V,D,type_", list(cases.LOSSES))
def test_loss_and_gradients(env, T, V, D, type_):
    Case(env, T, V, D, type_, with_lse=True).check()
