"""The forms of tiles that the sizes of the GPU tests take, from what their calls launch, without a GPU: a rule of choice that changes must not empty those tests without a word."""
import pytest

import eight_bit_cases as cases
import launch_recorder
from launch_recorder import A, INT, POINTER, SIZE

E4M3, E5M2, F32, BF16 = 0, 1, 0, 1
SHAPES = {"wide": (2, 2, 4, 4), "square": (2, 2, 2, 2), "thin": (4, 1, 1, 2)}
TILES = {"wide": (256, 256), "square": (128, 128), "thin": (128, 64)}


def form(launch):      # (names with bf16 among their arguments stay mangled where c++filt does not know it)
    return next(f for f, shape in SHAPES.items() if "RingForm<%d, %d, %d, %d," % shape in launch.name or "RingFormILi%dELi%dELi%dELi%dE" % shape in launch.name)


def product(M, N, K, y_type):
    return ("cdl_block8_gemm", [(POINTER, A)] * 4 + [(INT, v) for v in (M, N, K, E4M3, E4M3)] + [(POINTER, A), (INT, y_type), (POINTER, A), (SIZE, 1 << 40), (POINTER, None)])


def backward(T, V, D, type_):
    return ("cdl_head_loss_bwd", [(POINTER, A), (POINTER, A), (INT, type_)] + [(POINTER, A)] * 3 + [(POINTER, None)] + [(INT, v) for v in (T, V, D)] +
            [(POINTER, A)] * 3 + [(SIZE, 1 << 50), (POINTER, None)])


@pytest.mark.parametrize("y_type", [F32, BF16])
def test_products_of_the_gpu_tests(tmp_path, y_type):
    for (size, (want, split)), (launches, _) in zip(cases.PRODUCTS.items(), launch_recorder.record(tmp_path, [product(*size, y_type) for size in cases.PRODUCTS])):
        assert form(launches[0]) == want, size
        assert ["block8_gemm_kernel" in l.name for l in launches] == [True, False][:len(launches)] and (len(launches) == 2) == split, size
    assert {(f, s) for f, s in cases.PRODUCTS.values()} == {(f, s) for f in SHAPES for s in (False, True)}      # every form, whole and split
    assert {cases.PRODUCTS[size][0] for size in cases.ALL_FORMATS} == set(SHAPES)


def test_losses_of_the_gpu_tests(tmp_path):
    calls = [backward(T, V, D, BF16 if type_ == "bfloat16" else F32) for T, V, D, type_ in cases.LOSSES]
    for ((T, V, D, type_), (gradient, d_h, d_w, pieces, split)), (launches, _) in zip(cases.LOSSES.items(), launch_recorder.record(tmp_path, calls)):
        size = (T, V, D, type_)
        assert [form(l) for l in launches if "head_gradient_kernel" in l.name] == [gradient] * pieces, size
        products = [l for l in launches if "head_product_kernel" in l.name]
        assert [form(l) for l in products] == [d_h, d_w] * pieces, size
        p, q = TILES[d_h]
        assert (products[0].grid[0] > -(-(-(-D // p) * -(-T // q)) // 8) * 8) == split, size
