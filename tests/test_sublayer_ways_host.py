"""What a call of a feed-forward sublayer launches may depend on its sizes, not on which outputs it has: without a GPU."""
import itertools
import re

import pytest

import launch_recorder
from launch_recorder import A, INT, POINTER, SIZE

F32, BF16, E4M3 = 0, 1, 0
NONE, RELU, GELU, SILU = 0, 1, 2, 3
WS = [(POINTER, A), (SIZE, 1 << 60), (POINTER, None)]


def product(M, N, K, y_type, act, sides, kept):
    """`kept`: which results before the activation are asked for"""
    name = "cdl_block8_gemm_act" if sides == 1 else "cdl_block8_gemm_gated"
    z = [(POINTER, A if k else None) for k in kept]
    tail = [(POINTER, A), (INT, act), (POINTER, A), (POINTER, A)] if sides == 1 else [(POINTER, A), (POINTER, A), (INT, act), (POINTER, A)]
    return (name, [(POINTER, A)] * (2 + 2 * sides) + [(INT, v) for v in (M, N, K, E4M3, E4M3)] + tail + z + [(INT, y_type)] + WS)


def order(launches):
    """The order in which a product's sums are formed: of parts of the contraction in memory, of eight waves in a block, or of K-tiles one after the other, which all tiles have alike."""
    names = [l.name for l in launches]
    return "parts" if "finish" in names[-1] else "thin" if "thin" in names[0] else "tiles"


# among them sizes whose estimates of two ways lie within what storing z adds to one of them
SIZES = list(itertools.product((1, 16, 40, 64, 96, 128, 200, 300, 512, 1000, 2048, 4096, 9000), (100, 512, 768, 1024, 2048, 4096, 8192), (128, 512, 768, 1024, 2048, 4096, 8192, 32768)))


@pytest.mark.parametrize("sides", [1, 2])
@pytest.mark.parametrize("y_type", [F32, BF16])
def test_the_order_of_sums_does_not_go_by_what_is_kept(tmp_path, sides, y_type):
    choices = [(False,), (True,)] if sides == 1 else list(itertools.product((False, True), repeat=2))
    for act in (NONE, GELU, SILU):
        seen = [[order(launches) for launches, _ in launch_recorder.record(tmp_path, [product(*size, y_type, act, sides, kept) for size in SIZES])] for kept in choices]
        assert {"parts", "thin", "tiles"} <= set(seen[0])
        off = [size for i, size in enumerate(SIZES) if len({s[i] for s in seen}) > 1]
        assert not off, (act, len(off), off[:10])


@pytest.mark.parametrize("type_", [F32, BF16])
def test_rows_of_a_gradient_alone_are_not_one_block(tmp_path, type_):
    """Few rows are one block's for the sake of their sums (weight, bias).  The gradient of x alone takes the blocks that its rows fill."""
    def call(rows, cols, d_weight, d_bias):
        return ("cdl_layer_norm_bwd", [(POINTER, A), (INT, type_), (POINTER, A), (POINTER, None), (POINTER, None), (INT, 0)] + [(POINTER, A)] * 4 + [(INT, rows), (INT, cols), (POINTER, A),
                (POINTER, d_weight), (POINTER, d_bias)] + WS)
    sizes = {(64, 128): 4, (64, 256): 4, (16, 512): 4, (16, 1024): 4, (15, 768): 4, (4, 2048): 4, (4, 4096): 4, (3, 8000): 3, (4, 16384): 4, (1, 16384): 1, (600, 300): 150, (5000, 16384): 250}
    for d_weight, d_bias in ((None, None), (A, A), (A, None), (None, A)):
        for ((rows, cols), blocks), (launches, _) in zip(sizes.items(), launch_recorder.record(tmp_path, [call(*size, d_weight, d_bias) for size in sizes])):
            some = d_weight or d_bias
            few = some and rows <= 64
            assert launches[0].grid[0] == (1 if few else blocks) and len(launches) == (2 if some and not few else 1), (rows, cols)


@pytest.mark.parametrize("sides", [1, 2])
@pytest.mark.parametrize("y_type", [F32, BF16])
def test_blocks_of_few_rows(tmp_path, sides, y_type):
    """16 to 64 rows of a in a block; exact products of two projections 32 at most, more would not fit the registers"""
    rows = {2 if sides == 2 and y_type == F32 else 4}
    seen = set()
    for launches, _ in launch_recorder.record(tmp_path, [product(M, N, K, y_type, SILU, sides, (False,) * sides) for M in (1, 16, 20, 52, 64, 128) for N in (1000, 2048, 4096) for K in (500, 768, 1536, 3000)]):
        if order(launches) == "thin":
            form = re.search(r"(?:true|false), (\d)|Lb[01]ELi(\d)E", launches[0].name)      # (names with bf16 stay mangled)
            seen.add(int(form.group(1) or form.group(2)))
    assert {1, 2} <= seen and max(seen) in rows
