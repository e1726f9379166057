"""The largest sizes that the operators in eight bits accept: a grid holds fewer than 2^32 threads, so what has more entries takes several launches, or is refused."""
import pytest

import launch_recorder
from launch_recorder import A, FLOAT, INT, INT64, POINTER, SIZE

F32, BF16, E4M3 = 0, 1, 0
OK, RANGE = 0, -3
WS = [(POINTER, A), (SIZE, 1 << 60), (POINTER, None)]


def dropout(n, type_):
    return ("cdl_dropout", [(POINTER, A), (POINTER, A), (INT, type_), (INT64, n), (FLOAT, 0.5), (INT64, 3), (INT64, 5), (POINTER, A), (POINTER, None)])


def forward(T, V, D, type_):
    return ("cdl_head_loss_fwd", [(POINTER, A), (POINTER, A), (INT, type_), (POINTER, A), (INT, T), (INT, V), (INT, D), (POINTER, A), (POINTER, A)] + WS)


def backward(T, V, D, type_):
    return ("cdl_head_loss_bwd", [(POINTER, A), (POINTER, A), (INT, type_)] + [(POINTER, A)] * 3 + [(POINTER, None), (INT, T), (INT, V), (INT, D), (POINTER, A), (POINTER, A)] + WS)


def product(M, N, K, y_type):
    return ("cdl_block8_gemm", [(POINTER, A)] * 4 + [(INT, v) for v in (M, N, K, E4M3, E4M3)] + [(POINTER, A), (INT, y_type)] + WS)


def threads(launches, kernel):
    return sum(l.grid[0] * l.threads for l in launches if kernel in l.name)


def check(recorded):
    for launches, _ in recorded:
        assert launches and all(0 < l.grid[0] and l.grid[0] * l.threads < 1 << 32 and l.grid[1:] == (1, 1) for l in launches), launches


@pytest.mark.parametrize("type_", [F32, BF16])
def test_as_many_threads_as_entries(tmp_path, type_):
    sizes = [1, 2049, (1 << 34) - 1, 1 << 34, (1 << 34) + 1, 1 << 35, (1 << 35) + 5, 1 << 40]
    recorded = launch_recorder.record(tmp_path, [dropout(n, type_) for n in sizes])
    check(recorded)
    for n, (launches, _) in zip(sizes, recorded):
        assert n <= 8 * threads(launches, "dropout_kernel") < n + 8 * 256
    rows = 1 << 20
    recorded = launch_recorder.record(tmp_path, [backward(rows, 100, 4096, type_), backward(0, 1 << 30, 1 << 10, type_), forward(64, 1 << 29, 33, type_), forward(64, 1000, 33, type_),
                                                 product(1 << 20, 1 << 20, 0, type_), product(3, 5, 0, type_)])
    check(recorded)
    sums, zeros, copies, small_copies, nothing, small = (r for r, _ in recorded)
    assert threads(sums, "head_sum_kernel") == rows * 4096 and threads(zeros, "head_zero_kernel") == 1 << 40
    assert threads(copies, "head_rows_kernel") == ((1 << 29) + 64) * 8 and threads(nothing, "zero_kernel") == 1 << 40
    assert [l.grid[0] for l in small_copies if "head_rows_kernel" in l.name] == [2, 32] and [l.grid[0] for l in small] == [1]      # (as before: one launch)


def test_quantizer_refuses_more_blocks_than_a_grid_holds(tmp_path):
    import paper_2501_09849_amd as cdl
    f = cdl.load().cdl_block8_quantize
    for rows, cols in ((1, 2 ** 31 - 1), (2 ** 31 - 1, 1), (1 << 20, 1 << 20)):
        assert f(A, BF16, rows, cols, 0, E4M3, A, A, A, A, None) == RANGE
    check(launch_recorder.record(tmp_path, [("cdl_block8_quantize", [(POINTER, A), (INT, BF16), (INT, rows), (INT, cols), (INT, 0), (INT, E4M3)] + [(POINTER, A)] * 4 + [(POINTER, None)])
                                            for rows, cols in ((1, 2 ** 31 - 128), (2 ** 31 - 128, 100), (1 << 18, 1 << 19))]))
