"""What the entry points of a network in eight bits refuse, the scratch that they ask for and what they launch, without a GPU."""
import ctypes
import os

import numpy as np
import pytest
import torch

import launch_recorder
from launch_recorder import FLOAT, INT, INT64, POINTER, SIZE

OK, NULL, PARAM, RANGE, ALIGN, WS = 0, -1, -2, -3, -4, -5
FAKE = 0x1000      # aligned, never dereferenced: every refusal comes first
F32, BF16, E4M3, E5M2 = 0, 1, 0, 1
BIG = 1 << 40


@pytest.fixture(scope="module")
def cdl():
    import paper_2501_09849_amd as pkg
    import paper_2501_09849_amd.build as b
    if not os.path.exists(b.LIB_PATH):
        b.build_lib()
    pkg.load()
    return pkg


def test_pitches(cdl):
    assert [cdl.block8_pitch(n) for n in (-1, 0, 1, 127, 128, 129, 2**31 - 1)] == [0, 0, 128, 128, 128, 256, 2**31]


def test_scratch_of_products(cdl):
    f = cdl.block8_gemm_workspace_bytes
    assert f(0, 5, 5) == f(5, 0, 5) == f(5, 5, 0) == f(-1, 5, 5) == 0
    assert f(256, 256, 256) == 0                                                # short: not split
    assert f(256, 256, 1 << 20) >= 2 * 256 * 256 * 4                            # few tiles, long: in parts
    assert f(65536, 4096, 1 << 20) == 0                                         # tiles enough
    assert f(256, 256, 1 << 20) % 256 == 0


def test_scratch_of_the_loss(cdl):
    f = cdl.head_loss_workspace_bytes
    assert f(0, 100, 8, F32, True) == 0 and f(-1, 100, 8, F32) == 0 and f(5, 100, 8, 2) == 0
    assert f(1 << 22, 1 << 23, 8, BF16) == 0                                    # beyond the limits
    for type_ in (F32, BF16):
        assert 0 < f(100, 1000, 65, type_) < f(100, 1000, 65, type_, True)
        assert f(100, 1000, 65, type_, True) % 256 == 0
    # bf16 operands on whole K-tiles are read in place; the logits are nowhere near
    assert f(8192, 128000, 2048, BF16) < 8192 * 128000 // 8


def test_quantizer_refuses_before_any_gpu_work(cdl):
    f = cdl.load().cdl_block8_quantize
    good = (FAKE, BF16, 8, 8, 0, E4M3, FAKE, FAKE, FAKE, FAKE, None)

    def but(**at):
        a = list(good)
        for k, v in at.items():
            a[int(k[1:])] = v
        return f(*a)
    assert but(_2=-1) == but(_3=-1) == but(_1=2) == but(_1=-1) == but(_5=2) == PARAM
    assert but(_0=None) == NULL
    assert but(_6=None) == but(_7=None) == but(_8=None) == but(_9=None) == NULL          # a pair is whole or absent
    assert but(_6=None, _7=None, _8=None, _9=None) == NULL
    for k in ("_0", "_6", "_7", "_8", "_9"):
        assert but(**{k: FAKE + 8}) == ALIGN
    assert f(None, F32, 0, 8, 0, E4M3, FAKE, FAKE, None, None, None) in (OK, -6)          # nothing to read (-6: fills of scales need a device)


def test_product_refuses_before_any_gpu_work(cdl):
    f = cdl.load().cdl_block8_gemm
    good = (FAKE, FAKE, FAKE, FAKE, 8, 8, 8, E4M3, E4M3, FAKE, F32, None, 0, None)

    def but(**at):
        a = list(good)
        for k, v in at.items():
            a[int(k[1:])] = v
        return f(*a)
    assert but(_4=-1) == but(_5=-1) == but(_6=-1) == but(_7=2) == but(_8=-1) == but(_10=2) == PARAM
    assert but(_6=(1 << 23) + 1) == but(_4=(1 << 30) + 1) == but(_5=(1 << 30) + 1) == but(_4=1 << 23, _5=(1 << 21) + 1) == RANGE
    for k in ("_0", "_1", "_2", "_3", "_9"):
        assert but(**{k: None}) == NULL and but(**{k: FAKE + 8}) == ALIGN
    need = cdl.block8_gemm_workspace_bytes(8, 8, 1 << 20)
    assert need > 0
    assert but(_6=1 << 20) == WS and but(_6=1 << 20, _11=FAKE, _12=need - 1) == WS and but(_6=1 << 20, _11=FAKE + 64, _12=need) == ALIGN
    assert but(_4=0, _9=None) == but(_5=0, _0=None) == OK                                # nothing to do


def test_loss_refuses_before_any_gpu_work(cdl):
    L = cdl.load()
    need, train = cdl.head_loss_workspace_bytes(8, 9, 8, BF16), cdl.head_loss_workspace_bytes(8, 9, 8, BF16, True)
    forward = (FAKE, FAKE, BF16, FAKE, 8, 9, 8, FAKE, FAKE, FAKE, need, None)
    backward = (FAKE, FAKE, BF16, FAKE, FAKE, FAKE, FAKE, 8, 9, 8, FAKE, FAKE, FAKE, train, None)

    def but(f, good, **at):
        a = list(good)
        for k, v in at.items():
            a[int(k[1:])] = v
        return f(*a)
    for f, good, T in ((L.cdl_head_loss_fwd, forward, 4), (L.cdl_head_loss_bwd, backward, 7)):
        T, V, D = "_%d" % T, "_%d" % (T + 1), "_%d" % (T + 2)
        assert but(f, good, **{T: -1}) == but(f, good, **{V: -1}) == but(f, good, **{D: -1}) == but(f, good, _2=2) == but(f, good, **{V: 0}) == PARAM
        assert but(f, good, **{D: (1 << 20) + 1}) == but(f, good, **{T: (1 << 22) + 1}) == but(f, good, **{V: (1 << 30) + 1}) == RANGE
        assert but(f, good, **{T: 1 << 22, V: (1 << 22) + 1}) == RANGE
        assert but(f, good, _0=None) == but(f, good, _1=None) == but(f, good, _3=None) == NULL
        assert but(f, good, _0=FAKE + 8) == but(f, good, _1=FAKE + 8) == but(f, good, _3=FAKE + 4) == ALIGN
    assert but(L.cdl_head_loss_fwd, forward, _8=None) == NULL and but(L.cdl_head_loss_fwd, forward, _7=FAKE + 2) == ALIGN
    assert but(L.cdl_head_loss_fwd, forward, _9=None) == but(L.cdl_head_loss_fwd, forward, _10=need - 1) == WS
    assert but(L.cdl_head_loss_fwd, forward, _9=FAKE + 64) == ALIGN
    assert but(L.cdl_head_loss_bwd, backward, _4=None) == but(L.cdl_head_loss_bwd, backward, _10=None, _11=None) == NULL
    assert but(L.cdl_head_loss_bwd, backward, _13=train - 1) == WS and but(L.cdl_head_loss_bwd, backward, _10=FAKE + 8) == ALIGN
    assert but(L.cdl_head_loss_fwd, forward, _4=0, _0=None, _3=None, _8=None, _9=None, _10=0) == OK


def test_dropout_refuses_before_any_gpu_work(cdl):
    f = cdl.load().cdl_dropout
    for p in (-0.1, 1.1, float("nan"), float("inf")):
        assert f(FAKE, None, BF16, 8, p, 0, 0, FAKE, None) == PARAM
    assert f(FAKE, None, 2, 8, 0.5, 0, 0, FAKE, None) == f(FAKE, None, BF16, -1, 0.5, 0, 0, FAKE, None) == f(FAKE, None, BF16, BIG + 1, 0.5, 0, 0, FAKE, None) == PARAM
    assert f(None, None, BF16, 8, 0.5, 0, 0, FAKE, None) == f(FAKE, None, BF16, 8, 0.5, 0, 0, None, None) == NULL
    assert f(FAKE + 4, None, BF16, 8, 0.5, 0, 0, FAKE, None) == f(FAKE, FAKE + 4, BF16, 8, 0.5, 0, 0, FAKE, None) == f(FAKE, None, BF16, 8, 0.5, 0, 0, FAKE + 4, None) == ALIGN
    assert f(None, None, BF16, 0, 0.5, 0, 0, None, None) == OK


def test_types_are_those_of_the_tensors(cdl):
    x = torch.zeros(8, 8, dtype=torch.float16)
    q = torch.zeros(8, 128, dtype=torch.uint8)
    with pytest.raises((TypeError, ValueError)):
        cdl.cdl_block8_quantize(x, 8, 8, q, q, stream=0)
    with pytest.raises((TypeError, ValueError)):
        cdl.cdl_dropout(x, 64, 0.5, 0, 0, x, stream=0)
    with pytest.raises((TypeError, ValueError)):
        cdl.cdl_dropout(torch.zeros(8), 8, 0.5, 0, 0, torch.zeros(8, dtype=torch.bfloat16), stream=0)


@pytest.mark.parametrize("seed", [-1, 1.5, 1 << 64, None])
def test_a_seed_is_an_unsigned_integer_of_64_bits(cdl, seed):
    x = torch.zeros(8)
    with pytest.raises((TypeError, OverflowError, ValueError, ctypes.ArgumentError)):
        cdl.cdl_dropout(x, 8, 0.5, seed, 0, x, stream=0)


def test_seeds_reach_the_whole_range(cdl):
    x = torch.zeros(8)
    for seed in ((1 << 64) - 1, np.uint64((1 << 64) - 1)):
        with pytest.raises(cdl.CdlError) as e:      # (accepted: what is refused is the probability)
            cdl.cdl_dropout(x, 8, 2.0, seed, seed, x, stream=0)
        assert e.value.status == PARAM


FORMS = {(2, 2, 4, 4): "wide", (2, 2, 2, 2): "square", (4, 1, 1, 2): "thin"}


def _form(launch):      # (names with bf16 among their arguments stay mangled where c++filt does not know it)
    return next(form for shape, form in FORMS.items() if "RingForm<%d, %d, %d, %d," % shape in launch.name or "RingFormILi%dELi%dELi%dELi%dE" % shape in launch.name)


def _product(M, N, K, y_type=BF16):
    A = launch_recorder.A
    return ("cdl_block8_gemm", [(POINTER, A)] * 4 + [(INT, M), (INT, N), (INT, K), (INT, E4M3), (INT, E5M2), (POINTER, A), (INT, y_type), (POINTER, A), (SIZE, BIG), (POINTER, None)])


def test_forms_of_products(tmp_path):
    asked = {(4, 2048, 768): ("thin", 1), (64, 2048, 768): ("thin", 1), (1000, 1000, 520): ("thin", 1), (2000, 2000, 520): ("square", 1), (4096, 4096, 768): ("wide", 1),
             (65, 200, 1 << 20): ("square", 2), (4, 512, 128 * 47): ("thin", 1), (4, 512, 128 * 48): ("thin", 2), (2048, 2048, 1 << 16): ("wide", 2), (768, 768, 1 << 16): ("square", 2)}
    for (size, (form, count)), (launches, _) in zip(asked.items(), launch_recorder.record(tmp_path, [_product(*size) for size in asked])):
        assert _form(launches[0]) == form and len(launches) == count, size
        assert 8 <= launches[0].grid[0] <= 512 and launches[0].grid[0] % 8 == 0 and launches[0].lds <= 160 << 10
        assert "block8_sum_kernel" in launches[-1].name or count == 1


def test_launches_of_the_loss(tmp_path):
    A = launch_recorder.A

    def backward(T, V, D, type_, d_h=A, d_w=A):
        return ("cdl_head_loss_bwd", [(POINTER, A), (POINTER, A), (INT, type_), (POINTER, A), (POINTER, A), (POINTER, A), (POINTER, None), (INT, T), (INT, V), (INT, D), (POINTER, d_h),
                (POINTER, d_w), (POINTER, A), (SIZE, 1 << 50), (POINTER, None)])

    def count(launches, kernel):
        return sum(kernel in launch.name for launch in launches)
    whole, piecewise, padded, no_w, no_h = (r for r, _ in launch_recorder.record(tmp_path, [
        backward(512, 4096, 256, BF16), backward(8192, 32768, 256, BF16), backward(512, 4096, 250, BF16), backward(512, 4096, 256, BF16, d_w=None), backward(512, 4096, 256, BF16, d_h=None)]))
    assert count(whole, "head_gradient_kernel") == 1 and count(whole, "head_product_kernel") == 2 and count(whole, "head_rows_kernel") == 0
    assert count(piecewise, "head_gradient_kernel") == 2 and count(piecewise, "head_product_kernel") == 4      # pieces of 2^27 entries
    assert count(padded, "head_rows_kernel") == 2                                                             # rows that are not whole K-tiles are copied
    assert count(no_w, "head_product_kernel") == 1 and count(no_h, "head_product_kernel") == 1 and count(no_h, "head_sum_kernel") == 0
    few, many = (r for r, _ in launch_recorder.record(tmp_path, [
        ("cdl_head_loss_fwd", [(POINTER, A), (POINTER, A), (INT, BF16), (POINTER, A), (INT, T), (INT, 4096), (INT, 256), (POINTER, A), (POINTER, A), (POINTER, A), (SIZE, BIG), (POINTER, None)])
        for T in (16, 4096)]))
    assert [_form(r[0]) for r in (few, many)] == ["thin", "wide"] and len(few) == len(many) == 2
