"""Tensors of another type than a call of the operators in eight bits reads or writes are refused: they would be read and written beyond their ends, or as other numbers."""
import os

import pytest
import torch

F32, BF16, E4M3, E5M2 = 0, 1, 0, 1
RANGE, PARAM = -3, -2
f32, bf16, f16 = torch.float32, torch.bfloat16, torch.float16
WS = torch.zeros(1 << 20, dtype=torch.uint8)


@pytest.fixture(scope="module")
def cdl():
    import paper_2501_09849_amd as pkg
    import paper_2501_09849_amd.build as b
    if not os.path.exists(b.LIB_PATH):
        b.build_lib()
    pkg.load()
    return pkg


def zeros(dtype, *shape):
    return torch.zeros(shape, dtype=dtype)


def loss_arguments(**other):
    a = dict(h=zeros(bf16, 8, 64), w=zeros(bf16, 9, 64), target=zeros(torch.int64, 8), loss=zeros(f32, 8), lse=zeros(f32, 8), d_loss=zeros(f32, 8), d_lse=zeros(f32, 8),
             d_h=zeros(bf16, 8, 64), d_w=zeros(bf16, 9, 64), type=None, D=64)
    a.update(other)
    return a


def forward(cdl, **other):
    a = loss_arguments(**other)
    cdl.cdl_head_loss_fwd(a["h"], a["w"], a["target"], 8, 9, a["D"], a["loss"], a["lse"], WS, stream=0, type=a["type"])


def backward(cdl, **other):
    a = loss_arguments(**other)
    cdl.cdl_head_loss_bwd(a["h"], a["w"], a["target"], a["lse"], 8, 9, a["D"], a["d_h"], a["d_w"], WS, d_loss=a["d_loss"], d_lse=a["d_lse"], stream=0, type=a["type"])


@pytest.mark.parametrize("dtype", [bf16, f16, torch.float64, torch.int32])
def test_vectors_of_the_loss_are_fp32(cdl, dtype):
    for call, names in ((forward, ("loss", "lse")), (backward, ("lse", "d_loss", "d_lse"))):
        for name in names:
            with pytest.raises(TypeError):
                call(cdl, **{name: zeros(dtype, 8)})


@pytest.mark.parametrize("call,names", [(forward, ("h", "w")), (backward, ("h", "w", "d_h", "d_w"))])
def test_matrices_of_the_loss_are_of_one_type(cdl, call, names):
    for name in names:
        for dtype in (f32, f16):
            with pytest.raises(TypeError):
                call(cdl, **{name: zeros(dtype, 9, 64)})
    address = dict(h=1 << 20, type=BF16)                  # the type of an address holds for the tensors beside it
    with pytest.raises(TypeError):
        call(cdl, **dict(address, w=zeros(f32, 9, 64)))
    with pytest.raises(TypeError):
        call(cdl, h=1 << 20)
    for dtype in (torch.int32, f32):
        with pytest.raises(TypeError):
            call(cdl, target=zeros(dtype, 8))


def test_a_type_that_is_given_is_the_tensors(cdl):
    with pytest.raises(TypeError):
        forward(cdl, type=F32)
    with pytest.raises(TypeError):
        backward(cdl, type=F32)
    with pytest.raises(TypeError):
        cdl.cdl_dropout(zeros(bf16, 8), 8, 0.5, 0, 0, zeros(bf16, 8), type=F32, stream=0)
    with pytest.raises(TypeError):
        cdl.cdl_dropout(1 << 20, 8, 0.5, 0, 0, zeros(bf16, 8), type=F32, stream=0)
    with pytest.raises(TypeError):
        cdl.cdl_dropout(1 << 20, 8, 0.5, 0, 0, 1 << 20, add=zeros(f32, 8), type=BF16, stream=0)
    with pytest.raises(TypeError):
        quantize(cdl, x=zeros(bf16, 8, 8), type=F32)
    with pytest.raises(TypeError):
        product(cdl, y=zeros(bf16, 8, 8), y_type=F32)


def quantize(cdl, rows=8, **other):
    a = dict(x=zeros(f32, 8, 8), q=zeros(torch.uint8, 8, 128), scale=zeros(torch.uint8, 1, 128), q_t=zeros(torch.uint8, 8, 128), scale_t=zeros(torch.uint8, 1, 128), format=E4M3, type=None)
    a.update(other)
    cdl.cdl_block8_quantize(a["x"], rows, 8, a["q"], a["scale"], a["q_t"], a["scale_t"], format=a["format"], type=a["type"], stream=0)


def product(cdl, K=8, **other):
    a = dict(a=zeros(torch.uint8, 8, 128), a_scale=zeros(torch.uint8, 1, 128), b=zeros(torch.uint8, 8, 128), b_scale=zeros(torch.uint8, 1, 128), y=zeros(f32, 8, 8), a_format=E4M3,
             b_format=E4M3, y_type=None)
    a.update(other)
    cdl.cdl_block8_gemm(a["a"], a["a_scale"], a["b"], a["b_scale"], 8, 8, K, a["y"], None, a_format=a["a_format"], b_format=a["b_format"], y_type=a["y_type"], stream=0)


@pytest.mark.parametrize("dtype", [f32, bf16, torch.int16, torch.float8_e4m3fnuz])
def test_bytes_are_bytes(cdl, dtype):
    for name in ("q", "scale", "q_t", "scale_t"):
        with pytest.raises(TypeError):
            quantize(cdl, **{name: zeros(dtype, 8, 128)})
    for name in ("a", "a_scale", "b", "b_scale"):
        with pytest.raises(TypeError):
            product(cdl, **{name: zeros(dtype, 8, 128)})


def test_formats_are_those_of_the_tensors(cdl):
    own = {E4M3: torch.float8_e4m3fn, E5M2: torch.float8_e5m2}
    for format in (E4M3, E5M2):
        other = zeros(own[1 - format], 8, 128)
        for name in ("q", "q_t"):
            with pytest.raises(TypeError):
                quantize(cdl, format=format, **{name: other})
        for name, which in (("a", "a_format"), ("b", "b_format")):
            with pytest.raises(TypeError):
                product(cdl, **{name: other, which: format})


def test_what_fits_is_accepted(cdl):
    """... as far as the sizes, which the library refuses before it touches anything"""
    def refused(status, call, **other):
        with pytest.raises(cdl.CdlError) as e:
            call(cdl, **other)
        assert e.value.status == status
    for call in (forward, backward):
        for dtype, type_ in ((bf16, None), (bf16, BF16), (f32, None), (f32, F32)):
            refused(RANGE, call, h=zeros(dtype, 8, 64), w=zeros(dtype, 9, 64), d_h=zeros(dtype, 8, 64), d_w=zeros(dtype, 9, 64), type=type_, D=(1 << 20) + 1)
        refused(RANGE, call, h=1 << 20, type=BF16, D=(1 << 20) + 1)
        refused(RANGE, call, lse=1 << 20, loss=None, d_loss=None, d_lse=1 << 20, d_h=None, D=(1 << 20) + 1)
    for kind in (torch.uint8, torch.int8):
        for format, own in ((E4M3, torch.float8_e4m3fn), (E5M2, torch.float8_e5m2)):
            for values in (zeros(kind, 8, 128), zeros(own, 8, 128)):
                for scales in (zeros(kind, 1, 128), zeros(torch.float8_e8m0fnu, 1, 128)):
                    refused(RANGE, product, K=(1 << 23) + 1, a=values, b=values, a_scale=scales, b_scale=scales, a_format=format, b_format=format)
                    refused(PARAM, quantize, rows=-1, q=values, q_t=values, scale=scales, scale_t=scales, format=format)
    refused(PARAM, quantize, format=7)
    refused(PARAM, product, a_format=7)
    refused(PARAM, quantize, x=1 << 20, type=5)
    refused(RANGE, product, K=(1 << 23) + 1, y=1 << 20, y_type=BF16, a=1 << 20, a_scale=1 << 20)
