"""What the entry points of a feed-forward sublayer refuse, the scratch that they ask for and what they launch, without a GPU."""
import os

import pytest
import torch

import launch_recorder
from launch_recorder import A, FLOAT, INT, POINTER, SIZE

OK, NULL, PARAM, RANGE, ALIGN, WS = 0, -1, -2, -3, -4, -5
FAKE = 0x1000      # aligned, never dereferenced: every refusal comes first
F32, BF16, E4M3, E5M2 = 0, 1, 0, 1
NONE, RELU, GELU, SILU = 0, 1, 2, 3
BIG = 1 << 50
f32, bf16, u8 = torch.float32, torch.bfloat16, torch.uint8


@pytest.fixture(scope="module")
def cdl():
    import paper_2501_09849_amd as pkg
    import paper_2501_09849_amd.build as b
    if not os.path.exists(b.LIB_PATH):
        b.build_lib()
    pkg.load()
    return pkg


class Call:
    """A call that the library would take, and what becomes of it with other arguments"""

    def __init__(self, cdl, name, **args):
        self.f, self.args = getattr(cdl.load(), name), args

    def __call__(self, **other):
        assert set(other) <= set(self.args)
        a = dict(self.args)
        a.update(other)
        return self.f(*a.values())


def norm_fwd(cdl):
    return Call(cdl, "cdl_layer_norm_fwd", x=FAKE, type=BF16, weight=FAKE, bias=FAKE, rows=8, cols=8, eps=1e-5, y=FAKE, mean=FAKE, rstd=FAKE, q=FAKE, scale=FAKE, format=E4M3, stream=None)


def norm_bwd(cdl):
    return Call(cdl, "cdl_layer_norm_bwd", g=FAKE, type=BF16, x=FAKE, q=None, scale=None, format=E4M3, weight=FAKE, mean=FAKE, rstd=FAKE, add=FAKE, rows=8, cols=8, d_x=FAKE,
                d_weight=FAKE, d_bias=FAKE, ws=FAKE, ws_bytes=BIG, stream=None)


def product(cdl):
    return Call(cdl, "cdl_block8_gemm_act", a=FAKE, a_scale=FAKE, b=FAKE, b_scale=FAKE, M=8, N=8, K=8, a_format=E4M3, b_format=E4M3, bias=FAKE, act=GELU, add=FAKE, y=FAKE, z=FAKE,
                y_type=F32, ws=FAKE, ws_bytes=BIG, stream=None)


def gated(cdl):
    return Call(cdl, "cdl_block8_gemm_gated", a=FAKE, a_scale=FAKE, b=FAKE, b_scale=FAKE, up=FAKE, up_scale=FAKE, M=8, N=8, K=8, a_format=E4M3, b_format=E4M3, bias=FAKE, bias_up=FAKE,
                act=GELU, y=FAKE, z=FAKE, z_up=FAKE, y_type=F32, ws=FAKE, ws_bytes=BIG, stream=None)


def act_bwd(cdl):
    return Call(cdl, "cdl_act_bwd", g=FAKE, type=BF16, z=FAKE, q=None, scale=None, format=E4M3, act=GELU, rows=8, cols=8, d_z=FAKE, d_bias=FAKE, y=FAKE, ws=FAKE, ws_bytes=BIG, stream=None)


def gated_bwd(cdl):
    return Call(cdl, "cdl_gated_bwd", g=FAKE, type=BF16, z=FAKE, z_up=FAKE, q=None, scale=None, q_up=None, scale_up=None, format=E4M3, act=GELU, rows=8, cols=8, d_z=FAKE, d_up=FAKE,
                d_bias=FAKE, d_bias_up=FAKE, y=FAKE, ws=FAKE, ws_bytes=BIG, stream=None)


ALL = (norm_fwd, norm_bwd, product, gated, act_bwd, gated_bwd)


@pytest.mark.parametrize("make", ALL)
def test_numbers(cdl, make):
    call = make(cdl)
    sizes = [k for k in ("rows", "cols", "M", "N", "K") if k in call.args]
    for k in sizes:
        assert call(**{k: -1}) == PARAM, k
    for k in ("type", "y_type", "format", "a_format", "b_format"):
        if k in call.args:
            assert call(**{k: 2}) == call(**{k: -1}) == PARAM, k
    if "act" in call.args:
        assert call(act=4) == call(act=-1) == PARAM
    if "eps" in call.args:
        assert call(eps=-1e-9) == call(eps=float("nan")) == call(eps=float("inf")) == PARAM
    if make in (norm_fwd, norm_bwd):
        assert call(cols=0) == PARAM
        assert call(cols=16385) == call(rows=(1 << 30) + 1) == call(rows=(1 << 30) - 1, cols=16384 + 1) == RANGE
    elif "rows" in call.args:
        assert call(cols=(1 << 24) + 1) == call(rows=(1 << 30) + 1) == call(rows=1 << 21, cols=(1 << 23) + 1) == RANGE
    else:
        assert call(K=(1 << 23) + 1) == call(M=(1 << 30) + 1) == call(N=(1 << 30) + 1) == call(M=1 << 23, N=(1 << 21) + 1) == RANGE


@pytest.mark.parametrize("make,needed", [(norm_fwd, "x y"), (norm_bwd, "g mean rstd"), (product, "a a_scale b b_scale y"), (gated, "a a_scale b b_scale up up_scale y"), (act_bwd, "g"),
                                         (gated_bwd, "g")])
def test_what_has_to_be_there(cdl, make, needed):
    call = make(cdl)
    for k in needed.split():
        assert call(**{k: None}) == NULL, k


@pytest.mark.parametrize("make", ALL)
def test_alignment(cdl, make):
    call = make(cdl)
    for k, v in call.args.items():
        if v == FAKE and k != "ws":
            by = 2 if k in ("mean", "rstd") else 8
            assert call(**{k: FAKE + by}) == ALIGN, k
    for k in ("q", "scale", "q_up", "scale_up"):
        if k in call.args:
            assert call(**{k: FAKE + 8}) in (ALIGN, NULL)


def test_a_copy_in_eight_bits_is_whole_or_absent(cdl):
    call = norm_fwd(cdl)
    assert call(q=None) == call(scale=None) == NULL
    for make in (norm_bwd, act_bwd):
        call = make(cdl)
        z = "x" if make is norm_bwd else "z"
        assert call(**{z: None}) == call(q=FAKE) == call(scale=FAKE) == call(q=FAKE, scale=FAKE) == NULL      # one of the two
        assert call(**{z: None}, q=FAKE) == call(**{z: None}, scale=FAKE) == NULL
        assert call(**{z: None}, q=FAKE, scale=FAKE, rows=1000, ws_bytes=0) == WS                            # (as far as the next refusal)
    call = gated_bwd(cdl)
    kept = dict(z=None, z_up=None, q=FAKE, scale=FAKE, q_up=FAKE, scale_up=FAKE)
    assert call(**kept, rows=1000, ws_bytes=0) == WS
    for k in kept:
        assert call(**dict(kept, **{k: FAKE if kept[k] is None else None})) == NULL
    assert call(z=None, q=FAKE, scale=FAKE) == NULL      # both tensors or both in eight bits


def test_an_output_has_to_be_asked_for(cdl):
    assert norm_bwd(cdl)(d_x=None, d_weight=None, d_bias=None) == NULL
    assert act_bwd(cdl)(d_z=None, d_bias=None, y=None) == NULL
    assert gated_bwd(cdl)(d_z=None, d_up=None, d_bias=None, d_bias_up=None, y=None) == NULL


def test_scratch(cdl):
    norm, act, gate = cdl.layer_norm_bwd_workspace_bytes, cdl.act_bwd_workspace_bytes, cdl.gated_bwd_workspace_bytes
    for f in (norm, act, gate):
        assert f(0, 8) == f(-1, 8) == f(8, -1) == f((1 << 30) + 1, 8) == 0
        assert f(1000, 300) > 0 and f(1000, 300) % 256 == 0
        assert f(1 << 20, 300) <= 64 << 20      # not with the rows
    assert norm(8, 16385) == act(8, (1 << 24) + 1) == 0 and act(1000, 300) < gate(1000, 300) <= 2 * act(1000, 300)
    assert norm(8, 8) == act(8, 8) == gate(384, 8) == 0      # one block alone
    for make, f in ((norm_bwd, norm), (act_bwd, act), (gated_bwd, gate)):
        call, need = make(cdl), f(1000, 8)
        assert call(rows=1000, ws_bytes=need - 1) == call(rows=1000, ws=None) == WS and call(rows=1000, ws=FAKE + 128) == ALIGN
    for f, call in ((cdl.block8_gemm_act_workspace_bytes, product(cdl)), (cdl.block8_gemm_gated_workspace_bytes, gated(cdl))):
        assert f(0, 5, 5) == f(5, 0, 5) == f(5, 5, 0) == f(-1, 5, 5) == f(5, 5, (1 << 23) + 1) == 0
        assert f(1, 4096, 1024) == f(65536, 4096, 1024) == 0                          # finished in the kernel
        assert f(300, 300, 1 << 20) >= 300 * 300 * 4 and f(300, 300, 1 << 20) % 256 == 0
        big = dict(M=300, N=300, K=1 << 20)
        assert call(**big, ws_bytes=f(300, 300, 1 << 20) - 1) == call(**big, ws=None) == WS and call(**big, ws=FAKE + 128) == ALIGN
    assert norm_bwd(cdl)(d_weight=None, d_bias=None, ws=None, ws_bytes=0, d_x=FAKE + 8) == ALIGN      # (no scratch for d_x alone: the next refusal)


def zeros(dtype, *shape):
    return torch.zeros(shape, dtype=dtype)


def python_calls(cdl, t):
    """the Python calls on tensors of one type, with others in the place of single arguments; every one is refused for its sizes"""
    m = lambda d=t: zeros(d, 8, 8)      # noqa: E731
    v = lambda: zeros(f32, 8)      # noqa: E731
    b = lambda: zeros(u8, 8, 128)      # noqa: E731

    def with_defaults(f, defaults):
        return lambda **o: f(dict(defaults, **o))
    return {
        "layer_norm_fwd": (with_defaults(lambda a: cdl.cdl_layer_norm_fwd(a["x"], -1, 8, a["y"], a["mean"], a["rstd"], weight=a["weight"], bias=a["bias"], q=a["q"], scale=a["scale"], stream=0),
                                         dict(x=m(), y=m(), mean=v(), rstd=v(), weight=v(), bias=v(), q=b(), scale=b()))),
        "layer_norm_bwd": (with_defaults(lambda a: cdl.cdl_layer_norm_bwd(a["g"], -1, 8, a["mean"], a["rstd"], d_x=a["d_x"], d_weight=a["d_weight"], d_bias=a["d_bias"], x=a["x"], q=a["q"],
                                                                          scale=a["scale"], weight=a["weight"], add=a["add"], stream=0),
                                         dict(g=m(), x=m(), add=m(), d_x=m(), mean=v(), rstd=v(), weight=v(), d_weight=v(), d_bias=v(), q=b(), scale=b()))),
        "block8_gemm_act": (with_defaults(lambda a: cdl.cdl_block8_gemm_act(a["a"], a["a_scale"], a["b"], a["b_scale"], -1, 8, 8, a["y"], z=a["z"], bias=a["bias"], add=a["add"], stream=0),
                                          dict(y=m(), z=m(), add=m(), bias=v(), a=b(), a_scale=b(), b=b(), b_scale=b()))),
        "block8_gemm_gated": (with_defaults(lambda a: cdl.cdl_block8_gemm_gated(a["a"], a["a_scale"], a["b"], a["b_scale"], a["u"], a["u_scale"], -1, 8, 8, a["y"], z_gate=a["z"], z_up=a["zu"],
                                                                                bias_gate=a["bias"], bias_up=a["bias_up"], stream=0),
                                            dict(y=m(), z=m(), zu=m(), bias=v(), bias_up=v(), a=b(), a_scale=b(), b=b(), b_scale=b(), u=b(), u_scale=b()))),
        "act_bwd": (with_defaults(lambda a: cdl.cdl_act_bwd(a["g"], -1, 8, cdl.ACT_GELU, d_z=a["d"], d_bias=a["d_bias"], y=a["y"], z=a["z"], q=a["q"], scale=a["scale"], stream=0),
                                  dict(g=m(), z=m(), d=m(), y=m(), d_bias=v(), q=b(), scale=b()))),
        "gated_bwd": (with_defaults(lambda a: cdl.cdl_gated_bwd(a["g"], -1, 8, cdl.ACT_GELU, d_gate=a["d"], d_up=a["du"], d_bias_gate=a["d_bias"], d_bias_up=a["d_bias_up"], y=a["y"], z_gate=a["z"],
                                                                z_up=a["zu"], q_gate=a["q"], scale_gate=a["scale"], q_up=a["qu"], scale_up=a["scale_up"], stream=0),
                                    dict(g=m(), z=m(), zu=m(), d=m(), du=m(), y=m(), d_bias=v(), d_bias_up=v(), q=b(), scale=b(), qu=b(), scale_up=b()))),
    }


VECTORS = ("mean", "rstd", "weight", "bias", "bias_up", "d_weight", "d_bias", "d_bias_up")
BYTES = ("q", "qu", "a", "b", "u")
SCALES = ("scale", "scale_up", "a_scale", "b_scale", "u_scale")


@pytest.mark.parametrize("name", ["layer_norm_fwd", "layer_norm_bwd", "block8_gemm_act", "block8_gemm_gated", "act_bwd", "gated_bwd"])
def test_tensors_of_other_types(cdl, name):
    for t in (f32, bf16):
        call = python_calls(cdl, t)[name]
        with pytest.raises(cdl.CdlError) as e:
            call()
        assert e.value.status == PARAM
        import inspect
        names = inspect.getclosurevars(call).nonlocals["defaults"]
        for k in names:
            for bad in ([torch.float16, bf16, torch.float64, torch.int32] if k in VECTORS else [f32, bf16, torch.int16, torch.float8_e5m2] if k in BYTES else [f32, torch.int16] if k in SCALES
                        else [bf16 if t is f32 else f32, torch.float16]):
                if k in ("x", "g", "y") and bad in (f32, bf16) and name in ("layer_norm_fwd", "block8_gemm_act", "block8_gemm_gated") and k == ("x" if "norm" in name else "y"):
                    continue      # (it says what the type is)
                with pytest.raises(TypeError):
                    call(**{k: zeros(bad, 8, 128)})
        for k in names:
            if k not in VECTORS + BYTES + SCALES:
                with pytest.raises(ValueError):      # not contiguous
                    call(**{k: zeros(t, 8, 16)[:, ::2]})


WS_ = [(POINTER, A), (SIZE, 1 << 60), (POINTER, None)]


def c_product(M, N, K, y_type, act=GELU, sides=1):
    name = "cdl_block8_gemm_act" if sides == 1 else "cdl_block8_gemm_gated"
    tail = [(POINTER, A), (INT, act)] + [(POINTER, A)] * 3 if sides == 1 else [(POINTER, A), (POINTER, A), (INT, act)] + [(POINTER, A)] * 3
    return (name, [(POINTER, A)] * (2 + 2 * sides) + [(INT, v) for v in (M, N, K, E4M3, E4M3)] + tail + [(INT, y_type)] + WS_)


def way(launches):
    names = [l.name for l in launches]
    if "finish" in names[-1]:
        return "parts"
    assert len(launches) == 1
    if "thin" in names[0]:
        return "thin"
    shapes = {"wide": (2, 2, 4, 4, 2, 2), "pair": (2, 2, 2, 2, 2, 2), "small": (2, 2, 1, 1, 4, 4), "small gated": (2, 2, 2, 1, 3, 3)}
    return next(w.split()[0] for w, s in shapes.items() if "RingForm<%d, %d, %d, %d, %d, %d," % s in names[0] or "RingFormILi%dELi%dELi%dELi%dELi%dELi%dE" % s in names[0])


def test_ways_of_the_products(tmp_path):
    """Every way that a product can go is taken at sizes of the GPU tests."""
    import test_gpu_block8_act as gpu
    seen = {}
    for sides in (1, 2):
        for y_type in (F32, BF16):
            recorded = launch_recorder.record(tmp_path, [c_product(*size, y_type, act, sides) for size in gpu.SIZES for act in (NONE, GELU)])
            seen[sides, y_type] = {way(launches) for launches, _ in recorded}
            for launches, _ in recorded:
                assert all(l.grid[0] * l.threads < 1 << 32 for l in launches)
    assert seen[1, BF16] == seen[2, BF16] == seen[2, F32] == {"parts", "thin", "small", "pair", "wide"}
    assert seen[1, F32] == {"parts", "thin", "small", "pair"}


def test_scratch_is_asked_for_where_it_is_used(tmp_path, cdl):
    sizes = [(M, N, K) for M in (1, 16, 40, 100, 300, 1000, 5000, 70000) for N in (30, 400, 4096, 9000) for K in (100, 1000, 20000)]
    for sides, f in ((1, cdl.block8_gemm_act_workspace_bytes), (2, cdl.block8_gemm_gated_workspace_bytes)):
        for y_type in (F32, BF16):
            for act in (NONE, RELU, GELU, SILU):
                for size, (launches, _) in zip(sizes, launch_recorder.record(tmp_path, [c_product(*size, y_type, act, sides) for size in sizes])):
                    if way(launches) == "parts":
                        assert f(*size) >= sides * size[0] * size[1] * 4, size


@pytest.mark.parametrize("type_", [F32, BF16])
def test_largest_sizes(tmp_path, type_):
    """a grid holds fewer than 2^32 threads"""
    def norm(rows, cols, back):
        if back:
            return ("cdl_layer_norm_bwd", [(POINTER, A), (INT, type_), (POINTER, A), (POINTER, None), (POINTER, None), (INT, 0)] + [(POINTER, A)] * 4 + [(INT, rows), (INT, cols)] + [(POINTER, A)] * 3 + WS_)
        return ("cdl_layer_norm_fwd", [(POINTER, A), (INT, type_), (POINTER, A), (POINTER, A), (INT, rows), (INT, cols), (FLOAT, 0.5)] + [(POINTER, A)] * 5 + [(INT, 0), (POINTER, None)])

    def act(rows, cols):
        return ("cdl_act_bwd", [(POINTER, A), (INT, type_), (POINTER, A), (POINTER, None), (POINTER, None), (INT, 0), (INT, GELU), (INT, rows), (INT, cols)] + [(POINTER, A)] * 3 + WS_)
    calls = [norm(rows, cols, back) for rows, cols in ((1 << 30, 128), (1 << 29, 16384), (1, 16384)) for back in (False, True)]
    calls += [act(1 << 30, 1 << 14), act(1 << 20, 1 << 24), act(1, 1 << 24)]
    calls += [c_product(M, N, K, type_, sides=sides) for sides in (1, 2) for M, N, K in ((1 << 30, 1 << 14, 128), (1 << 14, 1 << 30, 128), (1, 1 << 30, 1 << 20), (1 << 30, 1, 128), (1 << 22, 1 << 22, 0))]
    for call, (launches, _) in zip(calls, launch_recorder.record(tmp_path, calls)):
        for l in launches:
            assert 0 < l.grid[0] < 1 << 31 and l.grid[1] <= 65535 and l.grid[0] * l.grid[1] * l.threads < 1 << 32, (call[0], l)
