"""The feed-forward sublayer of a network in eight bits, operator by operator, as cases that can be timed and compared.

Each case is one pass as a training or serving program makes it:

  norm       layer norm of the rows of x; forward also their copy in 8-bit floating point that the backward pass reads in the place of
             x.  Backward: the gradient of x, added to the one that comes along the residual, and those of weight and bias
  act        a block-scaled product with what stands behind it: z = a b^T + bias, y = act(z) + residual.  Backward: the gradient
             of z, and of the bias
  gated      both projections of a gated feed-forward block, the activation and the product: y = act(a g^T + bias) * (a u^T + bias).  Backward:
             the gradients of both projections' results, and of both biases

Matrices in 8-bit floating point have a scale, a power of two, for each block of 128 entries of a row, stored as its exponent plus 127: values
[rows][columns up to a multiple of 128], scales [blocks of columns][rows up to a multiple of 128].  Where a case keeps its
activations in eight bits, the backward pass reads them so.

`own` false: the plain form, elementary torch operations in 32 bits; true: the calls of the library.
"""
import math

import torch

own = False

BLOCK = 128
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}
FORMATS = {"e4m3": (torch.float8_e4m3fn, 8), "e5m2": (torch.float8_e5m2, 15)}      # largest value 1.75 * 2 ** that
ACTS = ("none", "relu", "gelu", "silu")
EPS = 1e-5


def _norm(rows, cols, type, back, kept):
    return {"kind": "norm", "rows": rows, "cols": cols, "type": type, "back": back, "kept": kept}


def _act(M, N, K, type, act, residual, keep):
    return {"kind": "act", "M": M, "N": N, "K": K, "type": type, "act": act, "residual": residual, "keep": keep}


def _act_back(rows, cols, type, act, kept):
    return {"kind": "act_back", "rows": rows, "cols": cols, "type": type, "act": act, "kept": kept}


def _gated(M, N, K, type, act, keep):
    return {"kind": "gated", "M": M, "N": N, "K": K, "type": type, "act": act, "keep": keep}


def _gated_back(rows, cols, type, act, kept):
    return {"kind": "gated_back", "rows": rows, "cols": cols, "type": type, "act": act, "kept": kept}


def listed():
    return [
        # the states of a few tokens at serving: a launch and little else
        dict(_norm(4, 1024, "bf16", False, False), name="norm_few_tokens"),
        # a full batch of tokens of a transformer layer, their states kept in eight bits for the backward pass
        dict(_norm(65536, 768, "bf16", False, True), name="norm_keep"),
        # its backward pass from those eight bits, onto the gradient along the residual
        dict(_norm(65536, 768, "bf16", True, True), name="norm_back_kept"),
        # a small model in fp32 throughout, odd sizes, states kept as they are
        dict(_norm(4099, 1021, "f32", True, False), name="norm_back_ragged"),
        # the up-projection of a few tokens at serving: the weights are read once, latency counts
        dict(_act(4, 4096, 1024, "bf16", "gelu", False, False), name="act_few_tokens"),
        # the down-projection over a full batch of tokens, onto the residual
        dict(_act(65536, 768, 2048, "bf16", "none", True, False), name="act_residual"),
        # a layer in fp32 with odd widths, its z kept for the backward pass
        dict(_act(1021, 1000, 520, "f32", "gelu", False, True), name="act_ragged"),
        # the backward pass of an up-projection's activation over a full batch of tokens
        dict(_act_back(65536, 2048, "bf16", "gelu", False), name="act_back"),
        # one token through a gated block at serving
        dict(_gated(1, 2048, 768, "bf16", "silu", False), name="gated_one_token"),
        # a full batch of tokens in training, both projections' results kept: the largest
        dict(_gated(65536, 2048, 768, "bf16", "silu", True), name="gated_keep"),
        # odd sizes in fp32
        dict(_gated(999, 1365, 520, "f32", "gelu", True), name="gated_ragged"),
        # the backward pass of the gated block, the projections' results kept in eight bits
        dict(_gated_back(65536, 2048, "bf16", "silu", True), name="gated_back_kept"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Sizes over the logarithm of the range, ragged ones as often as whole ones; never beyond the largest listed case."""
    kind = rng.choice(["norm", "norm", "act", "act", "act_back", "gated", "gated", "gated_back"])
    type = rng.choice(["bf16", "bf16", "f32"])
    if kind == "norm":
        rows, cols = _log_int(rng, 1, 65536), _log_int(rng, 16, 16384)
        if rng.random() < 0.5:
            cols = (cols + 63) // 64 * 64
        rows = max(1, min(rows, 65536 * 768 // cols))
        return _norm(rows, cols, type, rng.random() < 0.6, rng.random() < 0.5)
    act = rng.choice(ACTS)
    if kind in ("act_back", "gated_back"):
        rows, cols = _log_int(rng, 1, 65536), _log_int(rng, 16, 16384)
        if rng.random() < 0.5:
            cols = (cols + 63) // 64 * 64
        rows = max(1, min(rows, 65536 * 1024 // cols))
        return (_act_back if kind == "act_back" else _gated_back)(rows, cols, type, act, rng.random() < 0.5)
    M, N, K = _log_int(rng, 1, 65536), _log_int(rng, 16, 8192), _log_int(rng, 64, 8192)
    if rng.random() < 0.5:
        N, K = (N + 127) // 128 * 128, (K + 127) // 128 * 128
    M = max(1, min(M, 65536 * 2048 * 768 // (2 * N * K) if type == "f32" else 65536 * 2048 * 768 // (N * K), 65536 * 2048 // max(N, K)))
    if kind == "act":
        return _act(M, N, K, type, act, rng.random() < 0.5, rng.random() < 0.4)
    return _gated(M, N, K, type, act, rng.random() < 0.5)


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _blocks(n):
    return -(-n // BLOCK)


def _states(shape, gen):
    """States of a transformer: rows of their own size and mean, one entry in a hundred eight times as large."""
    x = torch.randn(shape, device="cuda", generator=gen)
    x = torch.where(torch.rand(shape, device="cuda", generator=gen) < 0.01, x * 8.0, x)
    row = torch.randn((shape[0], 2), device="cuda", generator=gen)
    return x * torch.exp2(row[:, :1]) + 0.5 * row[:, 1:]


def _randn(shape, gen, by=1.0):
    return torch.randn(shape, device="cuda", generator=gen) * by


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"case": c}
    t = TYPES[c["type"]]
    if c["kind"] == "norm":
        rows, cols = c["rows"], c["cols"]
        x = _states((rows, cols), gen).to(t)
        s["weight"], s["bias"] = 1.0 + _randn(cols, gen, 0.1), _randn(cols, gen, 0.1)
        if not c["back"]:
            s["x"], s["y"] = x, torch.empty_like(x)
            s["mean"], s["rstd"] = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
            if c["kept"]:
                s["q"], s["scale"] = _empty8(rows, cols)
            return s
        wide = x.double()
        mean = wide.mean(dim=1)
        s["mean"], s["rstd"] = mean.float(), torch.rsqrt((wide - mean[:, None]).square().mean(dim=1) + EPS).float()
        if c["kept"]:
            s["q"], s["scale"] = _plain_quantize(x.float(), "e4m3", False)
        else:
            s["x"] = x
        s["g"], s["add"] = _randn((rows, cols), gen, 2.0 ** -10).to(t), _randn((rows, cols), gen, 2.0 ** -9).to(t)
        s["d_x"] = torch.empty((rows, cols), dtype=t, device="cuda")
        s["d_weight"], s["d_bias"] = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
        if own:
            import paper_2501_09849_amd as cdl
            s["ws"] = torch.empty(max(256, cdl.layer_norm_bwd_workspace_bytes(rows, cols)), dtype=torch.uint8, device="cuda")
    elif c["kind"] in ("act_back", "gated_back"):
        rows, cols = c["rows"], c["cols"]
        s["g"] = _randn((rows, cols), gen, 2.0 ** -10).to(t)
        for side in _sides(c):
            z = _randn((rows, cols), gen, 1.5).to(t)
            if c["kept"]:
                s["q" + side], s["scale" + side] = _plain_quantize(z.float(), "e4m3", False)
            else:
                s["z" + side] = z
            s["d" + side], s["d_bias" + side] = torch.empty((rows, cols), dtype=t, device="cuda"), torch.empty(cols, device="cuda")
        if own:
            import paper_2501_09849_amd as cdl
            need = cdl.act_bwd_workspace_bytes(rows, cols) if c["kind"] == "act_back" else cdl.gated_bwd_workspace_bytes(rows, cols)
            s["ws"] = torch.empty(max(256, need), dtype=torch.uint8, device="cuda")
    else:
        M, N, K = c["M"], c["N"], c["K"]
        x = _randn((M, K), gen)
        s["a"], s["a_scale"] = _plain_quantize(torch.where(torch.rand((M, K), device="cuda", generator=gen) < 0.01, x * 8.0, x), "e4m3", False)
        for side in _sides(c):
            s["b" + side], s["b_scale" + side] = _plain_quantize(_randn((N, K), gen, K ** -0.5), "e4m3", True)
            s["bias" + side] = _randn(N, gen, 0.1)
            if c["keep"]:
                s["z" + side] = torch.empty((M, N), dtype=t, device="cuda")
        s["y"] = torch.empty((M, N), dtype=t, device="cuda")
        s["add"] = _randn((M, N), gen).to(t) if c.get("residual") else None
        if own:
            import paper_2501_09849_amd as cdl
            need = cdl.block8_gemm_act_workspace_bytes(M, N, K) if c["kind"] == "act" else cdl.block8_gemm_gated_workspace_bytes(M, N, K)
            s["ws"] = torch.empty(max(256, need), dtype=torch.uint8, device="cuda")
    return s


def _sides(c):
    return ("_gate", "_up") if c["kind"].startswith("gated") else ("",)


def _empty8(rows, cols):
    return (torch.empty((rows, _blocks(cols) * BLOCK), dtype=torch.uint8, device="cuda"),
            torch.empty((_blocks(cols), _blocks(rows) * BLOCK), dtype=torch.uint8, device="cuda"))


# ---- one pass -------------------------------------------------------------------------------------------------------

def run(state):
    return {"norm": _run_norm, "act": _run_act, "act_back": _run_act_back, "gated": _run_gated, "gated_back": _run_gated_back}[state["case"]["kind"]](state)


def _run_norm(s):
    c = s["case"]
    rows, cols = c["rows"], c["cols"]
    if own:
        import paper_2501_09849_amd as cdl
        if c["back"]:
            cdl.cdl_layer_norm_bwd(s["g"], rows, cols, s["mean"], s["rstd"], d_x=s["d_x"], d_weight=s["d_weight"], d_bias=s["d_bias"], x=s.get("x"), q=s.get("q"),
                                   scale=s.get("scale"), weight=s["weight"], add=s["add"], ws=s["ws"])
            return [s["d_x"], s["d_weight"], s["d_bias"]]
        cdl.cdl_layer_norm_fwd(s["x"], rows, cols, s["y"], s["mean"], s["rstd"], weight=s["weight"], bias=s["bias"], eps=EPS, q=s.get("q"), scale=s.get("scale"))
        out = [s["y"], s["mean"], s["rstd"]]
        return out + [s["q"].view(FORMATS["e4m3"][0]), s["scale"]] if c["kept"] else out
    if c["back"]:
        x, g = _plain_values(s["q"], s["scale"])[:, :cols] if c["kept"] else s["x"].float(), s["g"].float()
        n = (x - s["mean"][:, None]) * s["rstd"][:, None]
        h = g * s["weight"]
        d_x = (h - h.mean(dim=1, keepdim=True) - n * (h * n).mean(dim=1, keepdim=True)) * s["rstd"][:, None] + s["add"].float()
        return [d_x.to(s["g"].dtype), (g * n).sum(dim=0), g.sum(dim=0)]
    x = s["x"].float()
    mean = x.mean(dim=1, keepdim=True)
    n = x - mean
    rstd = 1.0 / torch.sqrt(n.square().mean(dim=1, keepdim=True) + EPS)
    out = [(n * rstd * s["weight"] + s["bias"]).to(s["x"].dtype), mean[:, 0], rstd[:, 0]]
    return out + [*_plain_quantize(x, "e4m3", False)] if c["kept"] else out


def _run_act(s):
    c = s["case"]
    if own:
        import paper_2501_09849_amd as cdl
        cdl.cdl_block8_gemm_act(s["a"], s["a_scale"], s["b"], s["b_scale"], c["M"], c["N"], c["K"], s["y"], z=s.get("z"), bias=s["bias"], act=_number(c["act"]), add=s["add"],
                                ws=s["ws"])
        return [s["y"], s["z"]] if c["keep"] else [s["y"]]
    t = s["y"].dtype
    z = _plain_values(s["a"], s["a_scale"]) @ _plain_values(s["b"], s["b_scale"]).t() + s["bias"]
    y = _plain_act(c["act"], z)[0]
    if s["add"] is not None:
        y = y + s["add"].float()
    return [y.to(t), z.to(t)] if c["keep"] else [y.to(t)]


def _run_gated(s):
    c = s["case"]
    if own:
        import paper_2501_09849_amd as cdl
        cdl.cdl_block8_gemm_gated(s["a"], s["a_scale"], s["b_gate"], s["b_scale_gate"], s["b_up"], s["b_scale_up"], c["M"], c["N"], c["K"], s["y"], z_gate=s.get("z_gate"),
                                  z_up=s.get("z_up"), bias_gate=s["bias_gate"], bias_up=s["bias_up"], act=_number(c["act"]), ws=s["ws"])
        return [s["y"], s["z_gate"], s["z_up"]] if c["keep"] else [s["y"]]
    t, a = s["y"].dtype, _plain_values(s["a"], s["a_scale"])
    gate = a @ _plain_values(s["b_gate"], s["b_scale_gate"]).t() + s["bias_gate"]
    up = a @ _plain_values(s["b_up"], s["b_scale_up"]).t() + s["bias_up"]
    y = (_plain_act(c["act"], gate)[0] * up).to(t)
    return [y, gate.to(t), up.to(t)] if c["keep"] else [y]


def _run_act_back(s):
    c = s["case"]
    if own:
        import paper_2501_09849_amd as cdl
        cdl.cdl_act_bwd(s["g"], c["rows"], c["cols"], _number(c["act"]), d_z=s["d"], d_bias=s["d_bias"], z=s.get("z"), q=s.get("q"), scale=s.get("scale"), ws=s["ws"])
        return [s["d"], s["d_bias"]]
    d = s["g"].float() * _plain_act(c["act"], _plain_kept(s, ""))[1]
    return [d.to(s["g"].dtype), d.sum(dim=0)]


def _run_gated_back(s):
    c = s["case"]
    if own:
        import paper_2501_09849_amd as cdl
        cdl.cdl_gated_bwd(s["g"], c["rows"], c["cols"], _number(c["act"]), d_gate=s["d_gate"], d_up=s["d_up"], d_bias_gate=s["d_bias_gate"], d_bias_up=s["d_bias_up"],
                          z_gate=s.get("z_gate"), z_up=s.get("z_up"), q_gate=s.get("q_gate"), scale_gate=s.get("scale_gate"), q_up=s.get("q_up"), scale_up=s.get("scale_up"), ws=s["ws"])
        return [s["d_gate"], s["d_up"], s["d_bias_gate"], s["d_bias_up"]]
    g, t = s["g"].float(), s["g"].dtype
    value, slope = _plain_act(c["act"], _plain_kept(s, "_gate"))
    d_gate, d_up = g * _plain_kept(s, "_up") * slope, g * value
    return [d_gate.to(t), d_up.to(t), d_gate.sum(dim=0), d_up.sum(dim=0)]


def _number(act):
    import paper_2501_09849_amd as cdl
    return {"none": cdl.ACT_NONE, "relu": cdl.ACT_RELU, "gelu": cdl.ACT_GELU, "silu": cdl.ACT_SILU}[act]


# ---- plain forms ----------------------------------------------------------------------------------------------------

def _plain_act(act, z):
    """(value, derivative)"""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z)), (z > 0).float()
    if act == "gelu":
        share = 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5)))
        return z * share, share + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    share = 1.0 / (1.0 + torch.exp(-z))
    return z * share, share * (1.0 + z * (1.0 - share))


def _plain_quantize(x, fmt, tiles):
    """(values, scales) of x in 32 bits: the smallest scale under which the largest magnitude is no larger than the format's, 2 ** -100 at least."""
    kind, top = FORMATS[fmt]
    rows, cols = x.shape
    p = torch.nn.functional.pad(x, (0, -cols % BLOCK, 0, -rows % BLOCK)).reshape(_blocks(rows), BLOCK, _blocks(cols), BLOCK)
    largest = p.abs().amax(dim=(1, 3) if tiles else 3, keepdim=True)
    fraction, exponent = torch.frexp(largest)      # largest = fraction * 2 ** exponent, fraction in [0.5, 1)
    exponent = torch.where(largest > 0, exponent - 1 - top + (fraction > 0.875).int(), -100).clamp(min=-100)
    q = (p * _power(-exponent)).to(kind)
    scale = (exponent + 127).to(torch.uint8).expand(-1, BLOCK, -1, -1).reshape(-1, _blocks(cols)).t().contiguous()
    return q.reshape(-1, _blocks(cols) * BLOCK)[:rows].contiguous(), scale


def _plain_values(q, scale):
    by = _power(scale[:, : q.shape[0]].int() - 127)
    return (q.float().reshape(q.shape[0], -1, BLOCK) * by.t()[:, :, None]).reshape(q.shape)


def _plain_kept(s, side):
    return s["z" + side].float() if "z" + side in s else _plain_values(s["q" + side], s["scale" + side])[:, : s["case"]["cols"]]


def _power(exponent):
    """2 ** exponent, exactly, for exponents from -126 to 127."""
    return ((exponent + 127) << 23).int().view(torch.float32)


# ---- what the work cannot do without ----------------------------------------------------------------------------------

def work(case):
    c = dict(case)
    size = SIZE[c["type"]]
    if c["kind"] == "norm":
        n = c["rows"] * c["cols"]
        kept = 1 + 1 / BLOCK
        if c["back"]:
            return {"bytes": n * (3 * size + (kept if c["kept"] else size)) + 8 * c["rows"] + 12 * c["cols"], "flops": 14 * n}
        return {"bytes": n * (2 * size + (kept if c["kept"] else 0)) + 8 * c["rows"] + 8 * c["cols"], "flops": 8 * n}
    sides = len(_sides(c))
    if c["kind"] in ("act_back", "gated_back"):
        n = c["rows"] * c["cols"]
        kept = 1 + 1 / BLOCK if c["kept"] else size
        return {"bytes": n * (size + sides * (kept + size)) + 4 * sides * c["cols"], "flops": 12 * n}
    M, N, K = c["M"], c["N"], c["K"]
    operands = M * K + _blocks(K) * M + sides * (N * K + _blocks(K) * _blocks(N) + 4 * N)
    results = M * N * size * (1 + (1 if c.get("residual") else 0) + (sides if c["keep"] else 0))
    return {"bytes": operands + results, "flops": 2 * sides * M * N * K}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------

def exact(case, seed):
    c = dict(case)
    s = prepare(case, seed)
    if c["kind"] == "norm":
        return _exact_norm(c, s)
    if c["kind"] in ("act_back", "gated_back"):
        g = s["g"].double()
        if c["kind"] == "act_back":
            d = [g * _exact_slope(c["act"], _exact_kept(s, ""))]
        else:
            gate, up = _exact_kept(s, "_gate"), _exact_kept(s, "_up")
            d = [_exact_slope(c["act"], gate) * up * g, _exact_value(c["act"], gate) * g]
        return d + [v.sum(dim=0) for v in d]
    a = _exact_values(s["a"], s["a_scale"])
    z = [torch.addmm(s["bias" + side].double(), a, _exact_values(s["b" + side], s["b_scale" + side]).t()) for side in _sides(c)]
    y = _exact_value(c["act"], z[0])
    if c["kind"] == "gated":
        y = y * z[1]
    elif s["add"] is not None:
        y = y + s["add"].double()
    return [y, *z] if c["keep"] else [y]


def _exact_values(q, scale):
    block = torch.arange(q.shape[1], device="cuda") // BLOCK
    return torch.ldexp(q.double(), scale.t()[: q.shape[0], block].int() - 127)


def _exact_kept(s, side):
    return s["z" + side].double() if "z" + side in s else _exact_values(s["q" + side], s["scale" + side])[:, : s["case"]["cols"]]


def _exact_value(act, z):
    if act == "gelu":
        return 0.5 * z * torch.erfc(-z / math.sqrt(2.0))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z.clamp(min=0.0) if act == "relu" else z


def _exact_slope(act, z):
    if act == "gelu":
        return 0.5 * torch.erfc(-z / math.sqrt(2.0)) + z * torch.exp(-z * z / 2.0) / math.sqrt(2.0 * math.pi)
    if act == "silu":
        return torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z)
    return (z > 0).double() if act == "relu" else torch.ones_like(z)


def _exact_norm(c, s):
    if c["back"]:
        x = _exact_values(s["q"], s["scale"])[:, : c["cols"]] if c["kept"] else s["x"].double()
        g, rstd = s["g"].double(), s["rstd"].double()[:, None]
        n = (x - s["mean"].double()[:, None]) * rstd
        h = g * s["weight"].double()
        one, two = h.sum(dim=1, keepdim=True), (h * n).sum(dim=1, keepdim=True)
        return [s["add"].double() + rstd * (h - (one + n * two) / c["cols"]), (g * n).sum(dim=0), g.sum(dim=0)]
    x = s["x"].double()
    var, mean = torch.var_mean(x, dim=1, correction=0)
    rstd = (var + EPS).rsqrt()
    out = [torch.addcmul(s["bias"].double(), (x - mean[:, None]) * rstd[:, None], s["weight"].double()), mean, rstd]
    if not c["kept"]:
        return out
    kind, top = FORMATS["e4m3"]
    full = torch.zeros((_blocks(c["rows"]) * BLOCK, _blocks(c["cols"]) * BLOCK), dtype=torch.float64, device="cuda")
    full[: c["rows"], : c["cols"]] = x
    size = full.unflatten(1, (-1, BLOCK)).abs().amax(dim=2)
    power = torch.ceil(torch.log2(size / (1.75 * 2.0 ** top))).clamp(min=-100)
    power += (size > 1.75 * torch.exp2(power + top)).double() - (size <= 1.75 * torch.exp2(power + top - 1)).double() * (power > -100)      # (where the logarithm rounds across a whole number)
    full /= torch.exp2(power).repeat_interleave(BLOCK, dim=1)
    return out + [full[: c["rows"]].to(kind).double(), (power + 127).t().to(torch.uint8)]
