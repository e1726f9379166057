"""The operators around a network trained and served in eight bits, as cases that can be timed and compared.

Four operators, each one pass as a training or serving program makes it:

  dropout   y = keep(x) * scale [+ add], the mask from a counter-based generator and never stored.  The backward pass is the
            same call on the gradient.
  quantize  a matrix into 8-bit floating point with one scale, a power of two, for each block of 128 entries of a row
            (activations, gradients) or each tile of 128 x 128 (weights), and the same of its transpose, which the backward
            products read.  A scale is stored as its exponent plus 127; values [rows][columns up to a multiple of 128],
            scales [blocks of columns][rows up to a multiple of 128], a tile's rows all with the tile's scale
  product   y[m,n] = sum over blocks of a_scale * b_scale * (sum over the block of a[m,k] * b[n,k]): the forward product of a
            layer, and on other operands its two backward products
  head      softmax cross entropy of a linear last layer over a large vocabulary: loss and log-sum of every token, and, in a
            training step, the gradients of the hidden states and of the vocabulary matrix

`own` false: the plain form, elementary torch operations in 32 bits; true: the calls of the library.  Tokens whose target is
negative are padding: no loss, no gradient.
"""
import math

import torch

own = False

BLOCK = 128
FORMATS = {"e4m3": (torch.float8_e4m3fn, 8), "e5m2": (torch.float8_e5m2, 15)}      # largest value 1.75 * 2 ** that
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _dropout(n, p, type, add):
    return {"kind": "dropout", "n": n, "p": p, "type": type, "add": add}


def _quantize(rows, cols, type, tiles, fmt="e4m3", both=True):
    return {"kind": "quantize", "rows": rows, "cols": cols, "type": type, "tiles": tiles, "format": fmt, "both": both}


def _product(M, N, K, tiles, out, fmt="e4m3"):
    return {"kind": "product", "M": M, "N": N, "K": K, "tiles": tiles, "out": out, "format": fmt}


def _head(T, V, D, type, train):
    return {"kind": "head", "T": T, "V": V, "D": D, "type": type, "train": train}


def listed():
    return [
        # the hidden units of a handful of tokens, an odd count of them: a launch and little else
        dict(_dropout(16 * 768 + 5, 0.1, "bf16", False), name="dropout_small"),
        # the activations of a transformer layer added to their residual, a full batch of tokens
        dict(_dropout(65536 * 768, 0.1, "bf16", True), name="dropout_residual"),
        # those activations into eight bits, rows for the forward product and columns for the weight gradient
        dict(_quantize(65536, 768, "bf16", False), name="quantize_activations"),
        # the weights of the up-projection of a transformer MLP, fp32 as the optimizer holds them
        dict(_quantize(3072, 768, "f32", True), name="quantize_weights"),
        # a few tokens through that layer at serving: the weights are read once, latency counts
        dict(_product(4, 3072, 768, True, "bf16"), name="product_few_tokens"),
        # the classifier of an ImageNet network: ragged widths
        dict(_product(1021, 1000, 520, True, "f32"), name="product_ragged"),
        # the up-projection over a full batch of tokens: the largest product
        dict(_product(65536, 3072, 768, True, "bf16"), name="product_forward"),
        # its weight gradient: few outputs, the contraction runs over the tokens, gradients in the wider-ranging format
        dict(_product(3072, 768, 65536, False, "f32", "e5m2"), name="product_weight_gradient"),
        # scoring of a few tokens against a vocabulary of odd size: the vocabulary matrix is read once
        dict(_head(16, 50021, 768, "bf16", False), name="head_score_few"),
        # a training step of a small model's last layer, everything in fp32, ragged token count
        dict(_head(1000, 32000, 768, "f32", True), name="head_train_f32"),
        # a training step of a middling model: odd vocabulary
        dict(_head(8192, 50021, 768, "bf16", True), name="head_train"),
        # a training step over a vocabulary whose logits alone would take gigabytes: the largest
        dict(_head(8192, 128000, 2048, "bf16", True), name="head_train_large"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Sizes over the logarithm of the range, ragged ones as often as whole tiles; never beyond the largest listed case."""
    kind = rng.choice(["dropout", "quantize", "product", "product", "head", "head"])
    type = rng.choice(["bf16", "bf16", "f32"])
    if kind == "dropout":
        return _dropout(_log_int(rng, 1, 65536 * 1536), rng.choice([0.0, 0.1, 0.25, round(rng.uniform(0.01, 0.9), 3)]), type, rng.random() < 0.5)
    if kind == "quantize":
        rows, cols = _log_int(rng, 1, 65536), _log_int(rng, 64, 8192)
        if rng.random() < 0.5:
            cols = (cols + 127) // 128 * 128
        rows = max(1, min(rows, 65536 * 1536 // cols))
        return _quantize(rows, cols, type, rng.random() < 0.4, rng.choice(["e4m3", "e4m3", "e5m2"]), rng.random() < 0.7)
    if kind == "product":
        M, N, K = _log_int(rng, 1, 65536), _log_int(rng, 16, 8192), _log_int(rng, 64, 8192)
        if rng.random() < 0.5:
            N, K = (N + 127) // 128 * 128, (K + 127) // 128 * 128
        M = max(1, min(M, 65536 * 3072 * 768 // (N * K), 65536 * 3072 // max(N, K)))
        if rng.random() < 0.25:      # the shape of a weight gradient
            M, N, K = N, K, M
        return _product(M, N, K, rng.random() < 0.6, rng.choice(["bf16", "f32"]), rng.choice(["e4m3", "e4m3", "e5m2"]))
    train = rng.random() < 0.7
    T, V, D = _log_int(rng, 1, 8192), _log_int(rng, 1000, 128000), _log_int(rng, 64, 4096)
    if rng.random() < 0.6:
        D = (D + 63) // 64 * 64
    most = (65536 if train else 131072) * 2 ** 22 if type == "f32" else 8192 * 128000 * 2048      # (fp32: six products for one)
    T = max(1, min(T, most // (V * D)))
    return _head(T, V, D, type, train)


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _activations(shape, gen):
    """Activations of a transformer: one entry in a hundred eight times as large."""
    x = torch.randn(shape, device="cuda", generator=gen)
    return torch.where(torch.rand(shape, device="cuda", generator=gen) < 0.01, x * 8.0, x)


def _blocks(n):
    return -(-n // BLOCK)


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"case": c}
    if c["kind"] == "dropout":
        n, t = c["n"], TYPES[c["type"]]
        s["x"] = torch.randn(n, device="cuda", generator=gen).to(t)
        s["add"] = torch.randn(n, device="cuda", generator=gen).to(t) if c["add"] else None
        s["key"], s["counter"] = (0x9E3779B97F4A7C15 * (seed + 1)) % 2 ** 63, 1000 * seed
        s["y"] = torch.empty_like(s["x"])
    elif c["kind"] == "quantize":
        rows, cols = c["rows"], c["cols"]
        x = torch.randn((rows, cols), device="cuda", generator=gen) * 0.02 if c["tiles"] else _activations((rows, cols), gen)
        s["x"] = x.to(TYPES[c["type"]])
        s["q"] = torch.empty((rows, _blocks(cols) * BLOCK), dtype=torch.uint8, device="cuda")
        s["scale"] = torch.empty((_blocks(cols), _blocks(rows) * BLOCK), dtype=torch.uint8, device="cuda")
        if c["both"]:
            s["q_t"] = torch.empty((cols, _blocks(rows) * BLOCK), dtype=torch.uint8, device="cuda")
            s["scale_t"] = torch.empty((_blocks(rows), _blocks(cols) * BLOCK), dtype=torch.uint8, device="cuda")
    elif c["kind"] == "product":
        M, N, K = c["M"], c["N"], c["K"]
        s["a"], s["a_scale"] = _plain_quantize(_activations((M, K), gen), c["format"], False)
        s["b"], s["b_scale"] = _plain_quantize(torch.randn((N, K), device="cuda", generator=gen) / math.sqrt(K), "e4m3", c["tiles"])
        s["y"] = torch.empty((M, N), dtype=TYPES[c["out"]], device="cuda")
        if own:
            import paper_2501_09849_amd as cdl
            s["ws"] = torch.empty(max(256, cdl.block8_gemm_workspace_bytes(M, N, K)), dtype=torch.uint8, device="cuda")
    else:
        T, V, D = c["T"], c["V"], c["D"]
        t = TYPES[c["type"]]
        s["h"] = torch.randn((T, D), device="cuda", generator=gen).to(t)
        s["w"] = (torch.randn((V, D), device="cuda", generator=gen) * (1.5 / math.sqrt(D))).to(t)
        target = torch.randint(0, V, (T,), device="cuda", generator=gen)
        s["target"] = torch.where(torch.rand(T, device="cuda", generator=gen) < 0.05, torch.full_like(target, -100), target)
        if c["train"]:      # the mean over the tokens that count
            s["d_loss"] = torch.full((T,), 1.0 / max(1, int((s["target"] >= 0).sum())), device="cuda")
        s["loss"], s["lse"] = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
        if own:
            import paper_2501_09849_amd as cdl
            kind = cdl.BF16 if c["type"] == "bf16" else cdl.F32
            s["ws"] = torch.empty(max(256, cdl.head_loss_workspace_bytes(T, V, D, kind, c["train"])), dtype=torch.uint8, device="cuda")
            if c["train"]:
                s["d_h"], s["d_w"] = torch.empty_like(s["h"]), torch.empty_like(s["w"])
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------

def run(state):
    return {"dropout": _run_dropout, "quantize": _run_quantize, "product": _run_product, "head": _run_head}[state["case"]["kind"]](state)


def _run_dropout(s):
    c = s["case"]
    if own:
        import paper_2501_09849_amd as cdl
        cdl.cdl_dropout(s["x"], c["n"], c["p"], s["key"], s["counter"], s["y"], add=s["add"])
        return s["y"]
    share = round(c["p"] * 65536)
    y = s["x"].float() * (65536.0 / (65536 - share))
    y = torch.where(_plain_halves(c["n"], s["key"], s["counter"]) >= share, y, torch.zeros_like(y))
    return (y if s["add"] is None else y + s["add"].float()).to(s["x"].dtype)


def _run_quantize(s):
    c = s["case"]
    if own:
        import paper_2501_09849_amd as cdl
        fmt = cdl.E4M3 if c["format"] == "e4m3" else cdl.E5M2
        cdl.cdl_block8_quantize(s["x"], c["rows"], c["cols"], s["q"], s["scale"], s.get("q_t"), s.get("scale_t"), tiles=c["tiles"], format=fmt)
        kind = FORMATS[c["format"]][0]
        out = [s["q"].view(kind), s["scale"]]
        return out + [s["q_t"].view(kind), s["scale_t"]] if c["both"] else out
    x = s["x"].float()
    out = [*_plain_quantize(x, c["format"], c["tiles"])]
    return out + [*_plain_quantize(x.t().contiguous(), c["format"], c["tiles"])] if c["both"] else out


def _run_product(s):
    c = s["case"]
    if own:
        import paper_2501_09849_amd as cdl
        fmt = cdl.E4M3 if c["format"] == "e4m3" else cdl.E5M2
        cdl.cdl_block8_gemm(s["a"], s["a_scale"], s["b"], s["b_scale"], c["M"], c["N"], c["K"], s["y"], s["ws"], a_format=fmt)
        return s["y"]
    return (_plain_values(s["a"], s["a_scale"]) @ _plain_values(s["b"], s["b_scale"]).t()).to(TYPES[c["out"]])


def _run_head(s):
    c = s["case"]
    T, V, D = c["T"], c["V"], c["D"]
    if own:
        import paper_2501_09849_amd as cdl
        cdl.cdl_head_loss_fwd(s["h"], s["w"], s["target"], T, V, D, s["loss"], s["lse"], s["ws"])
        if not c["train"]:
            return [s["loss"], s["lse"]]
        cdl.cdl_head_loss_bwd(s["h"], s["w"], s["target"], s["lse"], T, V, D, s["d_h"], s["d_w"], s["ws"], d_loss=s["d_loss"])
        return [s["loss"], s["lse"], s["d_h"], s["d_w"]]
    h, w, counts = s["h"].float(), s["w"].float(), s["target"] >= 0
    at = s["target"].clamp(min=0)[:, None]
    z = h @ w.t()
    top = z.max(dim=1, keepdim=True).values
    e = torch.exp(z - top)
    total = e.sum(dim=1, keepdim=True)
    lse = (top + torch.log(total))[:, 0]
    loss = torch.where(counts, lse - z.gather(1, at)[:, 0], torch.zeros_like(lse))
    if not c["train"]:
        return [loss, lse]
    del z
    g = torch.where(counts, s["d_loss"], torch.zeros_like(lse))[:, None]
    e *= g / total
    e.scatter_add_(1, at, -g)
    return [loss, lse, (e @ w).to(s["h"].dtype), (e.t() @ h).to(s["w"].dtype)]


# ---- plain forms ----------------------------------------------------------------------------------------------------

def _plain_halves(n, key, counter):
    """16 random bits for each of n entries: eight entries share a counter's four words of Philox 4x32 with ten rounds, two a word, low half first."""
    i = torch.arange(-(-n // 8), device="cuda") + counter
    m = 0xFFFFFFFF
    x = [i & m, i >> 32 & m, torch.zeros_like(i), torch.zeros_like(i)]
    k0, k1 = key & m, key >> 32 & m
    for _ in range(10):
        p, q = x[0] * 0xD2511F53, x[2] * 0xCD9E8D57
        x = [(q >> 32 & m) ^ x[1] ^ k0, q & m, (p >> 32 & m) ^ x[3] ^ k1, p & m]
        k0, k1 = k0 + 0x9E3779B9 & m, k1 + 0xBB67AE85 & m
    words = torch.stack(x, dim=1)
    return torch.stack([words & 0xFFFF, words >> 16], dim=2).reshape(-1)[:n]


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
    return q.float() * by.t().repeat_interleave(BLOCK, dim=1)


def _power(exponent):
    """2 ** exponent, exactly, for exponents from -126 to 127."""
    return ((exponent + 127) << 23).int().view(torch.float32)


# ---- what the work cannot do without ----------------------------------------------------------------------------------

def work(case):
    c = dict(case)
    size = {"f32": 4, "bf16": 2}
    if c["kind"] == "dropout":
        return {"bytes": c["n"] * size[c["type"]] * (3 if c["add"] else 2), "flops": 2 * c["n"]}
    if c["kind"] == "quantize":
        n = c["rows"] * c["cols"]
        return {"bytes": n * (size[c["type"]] + (2 if c["both"] else 1)), "flops": 3 * n}
    if c["kind"] == "product":
        M, N, K = c["M"], c["N"], c["K"]
        scales = _blocks(K) * (M + (_blocks(N) if c["tiles"] else N))
        return {"bytes": M * K + N * K + scales + M * N * size[c["out"]], "flops": 2 * M * N * K}
    T, V, D = c["T"], c["V"], c["D"]
    ends = (T * D + V * D) * size[c["type"]]
    return {"bytes": ends * (2 if c["train"] else 1) + 16 * T, "flops": 2 * T * V * D * (3 if c["train"] else 1)}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------

def exact(case, seed):
    c = dict(case)
    s = prepare(case, seed)
    if c["kind"] == "dropout":
        return _exact_dropout(c, s)
    if c["kind"] == "quantize":
        x = s["x"].double()
        out = [*_exact_quantize(x, c)]
        return out + [*_exact_quantize(x.t(), c)] if c["both"] else out
    if c["kind"] == "product":
        y = torch.zeros((c["M"], c["N"]), dtype=torch.float64, device="cuda")
        step = BLOCK * max(1, _blocks(c["K"]) // 16)
        for k in range(0, c["K"], step):      # a stretch of blocks at a time
            block = torch.arange(k, min(k + step, s["a"].shape[1]), device="cuda") // BLOCK
            a = torch.ldexp(s["a"][:, k:k + step].double(), s["a_scale"].t()[: c["M"], block].int() - 127)
            b = torch.ldexp(s["b"][:, k:k + step].double(), s["b_scale"].t()[: c["N"], block].int() - 127)
            y += a @ b.t()
        return y
    return _exact_head(c, s)


def _exact_dropout(c, s):
    """The generator by products of 16-bit halves, entry by entry."""
    e = torch.arange(c["n"], device="cuda")
    ctr = e // 8 + s["counter"]
    low, high, m = 0xFFFF, lambda v: v >> 16, 0xFFFFFFFF

    def product(v, by):      # (high, low) words of the 64-bit product of two 32-bit numbers
        a, b, u, w = high(v), v & low, by >> 16, by & low
        mid = a * w + high(b * w)
        cross = b * u + (mid & low)
        return a * u + high(mid) + high(cross), ((cross & low) << 16) | (b * w & low)

    w0, w1, w2, w3 = ctr & m, high(high(ctr)) & m, torch.zeros_like(ctr), torch.zeros_like(ctr)
    for r in range(10):
        k0, k1 = (s["key"] + r * 0x9E3779B9) & m, ((s["key"] >> 32) + r * 0xBB67AE85) & m
        (h0, l0), (h2, l2) = product(w0, 0xD2511F53), product(w2, 0xCD9E8D57)
        w0, w1, w2, w3 = h2 ^ w1 ^ k0, l2, h0 ^ w3 ^ k1, l0
    which = e % 8 // 2
    word = torch.where(which == 0, w0, torch.where(which == 1, w1, torch.where(which == 2, w2, w3)))
    bits = torch.where(e % 2 == 0, word & low, high(word))
    share = round(c["p"] * 65536)
    y = torch.where(bits >= share, s["x"].double() * 65536.0 / max(1, 65536 - share), 0.0)
    return y + s["add"].double() if c["add"] else y


def _exact_quantize(x, c):
    kind, top = FORMATS[c["format"]]
    rows, cols = x.shape
    full = torch.zeros((_blocks(rows) * BLOCK, _blocks(cols) * BLOCK), dtype=torch.float64, device="cuda")
    full[:rows, :cols] = x
    size = full.abs().unflatten(1, (-1, BLOCK)).amax(dim=2)
    if c["tiles"]:
        size = size.unflatten(0, (-1, BLOCK)).amax(dim=1).repeat_interleave(BLOCK, dim=0)
    power = torch.ceil(torch.log2(size / (1.75 * 2.0 ** top))).clamp(min=-100)
    power += (size > 1.75 * torch.exp2(power + top)).double() - (size <= 1.75 * torch.exp2(power + top - 1)).double() * (power > -100)      # (where the logarithm rounds across a whole number)
    full /= torch.exp2(power).repeat_interleave(BLOCK, dim=1)
    return full[:rows].to(kind).double(), (power + 127).t().to(torch.uint8)


def _exact_head(c, s):
    h, w = s["h"].double(), s["w"].double()
    ok = s["target"] >= 0
    loss, lse = torch.zeros(c["T"], dtype=torch.float64, device="cuda"), torch.zeros(c["T"], dtype=torch.float64, device="cuda")
    d_h, d_w = torch.zeros_like(h), torch.zeros_like(w)
    for t in range(0, c["T"], 2048):      # some tokens at a time
        part = slice(t, t + 2048)
        logits = h[part] @ w.t()
        lse[part] = torch.logsumexp(logits, dim=1)
        hit = torch.nn.functional.one_hot(s["target"][part].clamp(min=0), c["V"]).bool() & ok[part][:, None]
        loss[part] = torch.where(ok[part], lse[part], 0.0) - (logits * hit).sum(dim=1)
        if c["train"]:
            g = (torch.exp(logits - lse[part][:, None]) - hit.double()) * (s["d_loss"][part].double() * ok[part])[:, None]
            d_h[part] = g @ w
            d_w += g.t() @ h[part]
    return [loss, lse, d_h, d_w] if c["train"] else [loss, lse]
