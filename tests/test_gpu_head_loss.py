"""Cross entropy of a linear last layer over a vocabulary, forward and backward, against the formulas in 64 bits and against differences."""
import numpy as np
import pytest

import gpu_util as gu

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def env():
    import paper_2501_09849_amd as cdl
    return gu.torch_mod(), cdl


class Case:
    """inputs, one forward and backward call, the formulas in 64 bits with bounds on what rounding may do"""

    def __init__(self, env, T, V, D, type_, seed=0, padding=0.1, spread=1.5, with_lse=False, target=None, h=None, w=None):
        self.torch, self.cdl = torch, cdl = env
        self.T, self.V, self.D, self.type = T, V, D, getattr(torch, type_)
        gen = torch.Generator(device="cuda").manual_seed(1000 * seed + T + 3 * V + 7 * D)
        self.h = (torch.randn((T, D), device="cuda", generator=gen) if h is None else h).to(self.type)
        self.w = (torch.randn((V, D), device="cuda", generator=gen) * spread / max(1, D) ** 0.5 if w is None else w).to(self.type)
        t = torch.randint(0, V, (T,), device="cuda", generator=gen)
        if target is None:
            # some padding, by -100, by V and by numbers far out
            out = torch.tensor([-100, -1, V, V + 5, 2 ** 40, -2 ** 62], device="cuda")[torch.randint(0, 6, (T,), device="cuda", generator=gen)]
            t = torch.where(torch.rand(T, device="cuda", generator=gen) < padding, out, t)
        else:
            t = target
        self.target = t
        self.d_loss = torch.rand(T, device="cuda", generator=gen) + 0.25
        self.d_lse = torch.randn(T, device="cuda", generator=gen) * 0.2 if with_lse else None

    def scratch(self, train):
        kind = self.cdl.BF16 if self.type == self.torch.bfloat16 else self.cdl.F32
        n = self.cdl.head_loss_workspace_bytes(self.T, self.V, self.D, kind, train)
        return self.torch.full((max(256, n),), 0xff, dtype=self.torch.uint8, device="cuda")      # (NaN wherever something is read that was not written)

    def forward(self, h=None):
        torch = self.torch
        loss, lse = torch.full((self.T,), float("nan"), device="cuda"), torch.full((self.T,), float("nan"), device="cuda")
        self.cdl.cdl_head_loss_fwd(self.h if h is None else h, self.w, self.target, self.T, self.V, self.D, loss, lse, self.scratch(False))
        torch.cuda.synchronize()
        return loss, lse

    def backward(self, lse, want_h=True, want_w=True):
        torch = self.torch
        d_h = torch.full_like(self.h, float("nan")) if want_h else None
        d_w = torch.full_like(self.w, float("nan")) if want_w else None
        self.cdl.cdl_head_loss_bwd(self.h, self.w, self.target, lse, self.T, self.V, self.D, d_h, d_w, self.scratch(True), d_loss=self.d_loss, d_lse=self.d_lse)
        torch.cuda.synchronize()
        return d_h, d_w

    def check(self):
        torch = self.torch
        h, w = self.h.double(), self.w.double()
        T, V, D = self.T, self.V, self.D
        ok = (self.target >= 0) & (self.target < V)
        at = torch.where(ok, self.target, 0)
        z, size = h @ w.t(), h.abs() @ w.abs().t()
        lse = torch.logsumexp(z, dim=1)
        zt = z.gather(1, at[:, None])[:, 0]
        loss = torch.where(ok, lse - zt, 0.0)
        # A logit: D exact products (fp32: six products of parts for one, and what they leave out, below 2^-25 of it) summed in fp32.
        ez = ((D if self.type == torch.bfloat16 else 2 * D) + 2) * U * size
        # exp and its argument: a few roundings relative to |z|; at most 128 terms in a row, 64 rows of up to V / 2048 stretches
        e_sum = (256 + V / 2048 + 8 * (z.abs().amax(dim=1) + lse.abs())) * U
        e_lse = ez.amax(dim=1) + e_sum + 2 * U * lse.abs()
        e_loss = e_lse + ez.gather(1, at[:, None])[:, 0] + 2 * U * zt.abs()
        got_loss, got_lse = self.forward()
        assert ((got_lse.double() - lse).abs() <= e_lse).all(), float(((got_lse.double() - lse).abs() / e_lse).max())
        assert ((got_loss.double() - loss).abs() <= torch.where(ok, e_loss, 0.0)).all()
        again = self.forward()
        assert torch.equal(got_loss, again[0]) and torch.equal(got_lse, again[1])

        d = torch.where(ok, self.d_loss.double(), 0.0)
        c = d + (self.d_lse.double() if self.d_lse is not None else 0.0)
        p = torch.exp(z - lse[:, None])
        hit = torch.zeros_like(p).scatter_(1, at[:, None], ok.double()[:, None])
        g = c[:, None] * p - d[:, None] * hit
        # g: the error of p, that of the subtraction and divisions, and its rounding to bf16 (8 bits: within 2^-8; fp32 in three parts: none)
        eg = (c.abs()[:, None] * p) * (ez + e_lse[:, None] + e_sum[:, None] + 8 * U) + 8 * U * (d.abs()[:, None] * hit + g.abs())
        if self.type == torch.bfloat16:
            eg = eg + 2.0 ** -8 * (g.abs() + eg)
        ends = 2.0 ** -8 if self.type == torch.bfloat16 else 0.0
        n_terms = 1 if self.type == torch.bfloat16 else 2
        d_h, d_w = self.backward(got_lse)
        for got, ref, bound in ((d_h, g @ w, eg @ w.abs() + (n_terms * V + 8) * U * (g.abs() @ w.abs())),
                                (d_w, g.t() @ h, eg.t() @ h.abs() + (n_terms * T + 8) * U * (g.abs().t() @ h.abs()))):
            bound = bound + ends * (ref.abs() + bound)
            over = (got.double() - ref).abs() > bound + 1e-38
            assert not over.any(), (int(over.sum()), float((got.double() - ref).abs().max()))
            if ref.numel() >= 4096 and float(ref.norm()) > 0:      # errors of either sign: far below their bound as a whole
                assert float((got.double() - ref).norm() / ref.norm()) < (2.0 ** -8 if self.type == torch.bfloat16 else 2e-5)
        again = self.backward(got_lse)
        assert torch.equal(d_h, again[0]) and torch.equal(d_w, again[1])
        only_h, only_w = self.backward(got_lse, True, False), self.backward(got_lse, False, True)
        assert torch.equal(d_h, only_h[0]) and torch.equal(d_w, only_w[1])
        return got_loss, got_lse, d_h, d_w


# one token and one word, few tokens (64 a tile), whole and ragged tiles of 128 and of 256, widths that are no multiple of 64, 8 or 2
@pytest.mark.parametrize("T,V,D", [(1, 1, 1), (1, 1000, 64), (2, 3, 128), (5, 1001, 70), (16, 5003, 768), (64, 128, 64), (65, 129, 65), (100, 4097, 192), (128, 256, 33),
                                   (300, 2000, 320), (257, 2500, 1000), (1023, 3001, 96), (700, 513, 2048), (2048, 4096, 128), (2500, 8200, 72)])
@pytest.mark.parametrize("type_", ["bfloat16", "float32"])
def test_loss_and_gradients(env, T, V, D, type_):
    Case(env, T, V, D, type_).check()


@pytest.mark.parametrize("type_", ["bfloat16", "float32"])
def test_gradient_of_the_log_sum(env, type_):
    Case(env, 130, 700, 128, type_, with_lse=True).check()


@pytest.mark.parametrize("type_,T,V", [("bfloat16", 8192, 20000), ("float32", 8192, 7000), ("bfloat16", 5000, 60001)])
def test_vocabularies_in_pieces(env, type_, T, V):
    Case(env, T, V, 64, type_).check()


@pytest.mark.parametrize("type_", ["bfloat16", "float32"])
def test_sure_and_hopeless_tokens(env, type_):
    """Logits up to some hundreds: probabilities of exactly one and of zero, targets among either."""
    torch, _ = env
    T, V, D = 96, 300, 64
    case = Case(env, T, V, D, type_, spread=60.0, padding=0.0)
    z = case.h.double() @ case.w.double().t()
    case.target = torch.where(torch.arange(T, device="cuda") % 2 == 0, z.argmax(dim=1), z.argmin(dim=1))
    case.check()


@pytest.mark.parametrize("type_", ["bfloat16", "float32"])
def test_tokens_that_are_all_padding(env, type_):
    torch, _ = env
    case = Case(env, 70, 300, 64, type_, target=torch.full((70,), -100, device="cuda"))
    loss, lse, d_h, d_w = case.check()
    assert (loss == 0).all() and torch.isfinite(lse).all() and (d_h == 0).all() and (d_w == 0).all()


@pytest.mark.parametrize("type_", ["bfloat16", "float32"])
def test_defaults_of_the_upstream_gradients(env, type_):
    torch, cdl = env
    case = Case(env, 33, 200, 64, type_)
    _, lse = case.forward()
    case.d_loss, ones = torch.ones(33, device="cuda"), case.backward
    ref = ones(lse)
    case.d_loss = None
    got = case.backward(lse)
    assert torch.equal(ref[0], got[0]) and torch.equal(ref[1], got[1])
    assert torch.equal(case.forward()[1], lse)
    only = torch.full_like(lse, float("nan"))
    cdl.cdl_head_loss_fwd(case.h, case.w, case.target, 33, 200, 64, None, only, case.scratch(True))      # no loss asked for; the larger workspace
    assert torch.equal(only, lse)


def test_gradients_are_differences_of_the_loss(env):
    torch, _ = env
    T, V, D, step = 40, 90, 64, 2.0 ** -5
    case = Case(env, T, V, D, "float32", padding=0.1)
    _, lse = case.forward()
    d_h, d_w = case.backward(lse)
    gen = torch.Generator(device="cuda").manual_seed(8)
    ok = ((case.target >= 0) & (case.target < V)).double()
    for which, grad in (("h", d_h), ("w", d_w)):
        base = getattr(case, which)
        way = torch.randn(base.shape, device="cuda", generator=gen)
        way = way / way.norm(dim=1, keepdim=True)
        sums = []
        for sign in (1.0, -1.0):
            setattr(case, which, base + sign * step * way)
            sums.append(case.forward()[0].double())
        setattr(case, which, base)
        diff = float((case.d_loss.double() * (sums[0] - sums[1])).sum()) / (2 * step)
        dz = (way.double() @ case.w.double().t() if which == "h" else case.h.double() @ way.double().t()).abs().amax(dim=1)
        # third cumulant of a variable within [-a, a]: at most (2 a)^3; a loss within (D + 300) 2^-24 (1 + its terms)
        cubic = float((case.d_loss.double() * ok * (2 * dz) ** 3).sum()) * step ** 2 / 6
        noise = float((case.d_loss.double() * ok).sum()) * (2 * D + 400) * U * float((case.h.double().abs() @ case.w.double().abs().t()).max() + 10) / step
        assert abs(diff - float((grad.double() * way.double()).sum())) <= cubic + noise


@pytest.mark.parametrize("type_", ["bfloat16", "float32"])
def test_empty_sizes(env, type_):
    torch, cdl = env
    kind = getattr(torch, type_)
    w = torch.randn((5, 16), device="cuda").to(kind)
    none = torch.empty((0, 16), device="cuda", dtype=kind)
    no_target, no = torch.empty(0, dtype=torch.int64, device="cuda"), torch.empty(0, device="cuda")
    cdl.cdl_head_loss_fwd(none, w, no_target, 0, 5, 16, no, no)
    d_w = torch.full_like(w, 3.0)
    cdl.cdl_head_loss_bwd(none, w, no_target, no, 0, 5, 16, none, d_w)
    assert (d_w == 0).all()
    # no features: every word as likely as any
    T, V = 3, 7
    case = Case(env, T, V, 0, type_, target=torch.tensor([0, 6, -100], device="cuda"))
    loss, lse = case.forward()
    assert torch.allclose(lse, torch.full_like(lse, float(np.log(7))), rtol=1e-6) and float(loss[2]) == 0 and float(loss[0]) == float(lse[0])
    with pytest.raises(cdl.CdlError):
        cdl.cdl_head_loss_fwd(w, none, torch.zeros(5, dtype=torch.int64, device="cuda"), 5, 0, 16, no, torch.empty(5, device="cuda"))


def test_a_token_that_is_not_finite_spoils_no_other(env):
    torch, _ = env
    case = Case(env, 70, 300, 64, "bfloat16", padding=0.0)
    good = case.forward()
    case.h[17, 3] = float("nan")
    loss, lse = case.forward()
    rest = torch.arange(70, device="cuda") != 17
    assert torch.isnan(lse[17]) and torch.isnan(loss[17])
    assert torch.equal(loss[rest], good[0][rest]) and torch.equal(lse[rest], good[1][rest])
    d_h, _ = case.backward(lse)
    assert torch.isnan(d_h[17]).all() and torch.isfinite(d_h[rest].float()).all()


def test_refusals(env):
    torch, cdl = env
    case = Case(env, 8, 32, 16, "bfloat16")
    loss, lse = case.forward()
    with pytest.raises(cdl.CdlError):
        cdl.cdl_head_loss_fwd(case.h, case.w, case.target, 8, 32, 16, loss, lse, case.scratch(False)[:0])
    with pytest.raises(cdl.CdlError):
        cdl.cdl_head_loss_bwd(case.h, case.w, case.target, lse, 8, 32, 16, None, None, case.scratch(True))
    with pytest.raises(TypeError):
        cdl.cdl_head_loss_fwd(case.h, case.w.float(), case.target, 8, 32, 16, loss, lse, case.scratch(False))
    with pytest.raises(TypeError):
        cdl.cdl_head_loss_fwd(case.h, case.w, case.target.int(), 8, 32, 16, loss, lse, case.scratch(False))
    with pytest.raises(ValueError):
        cdl.cdl_head_loss_fwd(case.h.t(), case.w, case.target, 8, 32, 16, loss, lse, case.scratch(False))


@pytest.mark.parametrize("type_", ["bfloat16", "float32"])
def test_another_stream_and_a_graph(env, type_):
    torch, cdl = env
    T, V, D = 80, 1200, 128
    case = Case(env, T, V, D, type_)
    loss, lse = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    d_h, d_w, ws = torch.empty_like(case.h), torch.empty_like(case.w), case.scratch(True)

    def step():
        cdl.cdl_head_loss_fwd(case.h, case.w, case.target, T, V, D, loss, lse, ws)
        cdl.cdl_head_loss_bwd(case.h, case.w, case.target, lse, T, V, D, d_h, d_w, ws, d_loss=case.d_loss)

    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    with torch.cuda.graph(graph, stream=side):
        step()
    gen = torch.Generator(device="cuda").manual_seed(4)
    for i in range(4):
        case.h.copy_(torch.randn((T, D), device="cuda", generator=gen))
        graph.replay()
        torch.cuda.synchronize()
        ref = case.forward()
        assert torch.equal(loss, ref[0]) and torch.equal(lse, ref[1]), i
        ref = case.backward(ref[1])
        assert torch.equal(d_h, ref[0]) and torch.equal(d_w, ref[1]), i
