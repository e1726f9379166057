"""The loss of the last layer where logits are infinite, the lowest or no numbers, and where weights are the largest; its gradients against differences that they cannot miss."""
import pytest

import gpu_util as gu
from test_gpu_head_loss import U, Case

pytestmark = pytest.mark.gpu

SIZES = [(16, 1500, 128), (300, 900, 128), (2100, 4200, 128)]      # tokens for tiles of 128 x 64, 128 x 128 and 256 x 256: stretches of 32, 64 and 128 words


@pytest.fixture(scope="module")
def env():
    import paper_2501_09849_amd as cdl
    return gu.torch_mod(), cdl


def masked_case(env, T, V, D, type_, low):
    """Words without weights but `low` for the feature that is 1 in every token: 300 side by side, which hold whole stretches of every form, the last 200, and every seventh."""
    torch, _ = env
    case = Case(env, T, V, D, type_, with_lse=True)
    case.h[:, 0] = 1.0
    word = torch.arange(V, device="cuda")
    masked = ((word >= 100) & (word < 400)) | (word >= V - 200) | (word % 7 == 3)
    case.w[masked] = 0.0
    case.w[masked, 0] = low
    kept = torch.nonzero(~masked)[:, 0]
    ok = (case.target >= 0) & (case.target < V)
    case.target = torch.where(ok, kept[case.target.clamp(0, V - 1) % kept.numel()], case.target)
    return case, masked, kept, ok


def formulas(torch, case, kept, ok):
    """loss, log-sum, d_h, d_w of the kept words alone, in 64 bits; what rounding may do to a log-sum or loss: D products in 2 D sums (fp32: in parts), an exponential's argument, the sums of stretches"""
    h, w = case.h.double(), case.w[kept].double()
    place = torch.zeros(case.V, dtype=torch.int64, device="cuda")
    place[kept] = torch.arange(kept.numel(), device="cuda")
    at = place[torch.where(ok, case.target, kept[0])]
    z = h @ w.t()
    lse = torch.logsumexp(z, dim=1)
    loss = torch.where(ok, lse - z.gather(1, at[:, None])[:, 0], 0.0)
    d = torch.where(ok, case.d_loss.double(), 0.0)
    g = (d + case.d_lse.double())[:, None] * torch.exp(z - lse[:, None])
    g.scatter_add_(1, at[:, None], -d[:, None])
    error = (2 * case.D + 2) * U * (h.abs() @ w.abs().t()).amax(dim=1) * 2 + (256 + case.V / 2048 + 16 * z.abs().amax(dim=1)) * U
    return loss, lse, g @ w, g.t() @ h, error


@pytest.mark.parametrize("T,V,D", SIZES)
@pytest.mark.parametrize("type_", ["bfloat16", "float32"])
def test_words_of_the_lowest_weight(env, T, V, D, type_):
    """A vocabulary padded with words whose only weight is the type's lowest value: no share in the log-sum, no gradient."""
    torch, _ = env
    case, masked, kept, ok = masked_case(env, T, V, D, type_, torch.finfo(getattr(torch, type_)).min)
    loss, lse, d_h, d_w, error = formulas(torch, case, kept, ok)
    got_loss, got_lse = case.forward()
    assert ((got_lse.double() - lse).abs() <= error).all() and ((got_loss.double() - loss).abs() <= error).all()
    got_h, got_w = case.backward(got_lse)
    assert (got_w[masked] == 0).all()
    # errors of either sign: g's rounding to bf16 and the result's, or those of fp32
    norm = 2.0 ** -8 if type_ == "bfloat16" else 2e-5
    assert float((got_h.double() - d_h).norm()) <= norm * float(d_h.norm()) and float((got_w[kept].double() - d_w).norm()) <= norm * float(d_w.norm())


@pytest.mark.parametrize("T,V,D", SIZES)
def test_words_of_infinitely_small_logits(env, T, V, D):
    torch, _ = env
    case, masked, kept, ok = masked_case(env, T, V, D, "bfloat16", float("-inf"))
    loss, lse, _, d_w, error = formulas(torch, case, kept, ok)
    got_loss, got_lse = case.forward()
    assert ((got_lse.double() - lse).abs() <= error).all() and ((got_loss.double() - loss).abs() <= error).all()
    got_w = case.backward(got_lse, want_h=False)[1]      # (d_h has 0 times infinity)
    assert (got_w[masked] == 0).all() and float((got_w[kept].double() - d_w).norm()) <= 2.0 ** -8 * float(d_w.norm())


@pytest.mark.parametrize("T,V,D", SIZES)
def test_logits_that_are_all_infinite(env, T, V, D):
    """Tokens all of whose logits are -infinity: a log-sum of -infinity; one of whose logits is +infinity: +infinity; the others as ever."""
    torch, _ = env
    case = Case(env, T, V, D, "bfloat16", padding=0.0)
    case.h[:, 0], case.h[:, 1] = 0.0, 0.0
    plain = case.forward()
    case.w[:, 0] = -(2.0 ** 120)
    case.w[:, 1] = 0.0
    case.w[V // 2, 1] = 2.0 ** 120
    case.target[:3] = 0
    case.h[0, 0] = 2.0 ** 20      # (products beyond the range of fp32)
    case.h[1, 1] = 2.0 ** 20
    loss, lse = case.forward()
    assert float(lse[0]) == float("-inf") and float(lse[1]) == float("inf") and float(loss[1]) == float("inf")
    assert torch.equal(lse[2:], plain[1][2:]) and torch.equal(loss[3:], plain[0][3:]) and torch.isfinite(plain[1]).all()      # (the features that differ are zero there)


@pytest.mark.parametrize("type_", ["bfloat16", "float32"])
def test_no_numbers_are_never_hidden(env, type_):
    """A token with NaN: its loss, its d_h and all of d_w; a word with NaN: every token's loss and every gradient."""
    torch, _ = env
    T, V, D = 70, 300, 64
    case = Case(env, T, V, D, type_, padding=0.0)
    case.h[17, 3] = float("nan")
    loss, lse = case.forward()
    d_h, d_w = case.backward(lse)
    rest = torch.arange(T, device="cuda") != 17
    assert torch.isnan(loss[17]) and torch.isnan(lse[17]) and torch.isfinite(lse[rest]).all()
    assert torch.isnan(d_h[17]).all() and torch.isfinite(d_h[rest].float()).all() and torch.isnan(d_w).all()
    case = Case(env, T, V, D, type_, padding=0.0)
    case.w[40, 5] = float("nan")
    loss, lse = case.forward()
    d_h, d_w = case.backward(lse)
    assert torch.isnan(loss).all() and torch.isnan(lse).all() and torch.isnan(d_h).all() and torch.isnan(d_w).all()


def test_fp32_weights_up_to_the_largest(env):
    """An fp32 operand is used as three bf16 parts: also one that rounds to infinity as bf16."""
    torch, _ = env
    T, V, D = 40, 300, 64
    top = torch.finfo(torch.float32).max
    case = Case(env, T, V, D, "float32", padding=0.0)
    case.h[:, 0] = 2.0 ** -127 * torch.randint(2, 64, (T,), device="cuda").float()      # two logits up to 126
    case.w[7, 0], case.w[8, 0] = top, -top
    ok = torch.ones(T, dtype=torch.bool, device="cuda")
    every = torch.arange(V, device="cuda")
    case.d_lse = torch.zeros(T, device="cuda")
    loss, lse, _, d_w, error = formulas(torch, case, every, ok)
    got_loss, got_lse = case.forward()
    # (h's entry is 2^-126 to 2^-122, whose parts below 2^-126 the matrix cores take as zero; it has six bits, so one part holds it)
    assert ((got_lse.double() - lse).abs() <= error).all() and ((got_loss.double() - loss).abs() <= error).all()
    got_w = case.backward(got_lse, want_h=False)[1]
    assert float((got_w.double() - d_w)[:, 1:].norm()) <= 2e-5 * float(d_w[:, 1:].norm())


def test_gradient_of_a_token_is_the_difference_of_its_loss(env):
    """Every token for itself, along its own gradient, where the difference is largest."""
    torch, _ = env
    T, V, D, step = 40, 90, 64, 2.0 ** -5
    case = Case(env, T, V, D, "float32", padding=0.0)
    case.d_loss = torch.ones(T, device="cuda")
    every, ok = torch.arange(V, device="cuda"), torch.ones(T, dtype=torch.bool, device="cuda")
    case.d_lse = torch.zeros(T, device="cuda")
    _, lse, way, _, error = formulas(torch, case, every, ok)
    d_h, _ = case.backward(case.forward()[1])
    way = (way / way.norm(dim=1, keepdim=True)).float()
    high, low = (case.forward((case.h + sign * step * way).contiguous())[0].double() for sign in (1.0, -1.0))
    moved = ((case.h + step * way).double() - (case.h - step * way).double()) / (2 * step)      # (what the rounding of h has left of the direction)
    diff, along = (high - low) / (2 * step), (d_h.double() * moved).sum(dim=1)
    # the third derivative is a third cumulant: at most the cube of the range of dz; either loss within its rounding (twice, for the moved h)
    dz = moved @ case.w.double().t()
    bound = (dz.amax(dim=1) - dz.amin(dim=1)) ** 3 * step ** 2 / 6 + 2 * error / step + 1e-5
    assert (along > 10 * bound).all(), float((along / bound).min())      # zeros would not pass
    assert ((diff - along).abs() <= bound).all()


def test_gradient_of_the_vocabulary_is_the_difference_of_the_loss(env):
    torch, _ = env
    T, V, D, step = 40, 90, 64, 2.0 ** -4
    case = Case(env, T, V, D, "float32", padding=0.1)
    ok = (case.target >= 0) & (case.target < V)
    case.d_lse = torch.zeros(T, device="cuda")
    _, _, _, way, error = formulas(torch, case, torch.arange(V, device="cuda"), ok)
    _, d_w = case.backward(case.forward()[1])
    way = (way / way.norm()).float()
    base, sums, moved = case.w, [], []
    for sign in (1.0, -1.0):
        case.w = base + sign * step * way
        moved.append(case.w.double())
        sums.append(case.forward()[0].double())
    moved = (moved[0] - moved[1]) / (2 * step)
    weight = case.d_loss.double() * ok
    diff, along = float((weight * (sums[0] - sums[1])).sum()) / (2 * step), float((d_w.double() * moved).sum())
    dz = case.h.double() @ moved.t()
    bound = float((weight * ((dz.amax(dim=1) - dz.amin(dim=1)) ** 3 * step ** 2 / 6 + 2 * error / step)).sum()) + 1e-5
    assert along > 10 * bound, along / bound
    assert abs(diff - along) <= bound
