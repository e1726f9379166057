"""Dropout from a counter-based generator against a plain implementation of the published generator."""
import numpy as np
import pytest

import gpu_util as gu

pytestmark = pytest.mark.gpu


def philox(counter, key):
    """four words for each counter (two numpy uint64 arrays / a 64-bit key); J. Salmon et al., SC 2011, ten rounds"""
    m = np.uint64(0xFFFFFFFF)
    x = [counter & m, counter >> np.uint64(32), np.zeros_like(counter), np.zeros_like(counter)]
    k = [key & 0xFFFFFFFF, key >> 32]
    for _ in range(10):
        p, q = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(q >> np.uint64(32)) ^ x[1] ^ np.uint64(k[0]), q & m, (p >> np.uint64(32)) ^ x[3] ^ np.uint64(k[1]), p & m]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return x


def kept(n, p, seed, counter):
    with np.errstate(over="ignore"):
        ctr = np.arange((n + 7) // 8, dtype=np.uint64) + np.uint64(counter)
        words = np.stack(philox(ctr, seed), axis=1)
    halves = np.stack([words & np.uint64(0xFFFF), words >> np.uint64(16)], axis=2).reshape(-1)[:n]
    return halves >= np.uint64(round(p * 65536))


def test_the_generator_has_its_published_values():
    """the test vectors that accompany the paper"""
    word = lambda c, k: ["%08x" % int(w[0]) for w in philox(np.array([c], dtype=np.uint64), k)]      # noqa: E731
    assert word(0, 0) == ["6627e8d5", "e169c58d", "bc57ac4c", "9b00dbd8"]


@pytest.fixture(scope="module")
def env():
    import paper_2501_09849_amd as cdl
    return gu.torch_mod(), cdl


@pytest.mark.parametrize("n", [1, 2, 7, 8, 9, 2047, 2048, 2049, 65536 + 3, 9_000_011])
@pytest.mark.parametrize("type_", ["float32", "bfloat16"])
@pytest.mark.parametrize("add", [False, True])
def test_every_entry(env, n, type_, add):
    torch, cdl = env
    gen = torch.Generator().manual_seed(n)
    x, a = (torch.randn(n, generator=gen).to(getattr(torch, type_)) for _ in range(2))
    p, seed, counter = 0.3, 0x0123456789ABCDEF, (1 << 40) + 17
    y = torch.empty(n, dtype=x.dtype, device="cuda")
    cdl.cdl_dropout(x.cuda(), n, p, seed, counter, y, add=a.cuda() if add else None)
    scale = np.float32(65536.0 / (65536 - round(p * 65536)))
    ref = torch.where(torch.from_numpy(kept(n, p, seed, counter)), x.float() * float(scale), torch.zeros(()))
    ref = (ref + a.float() if add else ref).to(x.dtype)
    assert torch.equal(y.cpu(), ref)


@pytest.mark.parametrize("p", [0.0, 1.0 / 65536, 0.1, 0.5, 0.999, 1.0 - 1.0 / 65536, 1.0])
def test_probabilities(env, p):
    torch, cdl = env
    n = 1 << 20
    x = torch.ones(n, device="cuda")
    y = torch.empty_like(x)
    cdl.cdl_dropout(x, n, p, 99, 5, y)
    keep = kept(n, p, 99, 5)
    assert np.array_equal(y.cpu().numpy() != 0, keep)
    # the share of dropped entries within six standard deviations
    assert abs((~keep).mean() - p) <= 6 * np.sqrt(p * (1 - p) / n) + 2.0 ** -17
    if 0 < p < 1:
        assert float(y.max()) == float(np.float32(65536.0 / (65536 - round(p * 65536))))


def test_backward_in_place_and_parts(env):
    """The backward pass is the same call; y may be x or add; two parts of a tensor with counters a part apart are the whole."""
    torch, cdl = env
    n = 40_000
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, g = torch.randn(n, device="cuda", generator=gen), torch.randn(n, device="cuda", generator=gen)
    y, d = torch.empty_like(x), torch.empty_like(x)
    cdl.cdl_dropout(x, n, 0.25, 7, 0, y)
    cdl.cdl_dropout(g, n, 0.25, 7, 0, d)
    assert torch.equal(y != 0, d != 0)
    # linear in x: the derivative along g is dropout of g
    h = torch.empty_like(x)
    cdl.cdl_dropout(x + g, n, 0.25, 7, 0, h)
    assert ((h.double() - y.double() - d.double()).abs() <= 2.0 ** -22 * (x.abs() + g.abs()).double() * (4 / 3)).all()
    for which in ("x", "add"):
        a, b = x.clone(), g.clone()
        out = a if which == "x" else b
        cdl.cdl_dropout(a, n, 0.25, 7, 0, out, add=b)
        assert torch.equal(out, y + g)
    half = n // 2
    z = torch.empty_like(x)
    cdl.cdl_dropout(x[:half], half, 0.25, 7, 0, z[:half])
    cdl.cdl_dropout(x[half:], half, 0.25, 7, half // 8, z[half:])
    assert torch.equal(z, y)


def test_what_is_dropped_may_be_anything(env):
    torch, cdl = env
    n = 4096
    x = torch.full((n,), float("nan"), device="cuda")
    x[::2] = float("inf")
    y = torch.empty_like(x)
    cdl.cdl_dropout(x, n, 0.5, 3, 0, y)
    assert np.array_equal(~torch.isfinite(y).cpu().numpy(), kept(n, 0.5, 3, 0))


def test_counters_wrap(env):
    torch, cdl = env
    n, counter = 64, 2 ** 64 - 3
    y = torch.empty(n, device="cuda")
    cdl.cdl_dropout(torch.ones(n, device="cuda"), n, 0.5, 2 ** 64 - 1, counter, y)
    assert np.array_equal(y.cpu().numpy() != 0, kept(n, 0.5, 2 ** 64 - 1, counter))


def test_refusals(env):
    torch, cdl = env
    x = torch.zeros(16, device="cuda")
    for p in (-0.1, 1.5, float("nan")):
        with pytest.raises(cdl.CdlError):
            cdl.cdl_dropout(x, 16, p, 0, 0, x)
    with pytest.raises(TypeError):
        cdl.cdl_dropout(x, 16, 0.5, 0, 0, x.bfloat16())
    with pytest.raises(TypeError):
        cdl.cdl_dropout(x.double(), 16, 0.5, 0, 0, x.double())
    with pytest.raises(OverflowError):
        cdl.cdl_dropout(x, 16, 0.5, -1, 0, x)
