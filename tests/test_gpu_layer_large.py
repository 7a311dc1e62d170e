"""A layer's operators over more than four gigabytes: the rows at both ends are those of the same call on them alone."""
import pytest
import torch

from paper_2608_08020_amd import gambit as g

pytestmark = pytest.mark.gpu
DEV = "cuda"
E4M3, BF16 = torch.float8_e4m3fn, torch.bfloat16
ENDS = 5


@pytest.fixture(autouse=True)
def _release():
    yield
    torch.cuda.empty_cache()


def _big(n, *shape, dtype=BF16):
    """n rows, the ends of their own, the same block of rows again and again between."""
    x = torch.empty(n, *shape, dtype=dtype, device=DEV)
    gen = torch.Generator(device=DEV).manual_seed(n)
    some = torch.randn(1000, *shape, generator=gen, device=DEV).to(dtype)
    for a in range(0, n, 1000):
        x[a:a + 1000] = some[:min(1000, n - a)]
    for ends in (slice(0, ENDS), slice(n - ENDS, n)):
        x[ends] = torch.randn(ENDS, *shape, generator=gen, device=DEV).to(dtype)
    assert x.numel() * x.element_size() > 1 << 32
    return x


def _ends(n):
    return slice(0, ENDS), slice(n - ENDS, n)


def _same(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def test_norm():
    n, dim = 270_011, 8192
    x, w = _big(n, dim), torch.ones(dim, dtype=BF16, device=DEV)
    y = g.rms_norm(x, w)
    codes, scale = g.rms_norm(x, w, out_dtype=E4M3)
    for e in _ends(n):
        assert _same(y[e], g.rms_norm(x[e], w))
        c, s = g.rms_norm(x[e], w, out_dtype=E4M3)
        assert _same(codes[e], c) and torch.equal(scale[:, e], s)


def test_norm_of_heads_and_rotation():
    n = 1_700_003
    x = _big(n, 10, 128)
    q, k, _ = x.split([6, 2, 2], 1)
    w, table = torch.ones(128, dtype=BF16, device=DEV), torch.rand(50, 96, device=DEV)
    pos = torch.arange(n, dtype=torch.int32, device=DEV) % 50
    y = g.rms_norm(q, w)
    qo, ko = g.rotate(q, k, pos, table)
    for e in _ends(n):
        assert _same(y[e], g.rms_norm(q[e], w))
        a, b = g.rotate(q[e], k[e], pos[e].clone(), table)
        assert _same(qo[e], a) and _same(ko[e], b)


def test_gate():
    n, dim = 140_003, 8192
    x = _big(n, 2 * dim)
    codes, scale = g.quantize(x, gated=True)
    for e in _ends(n):
        c, s = g.quantize(x[e], gated=True)
        assert _same(codes[e], c) and torch.equal(scale[:, e], s)


def test_product_of_many_tokens():
    n, k = 1_060_003, 4096
    x, xs = _big(n, k, dtype=E4M3), torch.rand(k // 128, n, device=DEV)
    w, ws = torch.randn(40, k, device=DEV).to(E4M3), torch.rand(1, k // 128, device=DEV)
    y = g.linear_fp8(x, xs, w, ws)
    for e in _ends(n):  # (in as many tokens as take the same kernel)
        at = slice(e.start - 66_000 if e.start else 0, e.stop + (0 if e.start else 66_000))
        z = g.linear_fp8(x[at], xs[:, at].contiguous(), w, ws)
        assert _same(y[e], z[-ENDS:] if e.start else z[:ENDS])


def test_product_of_many_features():
    n, k = 1_060_003, 4096
    w, ws = _big(n, k, dtype=E4M3), torch.rand(-(-n // 128), k // 128, device=DEV)
    x, xs = torch.randn(70, k, device=DEV).to(E4M3), torch.rand(k // 128, 70, device=DEV)
    for m in (1, 20, 70):
        y = g.linear_fp8(x[:m], xs[:, :m].contiguous(), w, ws)
        at = (n - 80_000) // 128 * 128  # (as many as take the same kernel)
        z = g.linear_fp8(x[:m], xs[:, :m].contiguous(), w[at:], ws[at // 128:])
        assert _same(y[:, at:], z)


def test_draw():
    n, V = 16_400, 131_077
    z = _big(n, V)
    u = torch.rand(n, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV)
    for par in (dict(top_p=0.9), dict(top_k=30), dict()):
        got = g.sample(z, u, **par)
        for e in _ends(n):
            assert torch.equal(got[e], g.sample(z[e], u[e].clone(), **par))
