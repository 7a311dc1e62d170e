"""Tokens from logits and given random numbers on the GPU: the token is the definition's in float64, exactly."""
import math

import numpy as np
import pytest
import torch

from oracle.layer import draw
from paper_2608_08020_amd import gambit as g

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _rows(n, V, dtype, seed, spread=2.5, step=None):
    gen = torch.Generator().manual_seed(seed)
    z = spread * torch.randn(n, V, generator=gen)
    for r in range(n):
        at = torch.randint(0, V, (min(V, 1 + 5 * r),), generator=gen)
        z[r, at] += 3 + r
    if step:
        z = (z / step).round() * step
    return z.to(dtype).to(DEV), torch.rand(n, generator=gen).to(DEV)


def _check(z, u, **par):
    got = g.sample(z, u, **{k: v.to(DEV) if isinstance(v, torch.Tensor) else v for k, v in par.items()})
    assert got.dtype == torch.int32 and got.shape == u.shape
    zs, us = z.double().cpu().numpy(), u.double().cpu().numpy()
    one = lambda v, r: float(v[r]) if isinstance(v, torch.Tensor) else float(np.float32(v))  # noqa: E731
    want = []
    for r in range(len(us)):
        p = {k: one(v, r) for k, v in par.items()}
        if "top_k" in p:
            p["top_k"] = int(p["top_k"])
        want.append(draw(zs[r], us[r], **p))
    assert got.tolist() == want


FILTERS = [dict(), dict(temperature=0.7), dict(top_k=1), dict(top_k=20), dict(top_p=0.9), dict(top_p=0.5, temperature=1.5), dict(min_p=0.05),
           dict(top_k=40, top_p=0.95), dict(top_k=7, min_p=0.1, temperature=1.3), dict(top_p=0.8, min_p=0.02), dict(top_k=1000, top_p=0.99, min_p=0.001),
           dict(temperature=0.0), dict(temperature=8.0, top_p=0.3), dict(temperature=0.05), dict(top_p=0.999), dict(top_p=1e-6), dict(min_p=1.0)]


@pytest.mark.parametrize("V", [1, 2, 7, 8, 63, 64, 65, 511, 1000, 4097, 50257])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_draw(V, dtype):
    z, u = _rows(6, V, dtype, V)
    for f in FILTERS:
        _check(z, u, **f)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_draw_long_rows(dtype):
    z, u = _rows(4, 151936, dtype, 3)
    for f in FILTERS:
        _check(z, u, **f)
    z, u = _rows(2, 1 << 18, dtype, 4)
    for f in (dict(), dict(top_p=0.95), dict(top_k=50)):
        _check(z, u, **f)


@pytest.mark.parametrize("V", [5, 300, 20000, 150001])
@pytest.mark.parametrize("step", [0.5, 4.0, 100.0])
def test_ties(V, step):
    """Many equal logits: the lower index comes first, in top-k, in top-p and in greedy draws."""
    z, u = _rows(4, V, torch.float32, V, step=step)
    for f in FILTERS + [dict(top_k=V // 2), dict(top_k=V - 1), dict(top_k=V), dict(top_k=3, temperature=2.0), dict(top_k=max(1, V // 3), top_p=0.5)]:
        _check(z, u, **f)


@pytest.mark.parametrize("V", [1, 4, 10, 4096, 4097, 100000])
def test_equal_logits(V):
    z = torch.full((5, V), -3.25, device=DEV)
    u = torch.tensor([0.0, 0.25, 0.5, 0.75, 1 - 2.0 ** -24], device=DEV)
    for f in (dict(), dict(top_k=3), dict(top_p=0.5), dict(top_p=0.5, top_k=max(1, V // 2)), dict(min_p=1.0), dict(temperature=0.0), dict(temperature=math.inf),
              dict(top_p=0.25, temperature=100.0)):
        _check(z, u, **f)


def test_flat_rows_need_every_window():
    """Weights spread over tens of octaves, and whole rows in a few of them."""
    V = 30000
    z = torch.linspace(0, -40, V).repeat(4, 1)
    z[1] = torch.linspace(0, -1e-3, V)
    z[2] = -z[2].flip(0)
    z[3] = torch.where(torch.arange(V) % 2 == 0, 0.0, -25.0)
    u = torch.tensor([0.1, 0.9, 0.5, 0.99], device=DEV)
    for f in (dict(), dict(top_k=29000), dict(top_k=15003), dict(top_p=0.9999), dict(top_k=20000, top_p=0.999), dict(min_p=1e-9), dict(top_p=0.7)):
        _check(z.to(DEV), u, **f)
        _check(z.to(DEV, torch.bfloat16), u, **f)


def test_each_row_its_own_parameters():
    n = 40
    gen = torch.Generator().manual_seed(9)
    pick = lambda v, dt: torch.tensor(v, dtype=dt)[torch.randint(0, len(v), (n,), generator=gen)]  # noqa: E731
    for dtype in (torch.bfloat16, torch.float32):
        z, u = _rows(n, 3001, dtype, 6)
        _check(z, u, temperature=pick([0.0, 0.5, 1.0, 2.0, -1.0, 1e-30], torch.float32), top_k=pick([0, -3, 1, 5, 100, 3000, 9999], torch.int32),
               top_p=pick([0.0, 0.3, 0.9, 1.0, 2.0], torch.float32), min_p=pick([0.0, 0.1, 1.0, 7.0, -1.0], torch.float32))


def test_masked_and_not_finite_logits():
    V = 700
    z, u = _rows(9, V, torch.float32, 2)
    inf, nan = math.inf, math.nan
    z[0] = -inf                          # nothing to draw
    z[1] = nan
    z[2, :] = -inf
    z[2, 5] = -1e30                      # one token
    z[3, 1:] = torch.finfo(torch.float32).min
    z[4, ::3] = -inf
    z[4, 1::3] = nan
    z[5, 11] = z[5, 600] = inf           # counts as the largest finite value
    z[6, ::2] = -inf
    z[7] = torch.where(torch.arange(V, device=DEV) % 2 == 0, 0.0, -0.0)
    for f in FILTERS + [dict(top_k=699), dict(top_k=200, temperature=50.0)]:
        _check(z, u, **f)
    z16 = z.to(torch.bfloat16)
    for f in FILTERS:
        _check(z16, u, **f)
    assert g.sample(z, u)[:2].tolist() == [-1, -1]


def test_random_numbers_at_and_beyond_their_ends():
    z = torch.tensor([[0.0, 0, 0, -math.inf, 0, -math.inf]], device=DEV).repeat(6, 1)
    u = torch.tensor([0.0, -1.0, math.nan, 1.0, 5.0, 0.5], device=DEV)
    assert g.sample(z, u).tolist() == [0, 0, 0, 4, 4, 2]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lead", [0, 1, 3, 5, 7])
def test_rows_at_any_address(dtype, lead):
    """Rows that begin inside a 16-byte load, and end inside one; what stands beside them does not count."""
    V = 1003
    wide = torch.full((5, V + 14), 1e30, dtype=dtype, device=DEV)
    z, u = _rows(5, V, dtype, lead)
    wide[:, lead:lead + V] = z
    for f in (dict(), dict(top_k=9), dict(top_p=0.9), dict(temperature=0.0)):
        _check(wide[:, lead:lead + V], u, **f)
    assert torch.equal(g.sample(z[:1].expand(4, V), u[:4], top_p=0.9), g.sample(z[:1].repeat(4, 1), u[:4], top_p=0.9))


def test_shares_of_many_draws():
    """Over an even grid of random numbers each token comes as often as its weight says, to one draw at each of its two ends."""
    n = 4096
    z = torch.tensor([1.0, -2.0, 0.5, 3.0, 2.9, -math.inf, 0.0], device=DEV)
    u = ((torch.arange(n, device=DEV) + 0.5) / n).float()
    got = torch.bincount(g.sample(z.expand(n, 7), u, temperature=0.8).long(), minlength=7).double().cpu()
    want = torch.softmax(z.double().cpu() / float(np.float32(0.8)), 0) * n
    assert (got - want).abs().max() <= 2


def test_no_rows_and_given_output():
    assert g.sample(torch.empty(0, 9, device=DEV), torch.empty(0, device=DEV)).shape == (0,)
    z, u = _rows(3, 50, torch.float32, 1)
    out = torch.zeros(3, dtype=torch.int32, device=DEV)
    assert g.sample(z, u, out=out) is out
    assert torch.equal(out, g.sample(z, u))


def test_more_rows_than_one_set_of_launches_takes():
    n, V = 4099, 16500
    z = 2.5 * torch.randn(n, V, generator=torch.Generator(device=DEV).manual_seed(4), device=DEV).to(torch.bfloat16)
    u = torch.rand(n, generator=torch.Generator(device=DEV).manual_seed(5), device=DEV)
    k = torch.randint(0, 300, (n,), generator=torch.Generator(device=DEV).manual_seed(6), device=DEV, dtype=torch.int32)
    par = dict(temperature=u + 0.3, top_p=1 - 0.5 * u, min_p=0.01 * u)
    got = g.sample(z, u, top_k=k, **par)
    for at in (slice(0, 5), slice(4090, 4099)):
        assert torch.equal(got[at], g.sample(z[at], u[at].clone(), top_k=k[at].clone(), **{a: b[at].clone() for a, b in par.items()}))
    _check(z[4095:].clone(), u[4095:].clone(), top_k=k[4095:].clone(), **{a: b[4095:].clone() for a, b in par.items()})


@pytest.mark.parametrize("V", [8190, 8192, 8200, 16370, 16384, 16400])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_where_rows_begin_to_be_cut_into_chunks(V, dtype):
    z, u = _rows(3, V, dtype, V)
    for par in FILTERS:
        _check(z, u, **par)


@pytest.mark.parametrize("many", [500, 700, 3000, 9000])
def test_many_values_where_the_filter_ends(many):
    V = 40000
    z, u = _rows(4, V, torch.float32, many, spread=1.0)
    z = z.clamp(max=4)
    at = torch.randperm(V, generator=torch.Generator().manual_seed(many))[:many].to(DEV)
    z[:, at] = 6 + 0.05 * torch.rand(4, many, generator=torch.Generator().manual_seed(1)).to(DEV)  # one bin
    z[1, at[::2]] = 6.03125  # half of them equal
    z[2, at] = 6.0
    for par in (dict(top_k=many // 3), dict(top_p=0.2), dict(top_k=many // 2, top_p=0.6), dict(top_p=0.4, min_p=0.5), dict(top_k=many - 1)):
        _check(z, u, **par)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_long_rows_with_masked_and_not_finite_logits(dtype):
    V, n = 40000, 10
    z, u = _rows(n, V, torch.float32, 8)
    z = z.to(dtype)
    ints = z.view(torch.int16 if dtype == torch.bfloat16 else torch.int32)
    quiet, signalling = (0x7FC0, 0x7F81) if dtype == torch.bfloat16 else (0x7FC00000, 0x7F800001)
    z[0, ::2] = math.nan
    ints[1, ::3] = signalling  # as bits: copies keep them
    ints[2, 5::7] = quiet - (1 << (16 if dtype == torch.bfloat16 else 32)) | (1 << 15 if dtype == torch.bfloat16 else 1 << 31)  # negative
    z[3, 100] = math.inf
    z[4, 7::5] = math.inf
    z[5] = -math.inf
    z[5, 31234] = 1.5
    z[6] = math.nan
    z[7] = -math.inf
    z[8, :39000] = torch.finfo(dtype).min
    z[9] = -0.0
    z[9, 20000:] = 0.0
    assert torch.isnan(z[1, 0]) and torch.isnan(z[2, 5])
    for par in FILTERS:
        _check(z, u, **par)
