"""Packed tokens on the GPU: values that are not finite, and block scales of zero or next to it.

A position that a row sees counts for it whatever its weight: where its V is
not finite, that element of the row's output is not, however small the weight,
and however the row's positions were cut into tiles and chunks.  A position
that a row does not see never counts.
"""
import math

import numpy as np
import pytest
import torch

from test_gpu_packed import D, DEV, OUT, Kept, _causal, _check, _k_phys, _kin

pytestmark = pytest.mark.gpu

# q[5] >= 1/2 against K[5] = -4000: a score of -176 at most, e^-176 = 2^-255 of a row's other weights, nothing in fp32
LOW = -4000.0


def _queries(S, m, rows=slice(None)):
    q = S.normal(m, S.Hq, D)
    q[rows, :S.Hq // S.Hkv, 5] = q[rows, :S.Hq // S.Hkv, 5].abs() + 0.5
    return q


def _without(out, V, d):
    """Element d of KV head 0's rows and values as zeros."""
    out, V = out.clone(), V.clone()
    out[:, :out.shape[1] // V.shape[1], d] = 0
    V[:, 0, d] = 0
    return out, V


# 40: one tile that no row sees whole; 200: a token of a tile that every row sees; 3000: chunks of 256 positions,
# the first ones with no other weight
@pytest.mark.parametrize("n,low,at", [(40, 11, 10), (200, 11, 10), (200, 199, 190), (3000, 1500, 700), (3000, 2990, 2985)])
@pytest.mark.parametrize("bad", [math.inf, math.nan])
@pytest.mark.parametrize("out_dtype", OUT)
@pytest.mark.parametrize("tree", [False, True])
def test_a_value_that_is_not_finite_reaches_every_row_that_sees_it(n, low, at, bad, out_dtype, tree):
    S = Kept(8, 2, T=2, maxb=200)
    m, d = 4, 3
    k, v = S.normal(n, 2, D), S.normal(n, 2, D)
    k[:low, 0, 5] = LOW
    v[at, 0, d] = bad
    S.extend([1], [n], k=k, v=v)
    q = _queries(S, m)
    if tree:
        kn, vn = S.normal(m, 2, D), S.normal(m, 2, D)
        up = [-1, 0, 0, 2]
        out = S.pool.tree_attn(0, [1], [m], up, q, kn, vn, out_dtype=out_dtype)
        K, V = torch.cat([S.K[1], kn.double()]), torch.cat([S.V[1], vn.double()])
        sees = torch.cat([torch.ones(m, n, dtype=torch.bool, device=DEV), _kin(up)], 1)
    else:
        out = S.pool.prompt_attn(0, [1], [m], q, out_dtype=out_dtype)
        K, V, sees = S.K[1], S.V[1], _causal(n, m)
    hit = out[:, :4, d].double()
    assert not torch.isfinite(hit).any(), hit
    out, V = _without(out, V, d)
    _check(out, q, K, V, sees)


@pytest.mark.parametrize("n,low,at", [(40, 11, 10), (3000, 1500, 700)])
@pytest.mark.parametrize("out_dtype", OUT)
def test_a_nan_value_of_an_fp8_pool_reaches_every_row_that_sees_it(n, low, at, out_dtype):
    S = Kept(16, 2, T=2, maxb=200, fp8=True)
    m, d = 4, 3
    k, v = S.normal(n, 2, D), S.normal(n, 2, D)
    k[:low, 0, 5] = LOW
    v[at, 0, d] = math.nan
    S.extend([1], [n], k=k, v=v)
    q = _queries(S, m)
    out = S.pool.prompt_attn(0, [1], [m], q, out_dtype=out_dtype)
    assert torch.isnan(out[:, :8, d].double()).all()
    out, V = _without(out, S.V[1], d)
    _check(out, q, S.K[1], V, _causal(n, m))


@pytest.mark.parametrize("bad", [math.inf, math.nan])
@pytest.mark.parametrize("out_dtype", OUT)
def test_a_draft_that_is_not_finite_reaches_its_branch_and_no_other(bad, out_dtype):
    S = Kept(8, 2, T=2, maxb=20)
    n, d = 70, 3
    S.extend([1], [n])
    up = [-1, 0, 1, -1, 3, 2]
    seen, free = [0, 1, 2, 5], [3, 4]
    q = _queries(S, 6, seen)
    kn, vn = S.normal(6, 2, D), S.normal(6, 2, D)
    kn[0, 0, 5] = LOW
    vn[0, 0, d] = bad
    out = S.pool.tree_attn(0, [1], [6], up, q, kn, vn, out_dtype=out_dtype)
    assert not torch.isfinite(out[seen, :4, d].double()).any()
    K, V = torch.cat([S.K[1], kn.double()]), torch.cat([S.V[1], vn.double()])
    sees = torch.cat([torch.ones(6, n, dtype=torch.bool, device=DEV), _kin(up)], 1)
    clean = V.clone()
    clean[n, 0, d] = 0.0                               # nodes 3 and 4 do not see it
    _check(out[free], q[free], K, clean, sees[free])
    out, V = _without(out, V, d)
    _check(out, q, K, V, sees)


# ------------------------------------------------------------ block scales next to zero --
@pytest.mark.parametrize("scale", [0.0, 1e-44, 1e-39, 2.0 ** -128, 2.0 ** -127, 2.0 ** -100])
@pytest.mark.parametrize("Hkv", [2, 12])
def test_write_into_a_begun_block_of_a_tiny_scale(Hkv, scale):
    """Codes of x / s (fp32 quotient) for scales whose reciprocal is beyond fp32; zero stays zero for any scale."""
    n, a = 9, 4
    S = Kept(Hkv, Hkv, T=2, maxb=2, fp8=True)
    S.pool.kv_alloc([0], [a + n])
    S.pool.kv_scale.fill_(scale)
    s = np.float32(scale)
    k, v = S.normal(n, Hkv, D), S.normal(n, Hkv, D)
    for x in (k, v):
        x[:, :, ::4] = 0.0
        x[:, :, 1::8] *= 2.0 ** -126                   # quotients inside E4M3FN's range
    S.pool.kv_write_layer(0, [0], [a], [n], k, v)
    b = int(S.pool.block_table[0, 0])
    t = np.arange(a, a + n)
    d = np.arange(D)
    for i, (x, cache) in enumerate(((k, S.pool.k_cache), (v, S.pool.v_cache))):
        y = x.float().cpu().numpy()
        with np.errstate(divide="ignore", invalid="ignore", over="ignore"):
            y = np.where(y == 0, y, y / s)
        want = torch.from_numpy(np.clip(y, -448, 448)).to(torch.float8_e4m3fn).float()
        idx = ((d // 16) * 16 + _k_phys(t)[:, None]) * 16 + d % 16 if i == 0 else d * 16 + t[:, None]
        got = cache[b].reshape(Hkv, -1)[:, torch.from_numpy(idx).to(DEV)].permute(1, 0, 2).cpu()
        got = got.contiguous().view(torch.float8_e4m3fn).float()
        assert torch.equal(got, want), (i, int((got != want).sum()))
        assert (S.pool.kv_scale[b].cpu().numpy() == s).all()
