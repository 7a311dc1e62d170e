"""Packed tokens on the GPU: values that are not finite.

A position that a row sees counts for it whatever its weight: where its V is
not finite, that element of the row's output is not, however small the weight,
and however the row's positions were cut into tiles and chunks.  A position
that a row does not see never counts.
"""
import math

import pytest
import torch

from test_gpu_packed import D, DEV, OUT, Kept, _causal, _check, _kin

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
