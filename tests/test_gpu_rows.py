"""Norms and rows to 8 bits on the GPU, against the definition in float64.

Of a normed value, relative to itself: the sum h is rounded once (2^-24); the
squares' sum is at most 32 additions in a lane, 6 among lanes, 16 among waves,
and a rounding each of the squares, the mean, eps' addition, and enters by its root
(28 2^-24); root, reciprocal and two products 4 2^-24: 2^-18 holds them all.
An output's own rounding is half a step (bf16 2^-8, fp32 2^-24, E4M3 2^-4, or
2^-10 of the scale where codes are subnormal).  silu's exponential and
reciprocal: 2^-21 + |a| 2^-23, with |a| < 30 below 2^-17.
"""
import numpy as np
import pytest
import torch

from oracle import layer
from oracle.formats import e4m3fn_to_f64, quantise_e4m3fn
from paper_2608_08020_amd import gambit as g

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
REL = 2.0 ** -18
HALF = {BF16: 2.0 ** -8, F32: 2.0 ** -24}


def _normal(seed, *shape, dtype=BF16):
    return torch.randn(shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).to(dtype)


def _np(t):
    return t.double().cpu().numpy()


def _values(codes):
    return e4m3fn_to_f64(codes.view(torch.uint8).cpu().numpy())


def _check_codes(codes, scale, y, rel):
    y = y.reshape(-1, y.shape[-1])
    want = layer.group_scales(y)
    got = _np(scale)
    assert got.shape == want.shape
    assert (np.abs(got - want) <= (rel + 2.0 ** -22) * want).all()
    s = np.repeat(got.T, 128, axis=1)[:, :y.shape[1]]
    err = np.abs(_values(codes).reshape(y.shape) * s - y)
    assert (err <= (2.0 ** -4 + 2 * rel) * np.abs(y) + 2.0 ** -10 * s).all()


def _check(out, y, rel=REL):
    half = HALF[out.dtype]
    err = np.abs(_np(out) - y)
    assert (err <= (rel + half) * np.abs(y) + 2.0 ** -133).all(), float((err / np.abs(y)).max())


@pytest.mark.parametrize("n,dim", [(1, 8), (3, 120), (17, 128), (5, 136), (2, 512), (3, 520), (3, 1024), (2, 1032), (4, 2048), (3, 2056),
                                   (33, 4096), (2, 4104), (2, 8192), (2, 8200), (2, 16384), (2, 16392), (2, 32768)])
@pytest.mark.parametrize("x,res,out", [(BF16, None, BF16), (BF16, BF16, F32), (F32, F32, BF16), (BF16, F32, F32), (F32, None, F32), (F32, BF16, BF16)])
def test_norm(n, dim, x, res, out):
    xt, w = _normal(n + dim, n, dim, dtype=x), 1 + _normal(2, dim, dtype=res or BF16) / 4
    r = None if res is None else _normal(3, n, dim, dtype=res) * 9
    y, h = layer.rms_norm(_np(xt), _np(w), 1e-5, None if r is None else _np(r))
    kept = None if r is None else torch.empty_like(r)
    got = g.rms_norm(xt, w, 1e-5, residual=r, residual_out=kept, out_dtype=out)
    assert got.dtype == out and got.shape == (n, dim)
    _check(got, y)
    if r is not None:
        _check(kept, h, 2.0 ** -24)


@pytest.mark.parametrize("n,heads,dim,x,res", [(1, 1, 16, BF16, None), (5, 1, 144, BF16, BF16), (3, 1, 4096, F32, BF16), (9, 1, 5120, BF16, F32),
                                               (4, 3, 128, BF16, None), (2, 1, 32752, BF16, None), (130, 1, 1008, F32, None)])
def test_norm_to_codes(n, heads, dim, x, res):
    xt = _normal(n, n, heads, dim, dtype=x) if heads > 1 else _normal(n, n, dim, dtype=x)
    w = 1 + _normal(2, dim) / 4
    r = None if res is None else _normal(3, *xt.shape, dtype=res)
    y, h = layer.rms_norm(_np(xt), _np(w), 1e-6, None if r is None else _np(r))
    codes, scale = g.rms_norm(xt, w, residual=r, out_dtype=E4M3)
    assert codes.shape == xt.shape and codes.dtype == E4M3
    _check_codes(codes, scale, y, REL)
    if r is not None:  # in place
        _check(r, h, 2.0 ** -24)


def test_norm_of_heads_within_packed_rows():
    x = _normal(4, 7, 12, 128)
    w = 1 + _normal(5, 128) / 4
    for part in (x[:, :8], x[:, 8:10], x[::2, 3:4], x.transpose(0, 1)[2:5]):
        _check(g.rms_norm(part, w), layer.rms_norm(_np(part), _np(w), 1e-6)[0])
    wide = _normal(6, 5, 300)  # rows of 300 values: not 16 bytes apart from one another, refused
    with pytest.raises(g.GambitError):
        g.rms_norm(wide[:, :128], _normal(7, 128))


def test_norm_in_place():
    x, w = _normal(8, 40, 4096), 1 + _normal(9, 4096) / 4
    y = layer.rms_norm(_np(x), _np(w), 1e-6)[0]
    assert g.rms_norm(x, w, out=x) is x
    _check(x, y)


def test_rows_of_zeros_and_of_extreme_values():
    w = torch.ones(4096, device=DEV)
    for dim in (128, 4096):
        x = _normal(10, 6, dim, dtype=F32)
        x[0] = 0
        x[1] *= 1e25       # squares leave fp32
        x[2] *= 1e37
        x[3] *= 1e-18      # below eps
        x[4] *= 1e-30      # squares vanish
        y = layer.rms_norm(_np(x), 1.0, 1e-6)[0]
        _check(g.rms_norm(x, w[:dim], out_dtype=F32), y)
        codes, scale = g.rms_norm(x, w[:dim], out_dtype=E4M3)
        _check_codes(codes, scale, y, REL)
        assert (_values(codes)[0] == 0).all()


def test_infinities_and_nan_stay_in_their_rows():
    for dim in (128, 2048):
        x = _normal(11, 5, dim)
        x[1, 3] = float("inf")
        x[3, 7] = float("nan")
        y = g.rms_norm(x, torch.ones(dim, device=DEV), out_dtype=F32)
        ref = layer.rms_norm(_np(x), 1.0, 1e-6)[0]
        assert torch.isfinite(y[[0, 2, 4]]).all() and torch.isnan(y[3]).all()
        assert torch.isnan(y[1, 3]) and (y[1, 4:] == 0).all()
        _check(y[[0, 2, 4]], ref[[0, 2, 4]])


@pytest.mark.parametrize("n,dim", [(1, 16), (3, 112), (1, 128), (67, 272), (5, 4096), (3, 12288), (300, 144)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_quantize_is_exact(n, dim, dtype):
    """Codes and scales are those of the fp32 quotients, bit for bit."""
    x = _normal(n + dim, n, dim, dtype=dtype) * torch.logspace(-9, 9, n, device=DEV)[:, None].to(dtype)
    codes, scale = g.quantize(x)
    xs = x.float().cpu().numpy()
    got = codes.view(torch.uint8).cpu().numpy()
    for b in range(-(-dim // 128)):
        part = xs[:, 128 * b:128 * b + 128]
        s = np.maximum(np.abs(part).max(1) / np.float32(448), np.float32(2.0 ** -60))
        assert np.array_equal(scale[b].cpu().numpy(), s)
        for r in range(n):
            assert np.array_equal(got[r, 128 * b:128 * b + 128], quantise_e4m3fn(part[r].astype(np.float64), s[r]))


@pytest.mark.parametrize("n,dim", [(1, 16), (5, 112), (9, 4096), (260, 144), (2, 12288)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gated(n, dim, dtype):
    x = 4 * _normal(n + dim, n, 2 * dim, dtype=dtype)
    codes, scale = g.quantize(x, gated=True)
    _check_codes(codes, scale, layer.gated(_np(x)), 2.0 ** -17)


def test_quantize_values_that_are_not_finite():
    x = torch.zeros(4, 256, device=DEV)
    x[0, 3], x[0, 4] = float("nan"), 7.0
    x[1, 5], x[1, 6] = float("inf"), -float("inf")
    x[2] = 2.0 ** -100
    codes, scale = g.quantize(x)
    v, s = _values(codes), _np(scale)
    assert np.isnan(v[0, 3]) and s[0, 0] == np.float32(7) / np.float32(448) and v[0, 4] == 448
    assert v[1, 5] == 448 and v[1, 6] == -448 and np.isfinite(s).all()
    assert (s[:, 2] == 2.0 ** -60).all() and (v[2] == 0).all() and (s[:, 3] == 2.0 ** -60).all() and (v[3] == 0).all()
    z = torch.zeros(1, 256, device=DEV)
    z[0, :4] = torch.tensor([-float("inf"), -200.0, 200.0, float("nan")], device=DEV)
    z[0, 128:] = 1
    v = _values(g.quantize(z, gated=True)[0])[0]
    assert v[0] == 0 and v[1] == 0 and v[2] == 448 and np.isnan(v[3])


def test_rows_of_other_strides():
    x = _normal(12, 9, 512)
    for part in (x[:, 128:384], x[::2, :256], x[:1].expand(5, 512)):
        codes, scale = g.quantize(part)
        c2, s2 = g.quantize(part.contiguous())
        assert torch.equal(codes.view(torch.uint8), c2.view(torch.uint8)) and torch.equal(scale, s2)


def test_no_rows():
    w = torch.ones(128, device=DEV)
    assert g.rms_norm(torch.empty(0, 128, device=DEV), w).shape == (0, 128)
    codes, scale = g.quantize(torch.empty(0, 128, device=DEV))
    assert codes.shape == (0, 128) and scale.shape == (1, 0)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_signalling_nan_counts_as_nan(dtype):
    x = _normal(3, 5, 512, dtype=dtype)
    bits = x.view(torch.int16 if dtype == BF16 else torch.int32)
    x[:, ::128] = 100.0  # a group's largest, just before it
    quiet = x.clone()
    bits[:, 1::8] = 0x7F81 if dtype == BF16 else 0x7F800001
    quiet[:, 1::8] = float("nan")
    assert torch.isnan(x[:, 1::8]).all()
    (c, s), (cq, sq) = g.quantize(x), g.quantize(quiet)
    assert torch.equal(s, sq) and torch.equal(c.view(torch.uint8), cq.view(torch.uint8)) and (s == 100 / 448).all()
    (c, s), (cq, sq) = g.quantize(x, gated=True), g.quantize(quiet, gated=True)
    assert torch.equal(s, sq) and torch.equal(c.view(torch.uint8), cq.view(torch.uint8))
    assert torch.isnan(g.rms_norm(x, torch.ones(512, device=DEV))).all()


@pytest.mark.parametrize("dim", [640, 768, 776, 1024, 4104, 5120, 6144, 8192])
def test_norm_at_other_lane_counts(dim):
    for n in (1, 3, 9):
        x, w, r = _normal(1, n, dim), _normal(2, dim, dtype=F32), _normal(3, n, dim, dtype=F32)
        y, h = layer.rms_norm(_np(x), _np(w), 1e-6, _np(r))
        out = torch.empty_like(r)
        _check(g.rms_norm(x, w, residual=r, residual_out=out, out_dtype=F32), y)
        assert np.abs(_np(out) - h).max() <= 2.0 ** -24 * np.abs(h).max()
        if dim % 16 == 0:
            _check_codes(*g.rms_norm(x, w, residual=r, residual_out=out, out_dtype=E4M3), y, REL)
