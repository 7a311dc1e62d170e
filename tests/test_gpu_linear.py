"""Products in E4M3 with scales of 128 on the GPU, against the definition in float64.

Products of codes are exact in fp32.  With S the sum of all magnitudes: a
block's 128 products are added in the matrix unit, fp32 output with 2^-23 of
their magnitudes' sum an addition.  For bf16 output the unit aligns groups of
eight products to the largest of a group and drops what lies 13 bits below, so
that the seven others lose at most 7 2^-13 of the largest, which the group's magnitudes
hold: 7 2^-13 S more.  Blocks are added in fp32 with two roundings each (factor,
fused addition), eight waves' sums at the end, (2 blocks + 10) 2^-24 S; then the
output's half step.
"""
import numpy as np
import pytest
import torch

from oracle import layer
from paper_2608_08020_amd import gambit as g

pytestmark = pytest.mark.gpu
DEV = "cuda"
E4M3 = torch.float8_e4m3fn
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def _inputs(m, n, k, seed=0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    kb, nb = -(-k // 128), -(-n // 128)
    x, w = ((100 * torch.randn(r, k, generator=gen, device=DEV)).clamp(-448, 448).to(E4M3) for r in (m, n))
    xs, ws = (torch.rand(s, generator=gen, device=DEV) + 0.1 for s in ((kb, m), (nb, kb)))
    return x, xs, w, ws


def _check(out, x, xs, w, ws):
    y, size = layer.linear(*(t.double().cpu().numpy() for t in (x, xs, w, ws)))
    unit = 128 * 2.0 ** -23 + (7 * 2.0 ** -13 if out.dtype == torch.bfloat16 else 0)
    tol = (unit + (2 * xs.shape[0] + 10) * 2.0 ** -24) * size + HALF[out.dtype] * np.abs(y)
    err = np.abs(out.double().cpu().numpy() - y)
    assert (err <= tol).all(), float((err / tol).max())


@pytest.mark.parametrize("m,n,k", [(1, 1, 16), (1, 16, 128), (3, 17, 144), (7, 33, 112), (16, 100, 1024), (17, 130, 1040), (31, 64, 2048), (33, 257, 1152),
                                   (64, 48, 8192), (65, 61, 256), (100, 129, 528), (128, 200, 1136), (129, 128, 128), (130, 257, 272), (200, 131, 1024),
                                   (300, 500, 640), (257, 384, 16)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_linear(m, n, k, dtype):
    args = _inputs(m, n, k, m + n + k)
    out = g.linear_fp8(*args, out_dtype=dtype)
    assert out.shape == (m, n) and out.dtype == dtype
    _check(out, *args)


@pytest.mark.parametrize("m,n,k", [(5, 16500, 256), (20, 16401, 384), (50, 16640, 272), (90, 16384, 128), (2100, 8195, 400), (4100, 4103, 144)])
def test_linear_of_many_features_or_tokens(m, n, k):
    args = _inputs(m, n, k, 1)
    out = g.linear_fp8(*args, out_dtype=torch.float32)
    rows = torch.randperm(m, generator=torch.Generator().manual_seed(2))[:64].to(DEV)
    rows = torch.cat([rows, torch.tensor([0, m - 1], device=DEV)])
    x, xs, w, ws = args
    _check(out[rows], x[rows], xs[:, rows], w, ws)


def test_every_row_and_feature_stands_for_itself():
    """NaN in one row of each operand reaches that row's and that feature's outputs alone."""
    for m, n in ((5, 40), (40, 70), (130, 300), (600, 260)):
        x, xs, w, ws = _inputs(m, n, 256)
        clean = g.linear_fp8(x, xs, w, ws)
        x.view(torch.uint8)[m // 2, 200] = 0x7F
        w.view(torch.uint8)[n - 1, 3] = 0x7F
        out = g.linear_fp8(x, xs, w, ws)
        nan = torch.zeros_like(out, dtype=torch.bool)
        nan[m // 2] = True
        nan[:, n - 1] = True
        assert torch.equal(torch.isnan(out), nan)
        assert torch.equal(out[~nan], clean[~nan])


def test_rows_do_not_depend_on_their_neighbours():
    """Within one choice of kernel, a token's outputs are the same bits whatever the other tokens are."""
    x, xs, w, ws = _inputs(700, 512, 1024)
    a = g.linear_fp8(x, xs, w, ws)
    p = torch.randperm(700, generator=torch.Generator().manual_seed(1)).to(DEV)
    assert torch.equal(g.linear_fp8(x[p], xs[:, p].contiguous(), w, ws), a[p])
    assert torch.equal(g.linear_fp8(x, xs, w, ws), a)


def test_output_given_and_no_tokens():
    x, xs, w, ws = _inputs(9, 24, 128)
    out = torch.full((9, 24), 7.0, device=DEV)
    assert g.linear_fp8(x, xs, w, ws, out=out) is out
    _check(out, x, xs, w, ws)
    assert g.linear_fp8(x[:0], xs[:, :0], w, ws).shape == (0, 24)


def test_after_quantize():
    """Rows straight from quantize: the product is that of the values the codes stand for."""
    gen = torch.Generator(device=DEV).manual_seed(5)
    v = torch.randn(37, 400, generator=gen, device=DEV).to(torch.bfloat16)
    x, xs = g.quantize(v)
    _, _, w, ws = _inputs(1, 200, 400)
    _check(g.linear_fp8(x, xs, w, ws, out_dtype=torch.float32), x, xs, w, ws)


@pytest.mark.parametrize("m,n,k", [(8, 8193, 144), (16, 8224, 1040), (17, 16383, 528), (32, 16384, 272), (33, 8191, 656), (64, 8192, 400), (128, 8188, 144), (129, 8191, 272),
                                   (1300, 4096, 272), (1300, 4099, 400), (4096, 4096, 128), (4100, 4103, 272), (4090, 4104, 656)])
def test_where_one_kernel_ends_and_the_next_begins(m, n, k):
    args = _inputs(m, n, k, 3)
    out = g.linear_fp8(*args)
    gen = torch.Generator().manual_seed(2)
    rows = torch.cat([torch.randperm(m, generator=gen)[:40], torch.tensor([0, m - 1])]).to(DEV)
    x, xs, w, ws = args
    _check(out[rows], x[rows], xs[:, rows], w, ws)
    if m > 64:  # every row, in some features
        at = (n - 1) // 128 * 128
        _check(out[:, at:], x, xs, w[at:], ws[at // 128:])


@pytest.mark.parametrize("m", [1, 9, 16, 40])
@pytest.mark.parametrize("k", [16, 496, 512, 528, 1536, 2064, 4096, 6160])
def test_stages_of_k(m, k):
    for n in (72, 8320):
        args = _inputs(m, n, k, 5)
        for dtype in (torch.bfloat16, torch.float32):
            _check(g.linear_fp8(*args, out_dtype=dtype), *args)


@pytest.mark.parametrize("m,n", [(3, 40), (40, 130), (50, 16400), (300, 260), (1300, 4096), (4096, 4104)])
def test_nothing_behind_the_outputs_is_written(m, n):
    args = _inputs(m, n, 272, 6)
    for dtype in (torch.bfloat16, torch.float32):
        whole = torch.full(((m + 2) * n,), 7.0, dtype=dtype, device=DEV)
        lead = 16 // whole.element_size()
        out = whole[lead:lead + m * n].view(m, n)
        g.linear_fp8(*args, out=out)
        assert (whole[:lead] == 7).all() and (whole[lead + m * n:] == 7).all()
        assert torch.equal(out, g.linear_fp8(*args, out_dtype=dtype))


@pytest.mark.parametrize("m,n,k", [(150, 6144, 272), (1024, 2048, 144), (1025, 2048, 400), (513, 4099, 272), (129, 16, 1040)])
def test_tiles_of_half_the_tokens(m, n, k):
    args = _inputs(m, n, k, 7)
    out = g.linear_fp8(*args)
    x, xs, w, ws = args
    at = (n - 1) // 128 * 128
    _check(out[:, at:], x, xs, w[at:], ws[at // 128:])
    rows = torch.tensor([0, 63, 64, m // 2, m - 1], device=DEV)
    _check(out[rows], x[rows], xs[:, rows], w, ws)


@pytest.mark.parametrize("m", [1, 16])
@pytest.mark.parametrize("n", [16385, 65536, 65537])
def test_few_tokens_and_many_features(m, n):
    args = _inputs(m, n, 400, 8)
    for dtype in (torch.bfloat16, torch.float32):
        _check(g.linear_fp8(*args, out_dtype=dtype), *args)
