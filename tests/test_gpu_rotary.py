"""Rotated queries, keys and layer writes on the GPU, against the definition in float64.

A turned value is two products and their sum in fp32: 3 2^-24 of the products'
magnitudes, and its own rounding: half a step of bf16 (2^-8) or of E4M3 (2^-4, or
2^-10 of the block's scale where codes are subnormal).
"""
import numpy as np
import pytest
import torch

from oracle import layer
from paper_2608_08020_amd import gambit as g
from test_gpu_packed import Kept

pytestmark = pytest.mark.gpu
DEV = "cuda"
D = 128
SUM = 3 * 2.0 ** -24


def _table(n_pos, rot):
    a = np.arange(n_pos)[:, None] * 1e4 ** (-2 * np.arange(rot // 2) / rot)
    return torch.from_numpy(np.concatenate([np.cos(a), np.sin(a)], 1)).to(DEV, torch.float32)


def _packed(N, hq, hkv, seed=0):
    x = torch.randn(N, hq + 2 * hkv, D, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).to(torch.bfloat16)
    return x.split([hq, hkv, hkv], 1)


def _np(t):
    return t.double().cpu().numpy()


def _turned(x, pos, table, pairs):
    return layer.turn(_np(x), _np(table[torch.as_tensor(np.asarray(pos), device=DEV).long()]), pairs)


def _check(got, ref, half=2.0 ** -8):
    y, size = ref
    err = np.abs(_np(got) - y)
    tol = SUM * size + half * (np.abs(y) + SUM * size)
    assert (err <= tol).all(), float((err / tol).max())


@pytest.mark.parametrize("n,hq,hkv", [(1, 8, 2), (5, 32, 8), (3, 3, 1), (64, 64, 8), (700, 40, 8)])
@pytest.mark.parametrize("rot,pairs", [(128, False), (128, True), (16, False), (16, True), (80, False), (112, True)])
def test_rotate(n, hq, hkv, rot, pairs):
    q, k, _ = _packed(n, hq, hkv, n)
    table = _table(1000, rot)
    pos = torch.randint(0, 1000, (n,), generator=torch.Generator().manual_seed(1)).to(DEV, torch.int32)
    qo, ko = g.rotate(q, k, pos, table, pairs=pairs)
    _check(qo, _turned(q, pos.cpu(), table, pairs))
    _check(ko, _turned(k, pos.cpu(), table, pairs))
    assert torch.equal(qo[..., rot:], q[..., rot:])


def test_rotate_in_place_and_one_side():
    q, k, _ = (t.contiguous() for t in _packed(9, 8, 2))
    table, pos = _table(50, 128), torch.arange(9, device=DEV, dtype=torch.int32) * 5
    ref = _turned(q, pos.cpu(), table, False)
    a, none = g.rotate(q, None, pos, table)
    assert none is None
    _check(a, ref)
    b, ko = g.rotate(q, k, pos, table, q_out=q)
    assert b is q and torch.equal(a, q)
    assert torch.equal(g.rotate(None, k, pos, table)[1], ko)


def test_positions_outside_the_table_give_nan():
    q, k, _ = _packed(4, 4, 1)
    pos = torch.tensor([0, -1, 9, 10], device=DEV, dtype=torch.int32)
    qo, _ = g.rotate(q, k, pos, _table(10, 64))
    assert torch.isfinite(qo[[0, 2]]).all() and torch.isnan(qo[[1, 3], :, :64]).all()
    assert torch.equal(qo[..., 64:], q[..., 64:])


def test_rotate_no_tokens():
    q, k, _ = _packed(0, 4, 1)
    qo, ko = g.rotate(q, k, torch.empty(0, device=DEV, dtype=torch.int32), _table(10, 64))
    assert qo.shape == (0, 4, D) and ko.shape == (0, 1, D)


CALLS = [  # held before, then written: per trace
    ([0, 0, 0], [1, 16, 40]),
    ([5, 16, 33, 0], [1, 16, 70, 0]),
    ([37, 3, 15, 48], [20, 1, 2, 0]),
]


@pytest.mark.parametrize("hq,hkv", [(8, 2), (32, 8), (3, 3), (80, 10)])
@pytest.mark.parametrize("rot,pairs", [(128, False), (128, True), (48, False), (16, True)])
@pytest.mark.parametrize("held,counts", CALLS)
@pytest.mark.parametrize("fp8", [False, True])
def test_write_rotated(hq, hkv, rot, pairs, held, counts, fp8):
    if hkv == 10:
        hq = 80
    T = len(held)
    s = Kept(hq, hkv, T=T, maxb=8, fp8=fp8, layers=2, seed=3)
    ids = list(range(T))
    s.pool.kv_alloc(ids, held)
    if any(held):
        s.pool.kv_write_layer(1, ids, [0] * T, held, s.normal(sum(held), hkv, D), s.normal(sum(held), hkv, D))
    before = [t.clone() for t in (s.pool.k_cache, s.pool.v_cache)]
    old = [s.tokens(i, 1, 0, held[i]) for i in ids]
    scale = s.pool.kv_scale.clone() if fp8 else None
    s.pool.kv_alloc(ids, counts)
    N = sum(counts)
    q, k, v = _packed(N, hq, hkv, 7)
    table = _table(120, rot)
    pos = np.concatenate([np.arange(a, a + c) for a, c in zip(held, counts)])
    qo = s.pool.kv_write_rotated(1, ids, held, counts, k, v, table, q=q, pairs=pairs)
    _check(qo, _turned(q, pos, table, pairs))
    y, size = _turned(k, pos, table, pairs)
    base = 0
    for i in ids:
        m = counts[i]
        kk, vv = s.tokens(i, 1, held[i], held[i] + m)
        ref = (y[base:base + m], size[base:base + m])
        if not fp8:
            _check(kk, ref)
            assert torch.equal(vv, v[base:base + m].double())
        else:
            blk = s.pool.block_table[i].cpu().numpy()[np.arange(held[i], held[i] + m) // 16]
            sc = s.cache(1)[2].cpu().numpy().astype(np.float64)
            for p in range(m):
                at, b = held[i] + p, blk[p]
                first = at // 16 * 16
                if first >= held[i]:  # the write starts the block: its scale is that of the turned keys in it
                    part = np.arange(max(first, held[i]), min(first + 16, held[i] + m)) - held[i]
                    floor = 2.0 ** -20 if first + 16 <= held[i] + m else 2.0 ** -6
                    want = max(np.abs(ref[0][part]).max() / 448, floor)
                    assert abs(sc[b, 0] - want) <= 2.0 ** -20 * want
                    want = max(float(v[base + part[0]:base + part[-1] + 1].double().abs().max()) / 448, floor)
                    assert abs(sc[b, 1] - want) <= 2.0 ** -23 * want
                else:
                    assert torch.equal(s.cache(1)[2][b], scale[1, b])
                lim = [448 * sc[b, 0], 448 * sc[b, 1]]
                for got, r, w in ((kk[p], ref[0][p], 0), (vv[p], _np(v[base + p]), 1)):
                    r = np.clip(r, -lim[w], lim[w])
                    tol = (2.0 ** -4 + 2.0 ** -20) * np.abs(r) + (2.0 ** -10 + 2.0 ** -13) * sc[b, w]
                    assert (np.abs(_np(got) - r) <= tol).all()
        base += m
    # the other layer, and what the traces held, are as they were
    for now, was in zip((s.pool.k_cache, s.pool.v_cache), before):
        assert torch.equal(now[0].view(torch.uint8), was[0].view(torch.uint8))
    if not fp8:
        for i in ids:
            for a, b in zip(s.tokens(i, 1, 0, held[i]), old[i]):
                assert torch.equal(a, b)


@pytest.mark.parametrize("fp8", [False, True])
def test_rows_pick_tokens(fp8):
    """`rows` takes the tokens of k, v and q out of larger buffers, as copies of them do."""
    rows = [7, 2, 2, 0, 9, 4]
    q, k, v = _packed(10, 8, 2, 5)
    table, out = _table(40, 64), []
    for picked in (True, False):
        s = Kept(8, 2, T=2, maxb=3, fp8=fp8)
        s.pool.k_cache.zero_()
        s.pool.v_cache.zero_()
        s.pool.kv_alloc([0, 1], [20, 4])
        if picked:
            qo = s.pool.kv_write_rotated(0, [0, 1], [16, 0], [2, 4], k, v, table, q=q, rows=rows)
        else:
            qo = s.pool.kv_write_rotated(0, [0, 1], [16, 0], [2, 4], k[rows], v[rows], table, q=q[rows])
        out.append([qo, s.pool.k_cache, s.pool.v_cache] + ([s.pool.kv_scale] if fp8 else []))
    for a, b in zip(*out):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_queries_in_place_without_queries_and_kept_plans():
    s = Kept(8, 2, T=2, maxb=4, layers=2)
    s.pool.kv_alloc([0, 1], [33, 5])
    q, k, v = (t.contiguous() for t in _packed(38, 8, 2))
    table = _table(64, 128)
    a = s.pool.kv_write_rotated(0, [0, 1], [0, 0], [33, 5], k, v, table, q=q)
    first = s.pool.k_cache[0].clone()
    # the next layer, and plain writes between them, go by the same plan
    s.pool.kv_write_layer(1, [0, 1], [0, 0], [33, 5], k, v)
    kk, _ = s.tokens(0, 1, 0, 33)
    assert torch.equal(kk, k[:33].double())
    assert s.pool.kv_write_rotated(1, [0, 1], [0, 0], [33, 5], k, v, table) is None
    assert torch.equal(s.pool.k_cache[1].view(torch.uint8), first.view(torch.uint8))
    assert s.pool.kv_write_rotated(0, [0, 1], [0, 0], [33, 5], k, v, table, q=q, q_out=q) is q
    assert torch.equal(a, q)


@pytest.mark.parametrize("bad", ["position", "rot", "shared"])
def test_refusals_leave_the_pool(bad):
    s = Kept(8, 2, T=2, maxb=4)
    s.pool.kv_alloc([0], [20])
    q, k, v = _packed(20, 8, 2)
    s.pool.kv_write_rotated(0, [0], [0], [20], k, v, _table(20, 128))
    s.pool.kv_fork([0], [1])
    was = s.pool.k_cache.clone()
    table = {"position": _table(19, 128), "rot": torch.zeros(64, 24, device=DEV), "shared": _table(20, 128)}[bad]
    ids = [0] if bad != "shared" else [1]
    if bad != "shared":
        s.pool.kv_free([1])
    with pytest.raises(g.GambitError):
        s.pool.kv_write_rotated(0, ids, [0], [20], k, v, table)
    assert torch.equal(was.view(torch.uint8), s.pool.k_cache.view(torch.uint8))


def test_values_that_are_not_finite():
    s = Kept(8, 2, T=1, maxb=2, fp8=True)
    s.pool.kv_alloc([0], [16])
    _, k, v = (t.contiguous() for t in _packed(16, 8, 2))
    k[3, 0, 5], k[4, 1, 70] = float("nan"), float("inf")
    s.pool.kv_write_rotated(0, [0], [0], [16], k, v, _table(16, 128))
    kk, _ = s.tokens(0, 0, 0, 16)
    assert torch.isnan(kk[3, 0, [5, 69]]).all()
    assert torch.isfinite(kk[[0, 1, 2] + list(range(5, 16))]).all() and torch.isfinite(s.pool.kv_scale[0]).all()


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("rot", [16, 128])
def test_signalling_nan_counts_as_nan(fp8, rot):
    got = []
    for bits in (0x7F81, 0x7FC0):
        s = Kept(8, 2, T=1, maxb=4, fp8=fp8, seed=3)
        s.pool.kv_alloc([0], [40])
        q, k, v = (t.contiguous() for t in _packed(40, 8, 2, 7))
        for t in (q, k, v):
            t[..., ::8] = 3.0  # before it
            t.view(torch.int16)[5:, :, 1::8] = bits
        qo = s.pool.kv_write_rotated(0, [0], [0], [40], k, v, _table(60, rot), q=q)
        got.append([torch.nan_to_num(qo.float(), nan=77.0)] + [torch.nan_to_num(t.float(), nan=77.0) for t in s.tokens(0, 0, 0, 40)] + ([s.pool.kv_scale] if fp8 else []))
    for a, b in zip(*got):
        assert torch.equal(a, b)
