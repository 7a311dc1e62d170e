"""Packed tokens on the GPU: every position counted once, kept plans, and fp8 steps checked in full.

Counting: with K = 0 every seen position's weight is exactly one, and V holds
7/8 at an (element, KV head) that names the position modulo 128 Hkv, zeros
elsewhere, so an output times the number of seen positions over 7/8 is a whole
number: how many of the seen positions carry that name.  7/8 is 448 times an
fp8 block's scale of 2^-9, and 56 times the 2^-6 of a block left open, so fp8
pools hold it exactly too, and a scale's logarithm, reciprocal and rounding to
bf16 are those of a power of two.  Sums, weights and the factors of the join
are then exact in the kernels; left are the reciprocal of the sum, a product
and what an instruction of one ulp may add (2^-20 for all), and a bf16
output's rounding, 2^-8.  A position left out or taken twice changes a count
by one, at least four times the bound.
"""
import numpy as np
import pytest
import torch

from oracle.attention import decode_attention
from test_gpu_packed import D, DEV, OUT, Kept, _causal, _check, _kin, _random_tree

pytestmark = pytest.mark.gpu


ONE = 0.875


def _named(lo, hi, Hkv):
    """V of positions [lo, hi): ONE at (position modulo 128, position / 128 modulo Hkv)."""
    u = torch.arange(lo, hi, device=DEV)
    v = torch.zeros(hi - lo, Hkv, D, device=DEV, dtype=torch.bfloat16)
    v[u - lo, torch.div(u, D, rounding_mode="floor") % Hkv, u % D] = ONE
    return v


def _count(out, V, sees):
    """out [m][Hq][D] against the counts of V's names among the seen positions."""
    g = out.shape[1] // V.shape[1]
    want = (sees.double() @ (V / ONE).reshape(V.shape[0], -1)).view(len(sees), V.shape[1], D).repeat_interleave(g, 1)
    rel = 2.0 ** -20 + (2.0 ** -8 if out.dtype == torch.bfloat16 else 0.0)
    assert float(want.max()) * rel < 0.25
    got = out.double() / ONE * sees.sum(1).double()[:, None, None]
    err = (got - want).abs()
    assert (err <= rel * want).all(), (float(err.max()), float(got[err > rel * want][0]), float(want[err > rel * want][0]))


def _extend(S, ids, counts):
    at = [S.pool.seq_len_of(t) for t in ids]
    v = torch.cat([_named(a, a + m, S.Hkv) for a, m in zip(at, counts)])
    S.extend(ids, counts, k=torch.zeros_like(v), v=v)


def _count_prompt(S, ids, counts, out_dtype):
    q = S.normal(sum(counts), S.Hq, D)
    out = S.pool.prompt_attn(0, ids, counts, q, out_dtype=out_dtype)
    base = 0
    for t, m in zip(ids, counts):
        if m:
            _count(out[base:base + m], S.V[t], _causal(S.V[t].shape[0], m))
        base += m


def _count_tree(S, ids, ups, out_dtype):
    counts = [len(u) for u in ups]
    N = sum(counts)
    vn = torch.cat([_named(S.pool.seq_len_of(t), S.pool.seq_len_of(t) + m, S.Hkv) for t, m in zip(ids, counts)])
    out = S.pool.tree_attn(0, ids, counts, [x for u in ups for x in u], S.normal(N, S.Hq, D), torch.zeros_like(vn), vn,
                           out_dtype=out_dtype)
    base = 0
    for t, m, up in zip(ids, counts, ups):
        if m:
            V = torch.cat([S.V[t], vn[base:base + m].double()])
            sees = torch.cat([torch.ones(m, S.V[t].shape[0], dtype=torch.bool, device=DEV), _kin(up)], 1)
            _count(out[base:base + m], V, sees)
        base += m


@pytest.mark.parametrize("out_dtype", OUT)
@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("heads,n", [((32, 8), 20011), ((8, 2), 12345), ((64, 4), 30000)])
def test_long_contexts_count_every_position_once(heads, n, fp8, out_dtype):
    S = Kept(*heads, fp8=fp8, T=2, maxb=(n + 200) // 16 + 8)
    _extend(S, [1], [n])
    _count_prompt(S, [1], [5], out_dtype)
    _count_prompt(S, [1], [131], out_dtype)
    _count_tree(S, [1], [_random_tree(np.random.default_rng(n), 21)], out_dtype)
    _extend(S, [1], [100])
    _count_prompt(S, [1], [64], out_dtype)


@pytest.mark.parametrize("out_dtype", OUT)
@pytest.mark.parametrize("fp8", [False, True])
def test_shared_prefixes_count_every_position_once(fp8, out_dtype):
    S = Kept(16, 4, fp8=fp8, T=12, maxb=400)
    _extend(S, [0, 1], [4999, 640])
    S.fork([0, 0, 0, 1, 1], [2, 3, 4, 5, 6])
    _extend(S, [2, 5, 6], [700, 16, 5])
    S.fork([2, 5], [7, 8])
    ids, counts = [8, 0, 2, 3, 5, 7, 1, 6], [3, 1, 8, 0, 20, 2, 32, 65]
    _extend(S, ids, counts)
    _count_prompt(S, ids, counts, out_dtype)
    rng = np.random.default_rng(8)
    _count_tree(S, ids, [_random_tree(rng, int(rng.integers(0, 30))) for _ in ids], out_dtype)


@pytest.mark.parametrize("fp8", [False, True])
def test_the_same_lists_after_the_pool_changed(fp8):
    """A kept plan is for the pool it was made from: the same tree and prompt lists before and after accepted tokens,
    a trace freed and made anew in other blocks, and a fork into a listed slot that was empty."""
    S = Kept(8, 2, fp8=fp8, T=6, maxb=40)
    _extend(S, [0, 1], [333, 47])
    S.V[3] = torch.zeros(0, 2, D, dtype=torch.float64, device=DEV)
    ups = [[-1, 0, 0], [-1], [-1, 0]]

    def both():
        _count_tree(S, [0, 1, 3], ups, torch.float32)
        _count_prompt(S, [1, 0], [2, 7], torch.float32)

    both()
    both()
    _extend(S, [0, 1], [2, 20])                        # the accepted tokens
    both()
    S.pool.kv_free([1])
    del S.K[1], S.V[1]
    _extend(S, [5], [64])                              # takes the blocks that trace 1 had
    _extend(S, [1], [67])                              # as long as it was, in others
    both()
    S.fork([0], [3])                                   # a listed slot that was empty
    both()
    S.pool.pool_check()


def test_the_same_write_list_after_the_pool_changed():
    S = Kept(4, 2, T=3, maxb=6)
    S.pool.kv_alloc([0], [30])
    k = S.normal(30, 2, D)
    S.pool.kv_write_layer(0, [0], [0], [30], k, k)
    S.pool.kv_free([0])
    S.pool.kv_alloc([1, 0], [20, 30])                  # trace 0 in other blocks
    S.pool.k_cache.zero_(), S.pool.v_cache.zero_()
    S.pool.kv_write_layer(0, [0], [0], [30], k, k)
    kk, vv = S.tokens(0, 0, 0, 30)
    assert torch.equal(kk, k.double()) and torch.equal(vv, k.double())
    assert all(not x.any() for x in S.tokens(1, 0, 0, 20))


def _fp8_codes(x, s):
    return (x.float() / s).clamp(-448, 448).to(torch.float8_e4m3fn).double()


def test_an_fp8_step_from_prompts_to_decode():
    """Accepted drafts in an fp8 cache attend as the definition over what the codes stand for; decode steps then
    quantise with the scale that the write left in the open block, or with the pool's in a block they open."""
    Hq, Hkv, scale = 16, 4, 2.0 ** -6
    S = Kept(Hq, Hkv, T=4, maxb=30, fp8=True, seed=4)
    S.extend([0, 1, 2], [75, 131, 16])
    pop, ups = [0, 1, 2], [[-1, 0, 1, 1], [-1, 0, 0, 2], [-1, 0]]
    path = [[0, 1, 3], [0, 2], []]
    counts, took = [4, 4, 2], [3, 2, 0]
    q, kn, vn = S.normal(10, Hq, D), S.normal(10, Hkv, D), S.normal(10, Hkv, D)
    S.pool.tree_attn(0, pop, counts, [x for u in ups for x in u], q, kn, vn)
    rows = [4 * i + j for i, p in enumerate(path) for j in p]
    at = [S.pool.seq_len_of(t) for t in pop]
    S.pool.kv_alloc(pop, took)
    S.pool.kv_write_layer(0, pop, at, took, kn, vn, rows=rows)
    for t, a, m in zip(pop, at, took):
        kk, vv = S.tokens(t, 0, a, a + m)
        S.K[t], S.V[t] = torch.cat([S.K[t], kk]), torch.cat([S.V[t], vv])
    picked = q[rows].contiguous()
    out = S.pool.prompt_attn(0, pop, took, picked, out_dtype=torch.float32)
    base = 0
    for t, m in zip(pop, took):
        if m:
            _check(out[base:base + m], picked[base:base + m], S.K[t], S.V[t], _causal(S.K[t].shape[0], m))
        base += m
    for _ in range(4):  # lengths 78, 133, 16: open blocks that writes left, and one that the first step opens
        qd, kd, vd = S.normal(3, Hq, D), S.normal(3, Hkv, D), S.normal(3, Hkv, D)
        out = S.pool.decode_attn_layer(0, pop, qd, kd, vd, new_dtype="bf16", out_dtype=torch.float32)
        for i, t in enumerate(pop):
            n = S.K[t].shape[0]
            sc = S.pool.kv_scale[int(S.pool.block_table[t, n // 16])]
            if n % 16 == 0:
                assert (sc == scale).all()
            kk, vv = S.tokens(t, 0, n, n + 1)
            assert torch.equal(kk[0], _fp8_codes(kd[i], sc[0]) * sc[0].double())
            assert torch.equal(vv[0], _fp8_codes(vd[i], sc[1]) * sc[1].double())
            S.K[t], S.V[t] = torch.cat([S.K[t], kk]), torch.cat([S.V[t], vv])
            ref = decode_attention(qd[i].double().cpu().numpy(), S.K[t].cpu().numpy(), S.V[t].cpu().numpy(), D ** -0.5)
            err = np.abs(out[i].cpu().numpy() - ref)
            assert (err <= 1e-3 + 2e-3 * np.abs(ref)).all()
    S.pool.pool_check()
