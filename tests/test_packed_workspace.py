"""What packed calls take of a pool's workspace: a caller who lowers max_splits
bounds the partials of every attention call by it, packed ones too."""
from __future__ import annotations

import os

import pytest

from oracle.pool import PoolModel
from test_packed_plan import _flat, _run, check_plan, harness  # noqa: F401  (a fixture)

PARTIAL = 4 * 128 + 8  # bytes of a partial row


def _size(T, Hq, Hkv, splits, maxb=2048, layers=1):
    from paper_2608_08020_amd import gambit
    if not os.path.exists(gambit.LIB_PATH):
        pytest.skip("libgambit.so not built")
    return gambit.workspace_size(gambit.PoolDesc(
        num_blocks=T * maxb, block_size=16, num_q_heads=Hq, num_kv_heads=Hkv, head_dim=128, kv_dtype=0, max_traces=T,
        max_blocks_per_trace=maxb, max_splits=splits, fp8_append_scale=0.0, num_layers=layers))


@pytest.mark.parametrize("T,Hq,Hkv", [(8, 32, 8), (64, 32, 8), (64, 1, 1), (512, 64, 8)])
def test_max_splits_bounds_the_partials(T, Hq, Hkv):
    one = _size(T, Hq, Hkv, 1)
    for splits in (8, 16, 64):
        # attention units of 64 bytes and a member's id besides
        least, most = T * Hq * PARTIAL * (splits - 1), T * (splits - 1) * (Hq * PARTIAL + Hkv * 2 * 64 + 4)
        # a packed plan's items grow with the partials: 64 bytes and a list entry for each of two plans
        most += T * (splits - 1) * 2 * (64 + 4) + (1 << 16)
        assert least <= _size(T, Hq, Hkv, splits) - one <= most
    assert _size(T, Hq, Hkv, 64) <= _size(T, Hq, Hkv, 0)


def test_small_pools_by_default():
    """Room for the partials of packed calls goes with the traces and heads, up to 262144 rows."""
    assert _size(8, 32, 8, 0) < 80 << 20
    assert _size(64, 1, 1, 0) < 80 << 20
    assert _size(64, 32, 8, 0) - _size(64, 32, 8, 1) < 262144 * PARTIAL + (16 << 20)


@pytest.mark.parametrize("splits", [1, 2, 5])
def test_plans_fit_few_partials(harness, splits):  # noqa: F811
    T, maxb = 4, 700
    m = PoolModel(num_blocks=T * maxb, n_kv_heads=8, head_dim=128, kv_dtype="bf16", max_traces=T, max_blocks_per_trace=maxb)
    lines = [f"create {T * maxb} 32 8 {T} {maxb} {splits} 0 1"]

    def alloc(t, n):
        m.alloc([t], [n])
        lines.append(f"alloc {t} {n}")

    alloc(0, 9000)
    m.fork([0, 0], [1, 2])
    lines.append("fork 0 1 0 2")
    alloc(3, 10000)
    calls = [([3], [1]), ([0, 1, 2, 3], [1, 2, 1, 5]), ([1, 3], [9000, 700]), ([0, 1, 2], [40, 40, 40])]
    for ids, counts in calls:
        lines.append("prompt 0 " + _flat(*zip(ids, counts)))
        lines.append(f"tree 0 {len(ids)} " + _flat(*zip(ids, [min(c, 9) for c in counts]),
                                                 [j - 1 for c in counts for j in range(min(c, 9))]))
    out = _run(harness, lines)
    assert all(o["status"] == 0 for o in out), out
    plans = out[4:]
    for (ids, counts), prompt, tree in zip(calls, plans[::2], plans[1::2]):
        for o, n, ups in ((prompt, counts, None),
                          (tree, [min(c, 9) for c in counts], [j - 1 for c in counts for j in range(min(c, 9))])):
            assert o["max_parts"] == T * splits
            check_plan(o, [list(r) for r in m.table], ids, n, 4, [int(x) for x in m.seq_len], ups)
            assert sum(k for k in o["nk"] if k > 1) <= T * splits
