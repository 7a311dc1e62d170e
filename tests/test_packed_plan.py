"""The packed-token calls' host code on the CPU, under sanitizers.

tests/host/packed_check.cpp compiles the pool's host source and the packed
calls' with g++ against a host-only HIP stand-in and prints the plans that
the calls stage.  Over random populations every plan must give each packed
token each position that it sees exactly once, through blocks that its own
row lists, with partials of its own; every refused call must say so before
anything is launched.
"""
from __future__ import annotations

import json
import os
import random
import shutil
import subprocess

import numpy as np
import pytest

from oracle.pool import PoolModel

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SRC = os.path.join(ROOT, "tests", "host", "packed_check.cpp")
INVALID, SHARED, UNSUPPORTED = -1, -3, -4
NO_LIMIT = 0x7FFFFFFF


@pytest.fixture(scope="module")
def harness(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("g++ not available")
    exe = str(tmp_path_factory.mktemp("packed") / "packed_check")
    cmd = [gxx, "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined",
           "-fno-sanitize-recover=all", "-Wno-subobject-linkage", "-I", os.path.join(ROOT, "tests", "host"), "-pthread", SRC,
           "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    return exe


def _run(exe, lines):
    r = subprocess.run([exe], input="\n".join(lines) + "\n", capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-4000:]
    return [json.loads(x) for x in r.stdout.splitlines()]


def _flat(*rows):
    return " ".join(str(x) for r in rows for x in r)


def _ancestors(up):
    out = []
    for j, u in enumerate(up):
        out.append((out[u] if u >= 0 else 0) | 1 << j)
    return out


def check_plan(plan, rows, ids, counts, g, length, ups=None):
    """rows: block rows per trace; length: positions per trace."""
    N = sum(counts)
    trace_of = [t for t, m in zip(ids, counts) for _ in range(m)]
    place = [j for m in counts for j in range(m)]
    base_of = [b for b, m in zip(np.cumsum([0] + list(counts)), counts) for _ in range(m)]
    size_of = [m for m in counts for _ in range(m)]
    sees = [length[t] if ups is not None else length[t] - m + j + 1 for t, m, j in zip(trace_of, size_of, place)]
    got = [[] for _ in range(N)]
    drafts = [0] * N
    for trace, jb0, end, tok, ntok, listed, pos0, kidx, draft, ndraft in plan["items"]:
        assert 0 < ntok * g <= 128
        toks = plan["list"][tok:tok + ntok] if listed else list(range(tok, tok + ntok))
        assert len(toks) == ntok and len(set(toks)) == ntok
        assert end <= length[trace] and 16 * jb0 <= max(end, 0) + 15
        for i, t in enumerate(toks):
            lim = end if pos0 == NO_LIMIT else min(end, pos0 + i + 1)
            assert lim <= sees[t]
            mine = rows[trace_of[t]]
            for j in range(jb0, -(-lim // 16)):
                assert rows[trace][j] == mine[j], "blocks of another trace"
            got[t].append((16 * jb0, lim, kidx))
            if draft >= 0:
                assert (draft, ndraft) == (base_of[t], size_of[t])
                drafts[t] += 1
    for k, (trace, jb0, end, _, _, listed, _, kidx, draft, _) in enumerate(plan["items"]):
        assert not listed or (kidx >= 0 and draft < 0)
        if end > 16 * jb0:
            assert plan["first"][4 * k:4 * k + 4] == [rows[trace][min(jb0 + b, (end - 1) // 16)] for b in range(4)]
    spans = []
    for t in range(N):
        at = 0
        for a, b, _ in sorted(got[t]):
            if b <= a:
                continue  # a chunk past what this row sees
            assert a == at, (t, got[t])
            at = b
        assert at == sees[t], (t, got[t], sees[t])
        assert drafts[t] == (ups is not None)
        kidx = sorted(k for *_, k in got[t])
        if plan["nk"][t] == 1:
            assert kidx == [-1]
        else:
            assert kidx == list(range(plan["nk"][t]))
            spans.append((plan["off"][t], plan["off"][t] + plan["nk"][t]))
    assert sorted(plan["merge"]) == [t for t in range(N) if plan["nk"][t] > 1]
    spans.sort()
    assert all(a[1] <= b[0] for a, b in zip(spans, spans[1:]))
    assert not spans or (spans[0][0] >= 0 and spans[-1][1] <= plan["max_parts"])
    if ups is not None:
        at, want = 0, []
        for m in counts:
            want += _ancestors(ups[at:at + m])
            at += m
        assert plan["anc"] == want


@pytest.mark.parametrize("seed", range(24))
def test_plans_cover_what_each_token_sees(harness, seed):
    rng = random.Random(seed)
    Hq, Hkv = rng.choice([(8, 2), (32, 8), (16, 1), (64, 8), (4, 4), (3, 3)])
    T, maxb = rng.choice([(3, 700), (12, 200), (40, 60)])
    nb = T * maxb
    splits = rng.choice([0, 1, 8])
    lines = [f"create {nb} {Hq} {Hkv} {T} {maxb} {splits} {seed % 2} 2"]
    m = PoolModel(num_blocks=nb, n_kv_heads=Hkv, head_dim=128, kv_dtype="bf16", max_traces=T, max_blocks_per_trace=maxb)
    checks = [None]
    for _ in range(14):
        live = [t for t in range(T) if m.seq_len[t]]
        empty = [t for t in range(T) if not m.seq_len[t]]
        if empty and rng.random() < 0.6:
            par = rng.sample(live, min(len(live), rng.randint(1, 3))) if rng.random() < 0.7 else []
            ch = rng.sample(empty, min(len(empty), max(1, 2 * len(par))))
            if par:
                par = [rng.choice(par) for _ in ch]
                m.fork(par, ch)
                lines.append("fork " + _flat(*zip(par, ch)))
            else:
                nt = [rng.randint(1, min(16 * maxb // 2, rng.choice([20, 400, 5000]))) for _ in ch]
                m.alloc(ch, nt)
                lines.append("alloc " + _flat(*zip(ch, nt)))
            checks.append(None)
        grow = [t for t in range(T) if m.seq_len[t] and rng.random() < 0.4]
        if grow:
            nt = [rng.randint(0, min(30, 16 * maxb - m.seq_len[t])) for t in grow]
            m.alloc(grow, nt)
            lines.append("alloc " + _flat(*zip(grow, nt)))
            checks.append(None)
        live = [t for t in range(T) if m.seq_len[t]]
        if not live:
            continue
        ids = rng.sample(live, rng.randint(1, len(live)))
        state = ([list(r) for r in m.table], list(m.seq_len))
        if rng.random() < 0.5:
            cap = rng.choice([1, 8, 40, 10000])
            counts = [rng.randint(0, min(cap, m.seq_len[t])) for t in ids]
            lines.append(f"prompt {rng.randrange(2)} " + _flat(*zip(ids, counts)))
            checks.append((state, ids, counts, None))
        else:
            ids += [t for t in range(T) if not m.seq_len[t]][:1]  # over no cached position
            counts = [rng.randint(0, rng.choice([1, 8, 64])) for _ in ids]
            ups = [rng.randint(-1, j - 1) for c in counts for j in range(c)]
            lines.append(f"tree {rng.randrange(2)} {len(ids)} " + _flat(*zip(ids, counts), ups))
            checks.append((state, ids, counts, ups))
    out = _run(harness, lines)
    plans = 0
    for o, c in zip(out, checks):
        assert o["status"] == 0, o
        if c is None:
            continue
        (rows, length), ids, counts, ups = c
        assert o["launched"] == (1 if sum(counts) else 0)
        if sum(counts):
            check_plan(o, rows, ids, counts, Hq // Hkv, length, ups)
            plans += 1
    assert plans > 3


def test_long_ranges_are_split_and_shared_blocks_read_once(harness):
    lines = ["create 4000 32 8 9 2100 0 0 1", "alloc 0 16000", "fork " + _flat(*[(0, t) for t in range(1, 8)]),
             "alloc 8 32000", "tree 0 8 " + _flat([(t) for k in range(8) for t in (k, 4)], [-1, 0, 1, 2] * 8),
             "prompt 0 8 16", "prompt 0 8 16", "prompt 0 8 32000"]
    out = _run(harness, lines)
    shared = [u for u in out[4]["items"] if u[5]]
    # 16000 positions = 1000 whole blocks that all eight hold: 32 tokens x 4 heads fill one tile
    assert sum(u[2] - 16 * u[1] for u in shared) == 16000 and all(u[4] == 32 for u in shared) and len(shared) > 16
    assert len(out[5]["items"]) > 16 and out[5] == out[6]
    assert len(out[7]["items"]) == 1000 and max(out[7]["nk"]) <= 2  # 32 tokens a tile


def test_write_items(harness):
    lines = ["create 100 8 2 4 20 0 1 2", "alloc 0 40 1 5 2 100", "write 1 47 0 3 37 1 4 1 2 0 0 0 0 0",
             "write 0 3 2 90 9 0 16 16 rows " + _flat([2] * 25), "free 0", "write 0 100 2 0 100"]
    out = _run(harness, lines)
    assert [o["status"] for o in out] == [0, 0, INVALID, 0, 0, 0]
    f32 = 2.0 ** -20
    assert out[3]["items"] == [[3 + 1 + 5, 0, 10, 16, 0], [3 + 1 + 6, 6, 0, 3, 2.0 ** -6], [1, 9, 0, 16, pytest.approx(f32)]]
    assert len(out[5]["items"]) == 7 and out[5]["items"][6][2:4] == [0, 4]


def test_refusals(harness):
    T = 6
    lines, want = ["create 200 32 8 6 20 0 0 2", "alloc 0 40 1 20 2 32", "fork 0 3"], [0, 0, 0]

    def refuse(line, status):
        lines.append(line)
        want.append(status)

    for call in ("prompt {} 0 5", "tree {} 1 0 2 -1 0", "write {} 5 0 35 5"):
        refuse(call.format(2), INVALID)            # layers are 0 and 1
        refuse(call.format(-1), INVALID)
    refuse("prompt 0 0 5 0 5", INVALID)            # the same trace twice
    refuse("prompt 0 6 5", INVALID)
    refuse("prompt 0 0 -1", INVALID)
    refuse("prompt 0 0 41", INVALID)               # more than it holds
    refuse("prompt 0 5 1", INVALID)                # an empty trace
    refuse("tree 0 1 0 65 " + _flat([-1] * 65), UNSUPPORTED)
    refuse("tree 0 1 0 2 -1 1", INVALID)           # its own parent
    refuse("tree 0 1 0 2 -1 2", INVALID)           # a later node
    refuse("tree 0 1 0 2 -2 0", INVALID)
    refuse("tree 0 2 0 2 1 2 -1 0 -1 2", INVALID)  # a parent past the second tree
    refuse("write 0 41 0 0 41", INVALID)           # outside the trace
    refuse("write 0 2 0 -1 2", INVALID)
    refuse("write 0 4 1 0 5", INVALID)             # fewer rows than tokens
    refuse("write 0 3 1 0 5 rows 0 1 2 3 0", INVALID)
    refuse("write 0 3 1 0 5 rows 0 1 -1 2 0", INVALID)
    refuse("write 0 1 0 31 1", SHARED)             # a block that the fork shares
    refuse("write 0 2147483647 2 1 2147483647", UNSUPPORTED)
    for bad in ("capturing 1", "device 1"):
        lines.append(bad), want.append(0)
        for call in ("prompt 0 0 5", "tree 0 1 0 2 -1 0", "write 0 5 0 35 5"):
            refuse(call, UNSUPPORTED if bad[0] == "c" else INVALID)
        lines.append(bad[:-1] + "0"), want.append(0)
    lines.append("decode 1 2"), want.append(0)     # layer 0 of 2: a step is open
    for call in ("prompt 0 0 5", "tree 0 1 0 2 -1 0", "write 0 5 0 35 5"):
        refuse(call, INVALID)
    lines.append("decode 1 2"), want.append(0)
    n0 = len(lines)
    lines += ["prompt 0", "prompt 0 0 0 1 0", "tree 0 0", "tree 1 2 0 0 5 0", "write 0 0", "write 0 0 0 0 0 2 3 0",
              "prompt 1 0 5", "tree 0 1 5 3 -1 -1 0", "write 0 1 0 32 1"]
    out = _run(harness, lines)
    assert [o["status"] for o in out[:n0]] == want
    assert all(o.get("launched", 0) == 0 for o in out[:n0])
    # calls of no tokens do nothing; the others go through
    assert [(o["status"], o["launched"]) for o in out[n0:]] == [(0, 0)] * 6 + [(0, 1)] * 3
