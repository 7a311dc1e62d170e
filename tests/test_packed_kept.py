"""The packed-token calls' kept plans on the CPU, under sanitizers (the harness of test_packed_plan.py).

A plan is made and uploaded by the first call of a kind that lists what it
lists, used by the next ones while the pool does not change, and never
afterwards, whatever of the pool changed.
"""
from __future__ import annotations

import pytest

from oracle.pool import PoolModel
from test_packed_plan import _flat, _run, check_plan, harness  # noqa: F401  (a fixture)

T, MAXB, HQ, HKV = 6, 60, 8, 2


class Pool:
    """Lines for the harness, and the pool they make."""

    def __init__(self):
        self.m = PoolModel(num_blocks=T * MAXB, n_kv_heads=HKV, head_dim=128, kv_dtype="bf16", max_traces=T,
                           max_blocks_per_trace=MAXB)
        self.lines = [f"create {T * MAXB} {HQ} {HKV} {T} {MAXB} 0 0 2"]
        self.checks = [None]

    def _do(self, line):
        self.lines.append(line)
        self.checks.append(None)

    def alloc(self, *pairs):
        self.m.alloc([t for t, _ in pairs], [n for _, n in pairs])
        self._do("alloc " + _flat(*pairs))

    def fork(self, p, c):
        self.m.fork([p], [c])
        self._do(f"fork {p} {c}")

    def free(self, t):
        self.m.free_traces([t])
        self._do(f"free {t}")

    def uploads(self):
        self.lines.append("uploads")
        self.checks.append("uploads")

    def _state(self):
        return [list(r) for r in self.m.table], [int(x) for x in self.m.seq_len]

    def tree(self, layer, ids, ups):
        counts = [len(u) for u in ups]
        flat = [x for u in ups for x in u]
        self.lines.append(f"tree {layer} {len(ids)} " + _flat(*zip(ids, counts), flat))
        self.checks.append((self._state(), ids, counts, flat))

    def prompt(self, layer, ids, counts):
        self.lines.append(f"prompt {layer} " + _flat(*zip(ids, counts)))
        self.checks.append((self._state(), ids, counts, None))

    def write(self, layer, *triples):
        self.lines.append(f"write {layer} {sum(n for *_, n in triples)} " + _flat(*triples))
        self.checks.append((self._state(), triples))

    def run(self, exe):
        """Every call's plan against the pool as it was then; the counts of uploads."""
        ups = []
        for o, c in zip(_run(exe, self.lines), self.checks):
            assert o["status"] == 0, o
            if c == "uploads":
                ups.append(o["uploads"])
            elif c is not None and len(c) == 2:
                (rows, _), triples = c
                want, src = [], 0
                for t, a, n in triples:
                    for j in range(a // 16, -(-(a + n) // 16)):
                        r0, r1 = max(a - 16 * j, 0), min(a + n - 16 * j, 16)
                        want.append([rows[t][j], src + 16 * j + r0 - a, r0, r1])
                    src += n
                assert [x[:4] for x in o["items"]] == want
            elif c is not None:
                (rows, length), ids, counts, flat = c
                check_plan(o, rows, ids, counts, HQ // HKV, length, flat)
        return ups


TREES = ([0, 1, 3], [[-1, 0, 0], [-1], [-1, 0]])


def _calls(P, layer):
    P.tree(layer, *TREES)
    P.prompt(layer, [1, 0], [2, 40])
    P.write(layer, (1, 17, 9))


CHANGES = {
    "accepted tokens": lambda P: P.alloc((0, 2), (1, 1)),
    "tokens of a listed trace that stay inside its block": lambda P: P.alloc((1, 1)),
    "a listed trace in other blocks": lambda P: (P.free(1), P.alloc((5, 40)), P.alloc((1, 47))),
    "a fork into a listed empty slot": lambda P: P.fork(0, 3),
    "a fork of a listed trace": lambda P: P.fork(0, 4),
    "the sharer of a listed trace's blocks ends": lambda P: P.free(2),
}


@pytest.mark.parametrize("what", CHANGES)
def test_the_same_lists_after_the_pool_changed(harness, what):  # noqa: F811
    P = Pool()
    P.alloc((0, 333), (1, 47))
    P.fork(0, 2)
    _calls(P, 0)
    CHANGES[what](P)
    _calls(P, 0)
    _calls(P, 1)
    P.run(harness)


def test_each_kind_of_call_keeps_its_plan(harness):  # noqa: F811
    """A step whose layers make a write, a prompt and a tree call uploads three plans, not three a layer."""
    P = Pool()
    P.alloc((0, 333), (1, 47))
    P.uploads()
    for _ in range(3):
        for layer in (0, 1):
            _calls(P, layer)
    P.uploads()
    P.alloc((0, 1))
    P.uploads()
    for layer in (0, 1):
        _calls(P, layer)
    P.uploads()
    P.prompt(0, [1, 0], [2, 41])                       # another list of one kind
    P.prompt(1, [1, 0], [2, 41])
    P.tree(1, *TREES)
    P.uploads()
    a, b, c, d, e = P.run(harness)
    assert (b - a, d - c, e - d) == (3, 3, 1)


def test_the_largest_trees_of_every_trace_fit_their_plan(harness):  # noqa: F811
    P = Pool()
    P.alloc(*[(t, 16 * MAXB - t) for t in range(T)])
    chains = [[j - 1 for j in range(64)] for _ in range(T)]
    for _ in range(2):
        P.tree(0, list(range(T)), chains)
        P.prompt(0, list(range(T)), [16 * MAXB - t for t in range(T)])
    P.run(harness)
