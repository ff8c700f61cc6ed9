"""The few-rows attention kernel's copies over a memory in pages: no wait can miss its phase.

A wait on a barrier's phase is by parity: it has to pass before the phase behind it completes, and must not begin before the phase
in front of it has. What has to happen before what, of the copies, the products, the warps that look V through and the softmax warps,
is a graph here; a wait is sound where the graph says both, whatever the timing. The order of the copies, their places and barriers are
the kernel's own (csrc/paged_ring.cuh, compiled for the host)."""
import os
import subprocess

import pytest

from paper_2602_06161_gb300 import build

SOURCE = r"""
#include <stdio.h>
#include "paged_ring.cuh"
using namespace cover::paged_ring;
int main(int, char** argv) {
  int n = 0;
  sscanf(argv[1], "%d", &n);
  printf("%d %d\n", kSlots, kBarriers);
  for (int i = 0; i < 2 * n; ++i) printf("%d %d %d\n", copy_at(i, n).is_v, copy_at(i, n).tile, slot_of(i));
  for (int g = 0; g < n; ++g) printf("%d %d %d %d\n", copy_of_k(g), copy_of_v(g, n), barrier_of(g), phase_of(g));
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    at = tmp_path_factory.mktemp("ring")
    (at / "ring.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-I", build.CSRC, "-o", str(at / "ring"), str(at / "ring.cpp")], check=True)
    return str(at / "ring")


def _schedule(program, n):
    rows = [[int(x) for x in line.split()] for line in subprocess.run([program, str(n)], check=True, capture_output=True,
                                                                     text=True).stdout.splitlines()]
    (slots, _), copies, tiles = rows[0], rows[1:2 * n + 1], rows[2 * n + 1:]
    return slots, copies, tiles


class Order:
    def __init__(self):
        self.after = {}

    def add(self, *chain):
        for a, b in zip(chain, chain[1:]):
            self.after.setdefault(a, set()).add(b)

    def holds(self, a, b):
        seen, todo = {a}, [a]
        while todo:
            x = todo.pop()
            if x == b:
                return True
            new = self.after.get(x, set()) - seen
            seen |= new
            todo += new
        return False


def _faults(n, slots, copies, barrier_of, screened):
    """Waits that may miss their phase. barrier_of(copy) -> (barrier, phase); screened(tile): the copies that the warps which look
    V of the tile through wait for."""
    order = Order()
    k_of, v_of = {}, {}
    for i, (is_v, tile, _) in enumerate(copies):
        (v_of if is_v else k_of)[tile] = i
    waits = []   # (event, copy)
    # copies: one warp, a place is taken when what was in it has been read by its product
    for i in range(2 * n):
        before = [("issue", i - 1)] if i else []
        if i >= slots:
            assert copies[i][2] == copies[i - slots][2]
            before.append(("pv" if copies[i - slots][0] else "s", copies[i - slots][1]))
        for b in before:
            order.add(b, ("issue", i))
        order.add(("issue", i), ("land", i))
    # products: one thread, in order
    last = None

    def then(*events):
        nonlocal last
        for e in events:
            if last is not None:
                order.add(last, e)
            last = e

    def s(g):
        waits.append((("wait k", g), k_of[g]))
        order.add(("land", k_of[g]), ("wait k", g))
        then(("wait k", g), ("s", g))

    for g in range(min(2, n)):
        s(g)
    for g in range(n):
        waits.append((("wait v", g), v_of[g]))
        order.add(("land", v_of[g]), ("wait v", g))
        order.add(("clean", g), ("pv", g))
        order.add(("weights", g), ("pv", g))
        then(("wait v", g), ("pv", g))
        if g + 2 < n:
            s(g + 2)
    # softmax: two streams, tiles in turn
    for g in range(n):
        order.add(("s", g), ("weights", g))
        if g >= 2:
            order.add(("weights", g - 2), ("weights", g))
    # the warps that look V through
    previous = None
    for g in range(n):
        for i in screened(g):
            e = ("screen", g, i)
            waits.append((e, i))
            order.add(("land", i), e)
            if previous:
                order.add(previous, e)
            previous = e
        order.add(previous, ("clean", g))
        previous = ("clean", g)
    by_phase = {}
    for i in range(2 * n):
        assert by_phase.setdefault(barrier_of(i), i) == i
    faults = []
    for event, i in waits:
        barrier, phase = barrier_of(i)
        behind, front = by_phase.get((barrier, phase + 1)), by_phase.get((barrier, phase - 1))
        if behind is not None and not order.holds(event, ("land", behind)):
            faults.append((event, behind))
        # what the waiter has done before it waits: its wait's predecessors but for the copy itself
        if front is not None and not any(order.holds(("land", front), a) for a, bs in order.after.items() if event in bs and a != ("land", i)):
            faults.append((event, front))
    # a barrier's phase begins behind the end of the one before it
    for (barrier, phase), i in by_phase.items():
        front = by_phase.get((barrier, phase - 1))
        if front is not None and not order.holds(("land", front), ("issue", i)):
            faults.append((("issue", i), front))
    return faults


@pytest.mark.parametrize("n", [1, 2, 3, 4, 5, 6, 7, 8, 9, 16, 23])
def test_no_wait_can_miss_its_phase(program, n):
    slots, copies, tiles = _schedule(program, n)
    assert [t[2] for t in copies] == [i % slots for i in range(2 * n)]
    for g, (k, v, barrier, phase) in enumerate(tiles):
        assert copies[k][:2] == [0, g] and copies[v][:2] == [1, g]
    assert sorted(c[:2] for c in copies) == sorted([v, g] for v in (0, 1) for g in range(n))
    barrier = lambda i: (("v" if copies[i][0] else "k", tiles[copies[i][1]][2]), tiles[copies[i][1]][3])  # noqa: E731
    assert _faults(n, slots, copies, barrier, lambda g: [tiles[g][1]]) == []


def test_a_barrier_a_place_can_be_missed(program):
    """Barriers that go with the places, every copy waited for by the warps that look V through: K1's place may be V2's before they look."""
    n = 6
    slots, copies, tiles = _schedule(program, n)
    first = [0] + [t[1] + 1 for t in tiles]
    faults = _faults(n, slots, copies, lambda i: (i % slots, i // slots), lambda g: list(range(first[g], tiles[g][1] + 1)))
    assert (("screen", 1, 3), 8) in faults
    assert all(e[0] == "screen" for e, _ in faults)
