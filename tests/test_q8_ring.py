"""The arrival barriers of the converting groups (csrc/stq_q8_ring.h) under every order of events (no GPU).

The model: a copying warp loads stage i once slot i % slots is free; copies land in any order, each completing a phase of
its barrier; group i % groups converts stage i once a wait by parity succeeds; the products take converted stages in order
and free their slots.  A wait by parity succeeds when the latest completed phase has the parity asked for.  All states that
any order of these steps can reach are visited."""
import ctypes as C
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SHAPES = [(2, 2), (3, 2), (4, 2), (5, 2), (6, 2), (4, 3), (5, 3)]


def explore(slots, groups, stages, bar, parity, waits):
    """Runs through all reachable states.  waits(group, i): whether the group waits for stage i's arrival.  Returns
    "ok", "early" (a group converted a stage that had not landed) or "stuck"."""
    def completed(landed, b):
        return sum(1 for i in range(stages) if bar(i) == b and landed >> i & 1)

    start = (0, 0, (0,) * groups, 0, 0)      # stages loaded, landed, next stage of each group, converted, products done
    seen, todo = {start}, [start]
    while todo:
        loaded, landed, at, converted, done = todo.pop()
        nexts = []
        if loaded < stages and loaded < done + slots:
            nexts.append((loaded + 1, landed, at, converted, done))
        for i in range(loaded):
            if not landed >> i & 1:
                nexts.append((loaded, landed | 1 << i, at, converted, done))
        for g in range(groups):
            i = at[g]
            while i < stages and not waits(g, i):
                i += 1
            if i >= stages:
                continue
            phases = completed(landed, bar(i))
            if phases == 0 and parity(i) == 0 or phases and (phases - 1) & 1 != parity(i):
                continue                      # (a fresh barrier counts as having completed a phase of parity 1)
            own = i % groups == g
            if own and not landed >> i & 1:
                return "early"
            nexts.append((loaded, landed, at[:g] + (i + 1,) + at[g + 1:], converted | (1 << i if own else 0), done))
        if done < stages and converted >> done & 1 and landed >> done & 1:
            nexts.append((loaded, landed, at, converted, done + 1))
        if not nexts and done < stages:
            return "stuck"
        for s in nexts:
            if s not in seen:
                seen.add(s)
                todo.append(s)
    return "ok"


@pytest.fixture(scope="module")
def ring(tmp_path_factory):
    d = tmp_path_factory.mktemp("ring")
    body = "".join(f"""
  if (slots == {s} && groups == {g}) {{
    using R = stq::ArrivalRing<{s}, {g}>;
    return what == 0 ? R::kBars : what == 1 ? R::bar(i) : R::parity(i);
  }}""" for s, g in SHAPES)
    src = d / "ring.cpp"
    src.write_text('#include "stq_q8_ring.h"\nextern "C" unsigned ring(int slots, int groups, int what, unsigned i) {' + body + "\n  return ~0u;\n}\n")
    lib = str(d / "ring.so")
    subprocess.check_call(["g++", "-std=c++17", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2604_06836_b200", "csrc"), "-o", lib, str(src)])
    f = C.CDLL(lib).ring
    f.restype = C.c_uint
    return f


@pytest.mark.parametrize("slots,groups", SHAPES)
def test_no_order_of_events_makes_a_group_miss_a_phase(ring, slots, groups):
    stages = 2 * ring(slots, groups, 0, 0) + 3
    assert explore(slots, groups, stages, lambda i: ring(slots, groups, 1, i), lambda i: ring(slots, groups, 2, i),
                   lambda g, i: i % groups == g) == "ok"
    assert ring(slots, groups, 0, 0) <= slots * groups


def test_the_model_tells_a_ring_that_can_fail():
    """A barrier to a slot, five slots, two groups: a group that waits for its own stages alone takes an old phase for the
    one it needs; one that waits for every stage can be passed by."""
    bar, parity = lambda i: i % 5, lambda i: i // 5 & 1
    assert explore(5, 2, 13, bar, parity, lambda g, i: i % 2 == g) == "early"
    assert explore(5, 2, 13, bar, parity, lambda g, i: True) == "stuck"
    assert explore(4, 2, 11, lambda i: i % 4, lambda i: i // 4 & 1, lambda g, i: i % 2 == g) == "ok"
