"""The prefix kernel's rules of waiting, from its own header, in every order in which its warps can
come (no GPU): a small program writes down what each warp does over a list of segments, and a search
walks all interleavings."""
import itertools
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2412_12094_b200", "csrc")

TURNS = r"""
#include <cstdio>
#include <cstdlib>
#include "prefix_sync.h"
// arguments: key tiles of slot 0 and of slot 1, segment by segment
int main(int argc, char** argv) {
  for (int x = 0; x < 2; ++x, std::printf("\n"))
    for (int i = 1; i + 1 < argc; i += 2) {
      const int n[2] = {std::atoi(argv[i]), std::atoi(argv[i + 1])}, both = n[0] < n[1] ? n[0] : n[1];
      for (int j = 0; j < n[x]; ++j) {
        if (sepllm::turn_waits(x, j, both)) std::printf("s%d ", x);
        if (j < both) std::printf("b0 e0 ");
        if (sepllm::turn_passes(j, both)) std::printf("a%d ", x ^ 1);
      }
      if (sepllm::turn_returns(x, both)) std::printf("s%d ", x);
    }
}
"""


def _compile(tmp, name, text):
    src, exe = tmp / (name + ".cpp"), tmp / name
    src.write_text(text)
    subprocess.run(["g++", "-std=c++17", "-I", CSRC, "-o", str(exe), str(src)], check=True)
    return str(exe)


@pytest.fixture(scope="module")
def turns(tmp_path_factory):
    exe = _compile(tmp_path_factory.mktemp("turns"), "turns", TURNS)

    def ops(segments):
        args = [str(n) for s in segments for n in s]
        out = subprocess.run([exe] + args, check=True, capture_output=True, text=True).stdout
        return [line.split() for line in out.split("\n")[:2]]
    return ops


def _walk(ops):
    """All interleavings of two warps.  A barrier completes with two arrivals, and each pair has to be one
    warp that waits and the other that hands over: a second hand-over before the first was taken would
    complete it without the waiter."""
    seen, todo = set(), [(0, 0, (None, None), (None, None))]    # places, warp that arrived, barrier waited at
    ended = False
    while todo:
        state = todo.pop()
        if state in seen:
            continue
        seen.add(state)
        pcs, pending, blocked = state[:2], state[2], state[3]
        if all(pcs[x] == len(ops[x]) for x in (0, 1)) and blocked == (None, None):
            assert pending == (None, None), "a hand-over that nobody took"
            ended = True
            continue
        moved = False
        for x in (0, 1):
            if blocked[x] is not None or pcs[x] == len(ops[x]):
                continue
            moved = True
            op, bar = ops[x][pcs[x]][0], int(ops[x][pcs[x]][1])
            pc = list(pcs)
            pc[x] += 1
            pend, block = list(pending), list(blocked)
            if op == "b":       # the other warp is not between its b and its e
                other = x ^ 1
                assert pcs[other] == 0 or ops[other][pcs[other] - 1][0] != "b", "both slots at the exponentials"
            elif op == "e":
                pass
            elif pend[bar] is None:
                pend[bar] = x
                block[x] = bar if op == "s" else None
            else:
                assert pend[bar] != x, f"barrier {bar} completed by slot {x} alone"
                pend[bar] = None
                if block[x ^ 1] == bar:
                    block[x ^ 1] = None
                else:
                    assert op == "s", f"barrier {bar} completed by two hand-overs"
            todo.append((pc[0], pc[1], tuple(pend), tuple(block)))
        assert moved, f"both slots wait: {state}"
    assert ended


SEGMENTS = [[(1, 1)] * n for n in (1, 2, 3, 5)] + [[(2, 1), (1, 2), (1, 1)], [(3, 3), (1, 0), (2, 2)],
                                                  [(0, 2), (1, 1), (1, 1)], [(4, 2), (2, 4), (1, 3), (5, 5)]]
SEGMENTS += [list(s) for s in itertools.product([(1, 1), (2, 1), (1, 2), (0, 1), (2, 2)], repeat=3)]


@pytest.mark.parametrize("segments", SEGMENTS, ids=str)
def test_turns_are_handed_over_one_at_a_time(turns, segments):
    _walk(turns(segments))


CLEARS = r"""
#include <cstdio>
#include <cstdlib>
#include "prefix_sync.h"
// arguments: alternate mode; then key tiles of slot 0 and slot 1 (in alternate mode of both together, and
// 0), segment by segment.  Every segment ends inside its last tile.
int main(int argc, char** argv) {
  const bool alt = std::atoi(argv[1]);
  int ph_z[2] = {0, 0}, ph_g[2] = {0, 0};
  for (int who = 0; who < 3; ++who, std::printf("\n"))
    for (int i = 2; i + 1 < argc; i += 2) {
      const int a = std::atoi(argv[i]), b = std::atoi(argv[i + 1]), n = a > b ? a : b, seg = i / 2 - 1;
      const int mine[2] = {alt ? (n + 1) / 2 : a, alt ? n / 2 : b};
      if (who < 2) {
        if (!sepllm::uses_last(alt, who, n, mine[who])) continue;
        std::printf("ask%d:%d answer%d:%d use:%d ", who, seg, who, ph_z[who], seg);
        ph_z[who] ^= 1;
      } else {
        for (int x = 0; x < 2; ++x)
          if (sepllm::uses_last(alt, x, n, mine[x])) {
            std::printf("request%d:%d ", x, ph_g[x]);
            ph_g[x] ^= 1;
          }
        std::printf("clear:%d ", seg);
        for (int x = 0; x < 2; ++x)
          if (sepllm::uses_last(alt, x, n, mine[x])) std::printf("done%d:0 ", x);
      }
    }
}
"""


@pytest.fixture(scope="module")
def clears(tmp_path_factory):
    exe = _compile(tmp_path_factory.mktemp("clears"), "clears", CLEARS)

    def ops(alt, segments):
        args = [str(int(alt))] + [str(n) for s in segments for n in s]
        out = subprocess.run([exe] + args, check=True, capture_output=True, text=True).stdout
        return [[(w.split(":")[0], int(w.split(":")[1])) for w in line.split()] for line in out.split("\n")[:3]]
    return ops


def _walk_clears(ops):
    """All interleavings of the slots' issuers and the clearing warp over barriers of one arrival: a wait for
    parity p passes when the phase under way has the other parity.  Nothing else holds them in step."""
    todo, seen = [((0, 0, 0), (0, 0), (0, 0))], set()    # places, phases complete of requests and of answers
    ended = False
    while todo:
        state = todo.pop()
        if state in seen:
            continue
        seen.add(state)
        pcs, asked, answered = state
        done = [set(n for op, n in ops[w][:pcs[w]] if op == name) for w, name in ((0, "ask0"), (1, "ask1"), (2, "clear"))]
        moved = False
        for w in range(3):
            if pcs[w] == len(ops[w]):
                continue
            op, n = ops[w][pcs[w]]
            x, a, z = int(op[-1]) if op[-1].isdigit() else 0, list(asked), list(answered)
            if op[:-1] == "ask":
                a[x] += 1
            elif op[:-1] == "done":
                z[x] += 1
            elif op[:-1] == "answer":
                if z[x] % 2 == n:
                    continue
            elif op[:-1] == "request":
                if a[x] % 2 == n:
                    continue
            elif op == "clear":
                assert n in done[0] | done[1], f"segment {n} cleared before it was asked for"
            elif op == "use":
                assert n in done[2], f"segment {n} used before it was cleared"
            moved = True
            todo.append((tuple(p + (v == w) for v, p in enumerate(pcs)), tuple(a), tuple(z)))
        if not moved:
            assert all(pcs[w] == len(ops[w]) for w in range(3)), f"all wait: {state}"
            ended = True
    assert ended


CLEAR_SEGMENTS = [list(s) for s in itertools.product([(1, 2), (2, 1), (2, 2)], repeat=4)]


@pytest.mark.parametrize("segments", CLEAR_SEGMENTS, ids=str)
def test_rows_behind_the_prefix_are_cleared_before_they_are_used(clears, segments):
    _walk_clears(clears(False, segments))


@pytest.mark.parametrize("segments", [list(s) for s in itertools.product([(1, 0), (2, 0), (5, 0)], repeat=3)], ids=str)
def test_they_are_in_alternate_mode(clears, segments):
    _walk_clears(clears(True, segments))
