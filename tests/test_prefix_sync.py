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
