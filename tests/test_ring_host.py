"""The rounds that a ring's producer looks after before it leaves (csrc/ring.h), against a model of the stages' barriers:
whatever may be in flight is waited for, and no wait is for a phase that cannot come."""
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_23296_b200", "csrc")
PROGRAM = """
#include <cstdio>
#include "ring.h"
int main() {
    for (int stages = 1; stages <= 5; ++stages)
        for (int it = 0; it <= 14; ++it)
            for (int ended = 0; ended < 2; ++ended) {
                const ring_rounds r = ring_in_flight(it, stages, ended);
                std::printf("%d %d %d %d %d\\n", stages, it, ended, r.first, r.end);
            }
}
"""


@pytest.fixture(scope="module")
def in_flight(tmp_path_factory):
    at = tmp_path_factory.mktemp("ring")
    (at / "ring.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-I", CSRC, "-o", str(at / "ring"), str(at / "ring.cpp")], check=True)
    out = subprocess.run([str(at / "ring")], check=True, capture_output=True, text=True).stdout
    rows = [tuple(map(int, line.split())) for line in out.splitlines()]
    return {r[:3]: range(r[3], r[4]) for r in rows}


@pytest.mark.parametrize("stages", [1, 2, 3, 4, 5])
def test_rounds_in_flight_when_the_producer_leaves(in_flight, stages):
    seen = set()
    for rounds in range(0, 13):                       # data rounds; round number `rounds` is the end
        for consumed in range(0, rounds + 1):         # the consumers give up on round `consumed` (or get to the end)
            # round i is issued once round i - stages has been consumed
            issued = min(rounds, consumed + stages)
            ended = issued == rounds and rounds - stages < consumed
            span = in_flight[stages, issued, int(ended)]
            seen.add((issued, ended))
            may_fly = set(range(consumed, issued))
            assert may_fly <= set(span), (rounds, consumed)
            for i in span:
                # phases of the stage, in order: its data rounds, and the end
                armed = [r for r in range(issued + (1 if ended else 0)) if r % stages == i % stages]
                assert armed[-1] == i, (rounds, consumed, i)      # nothing later in that stage: the parity is that phase's
                assert len(armed) - 1 == i // stages
    assert len(seen) > 12


def test_the_decode_looks_after_them_on_every_way_out():
    # the 8-bit decode's producer leaves its loop at one place, behind which the rounds of ring_in_flight are waited for
    with open(os.path.join(CSRC, "decode_q8.cu")) as f:
        producer = f.read().split("// Descriptors and page ids run kAhead rounds")[1].split("if (warp == kMerger)")[0]
    loop, after = producer.split("ring_in_flight(")
    assert "return" not in loop and "mbar_drain(" in after and "if (dead)" not in loop + after
