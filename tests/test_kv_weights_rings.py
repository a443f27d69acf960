"""How far the warps of the kernels for attention weights of many rows may be ahead of one another: the arithmetic of
csrc/kv_weights_rings.cuh, compiled for the host and walked through in every order in which the warps that decode keys, the one that issues the
products, and those of the two halves that read them out can take their steps.  No order may get stuck, no wait may return for another
phase than its own, and what is said about a tile of keys stays until both halves have read it."""
import ctypes
import random
import subprocess
from pathlib import Path

import pytest

CSRC = Path(__file__).resolve().parent.parent / "paper_2011_09398_b200" / "csrc"

MODEL = """
#include <stdlib.h>
#include <unordered_set>
#include <vector>
#include "kv_weights_rings.cuh"
using namespace lce;

enum { FINE, STUCK, TOO_EARLY, OVERWRITTEN };

// Products are done as they are issued, and rows of q always there: whatever takes longer only holds the others back.
struct State {
    uint16_t decoded;               // tiles of keys (first kernel) or halves of units (second) that are said something about
    uint8_t unit, step, half, wait; // of the issuer: what it does next, and whether it is through with the waits before it
    uint16_t issued[2];             // steps of each half
    uint16_t streamed;              // steps
    uint16_t looked[2], read[2];    // steps of which a half has read what is said about the keys; that it has read out
    bool operator==(const State &o) const
    {
        return decoded == o.decoded && unit == o.unit && step == o.step && half == o.half && wait == o.wait && issued[0] == o.issued[0] && issued[1] == o.issued[1] &&
               streamed == o.streamed && looked[0] == o.looked[0] && looked[1] == o.looked[1] && read[0] == o.read[0] && read[1] == o.read[1];
    }
};
struct Hash {
    size_t operator()(const State &s) const
    {
        size_t h = 0;
        for (size_t v : {(size_t)s.decoded, (size_t)s.unit, (size_t)s.step, (size_t)s.half, (size_t)s.wait, (size_t)s.issued[0], (size_t)s.issued[1], (size_t)s.streamed, (size_t)s.looked[0],
                         (size_t)s.looked[1], (size_t)s.read[0], (size_t)s.read[1]})
            h = (h ^ v) * 0x9E3779B97F4A7C15ull + (h >> 29);
        return h;
    }
};
struct Unit { int halves, steps; };
struct Said { uint32_t tile, unit, half; };   // what one entry is about; the first kernel's are for both halves

struct Model {
    bool second;
    std::vector<Unit> units;
    bool rule;                          // units without a second half wait for it
    std::vector<Said> said;
    std::vector<Said> seen[2];          // by the half's steps: the entry it needs
    std::vector<uint32_t> first_of;     // entries of the units in front (second kernel)

    void prepare()
    {
        uint32_t tile = 0;
        for (uint32_t u = 0; u < units.size(); ++u) {
            first_of.push_back(said.size());
            if (second)
                for (int h = 0; h < units[u].halves; ++h) said.push_back({0, u, (uint32_t)h});
            for (int i = 0; i < units[u].steps; ++i, ++tile) {
                if (!second) said.push_back({tile, u, 0});
                for (int h = 0; h < units[u].halves; ++h) seen[h].push_back(second ? Said{0, u, (uint32_t)h} : Said{tile, u, 0});
            }
        }
        first_of.push_back(said.size());
    }
    uint32_t place(const Said &s) const { return info_place(second, s.tile, s.unit, s.half); }
    static bool same(const Said &a, const Said &b) { return a.tile == b.tile && a.unit == b.unit && a.half == b.half; }
    // a wait for a step on the barrier that its half's steps share by twos, `done` steps of which are finished
    static bool passes(uint32_t done, uint32_t step, bool *wrong)
    {
        uint32_t phases = 0;
        for (uint32_t s = 0; s < done; ++s) phases += step_buffer(s) == step_buffer(step);
        const bool pass = (phases & 1) != step_parity(step);
        if (pass && phases <= step / 2) *wrong = true;
        return pass;
    }

    int walk(int64_t *states)
    {
        prepare();
        std::unordered_set<State, Hash> met;
        std::vector<State> stack{State{}};
        met.insert(stack[0]);
        bool wrong = false, overwritten = false;
        while (!stack.empty() && !wrong && !overwritten) {
            const State s = stack.back();
            stack.pop_back();
            int ways = 0;
            bool end = true;
            const auto go = [&](const State &n) {
                ++ways;
                if (met.insert(n).second) stack.push_back(n);
            };
            if (s.decoded < said.size()) {  // two tiles ahead of the products, or two units
                end = false;
                const Said &w = said[s.decoded];
                if (second ? w.unit < 2 || s.unit > w.unit - 2 : s.decoded < 2 || s.streamed > s.decoded - 2) {
                    for (int h = 0; h < 2; ++h)  // whoever still needs the entry whose place this takes
                        for (size_t i = s.looked[h]; i < seen[h].size(); ++i) {
                            bool there = false;
                            for (int e = 0; e < s.decoded; ++e) there = there || same(said[e], seen[h][i]);
                            if (there && place(seen[h][i]) == place(w) && !same(seen[h][i], w)) overwritten = true;
                        }
                    State n = s;
                    ++n.decoded;
                    go(n);
                }
            }
            if (s.unit < units.size()) {
                end = false;
                const Unit &u = units[s.unit];
                const uint32_t steps[2] = {s.issued[0], s.issued[1]};
                const auto wait = [&](int half, uint32_t step) { return passes(s.read[half], step, &wrong); };
                bool pass = true;
                State n = s;
                if (s.wait == 0) {  // in front of a unit, then of a step
                    if (s.step == 0 && s.half == 0) {
                        if (rule) pass = before_unit(u.halves, steps, wait);
                        if (second) pass = pass && s.decoded >= first_of[s.unit + 1];
                    }
                    if (!second && s.half == 0) pass = pass && s.decoded > s.streamed;
                    n.wait = 1;
                } else {
                    pass = before_step(s.half, steps, wait);
                    n.wait = 0;
                    ++n.issued[s.half];
                    if (++n.half == u.halves) {
                        n.half = 0;
                        ++n.streamed;
                        if (++n.step == u.steps) {
                            n.step = 0;
                            ++n.unit;
                        }
                    }
                }
                if (pass) go(n);
            }
            for (int h = 0; h < 2; ++h) {
                if (s.read[h] >= seen[h].size()) continue;
                end = false;
                State n = s;
                if (s.looked[h] == s.read[h]) {
                    if (!passes(s.issued[h], s.looked[h], &wrong)) continue;
                    ++n.looked[h];
                } else {
                    ++n.read[h];
                }
                go(n);
            }
            if (!ways && !end) { *states = (int64_t)met.size(); return STUCK; }
        }
        *states = (int64_t)met.size();
        return overwritten ? OVERWRITTEN : wrong ? TOO_EARLY : FINE;
    }
};

extern "C" int walk(int second, int count, const int *halves, const int *steps, int rule, int64_t *states)
{
    Model m{second != 0, {}, rule != 0};
    for (int i = 0; i < count; ++i) m.units.push_back({halves[i], steps[i]});
    return m.walk(states);
}
"""
FINE, STUCK, TOO_EARLY, OVERWRITTEN = range(4)


@pytest.fixture(scope="module")
def walk(tmp_path_factory):
    where = tmp_path_factory.mktemp("kv_weights_rings")
    (where / "model.cpp").write_text(MODEL)
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-shared", "-fPIC", f"-I{CSRC}", "-o", str(where / "model.so"), str(where / "model.cpp")], check=True)
    lib, states = ctypes.CDLL(str(where / "model.so")), ctypes.c_int64(0)

    def call(second, units, rule=True):
        array = lambda values: (ctypes.c_int * len(units))(*values)
        result = lib.walk(int(second), len(units), array([u[0] for u in units]), array([u[1] for u in units]), int(rule), ctypes.byref(states))
        return result, states.value
    return call


# (halves, steps) of a block's units: long and short ones, second halves that come and go
UNITS = [[(2, 14)], [(1, 20)], [(2, 1), (1, 16)], [(2, 2), (1, 16), (2, 3)], [(2, 2), (1, 1), (1, 1), (1, 12), (2, 2)], [(1, 3), (2, 1), *[(1, 1)] * 9, (2, 2)],
         [(2, 1)] * 8, [(1, 1)] * 12, [(2, 1), (1, 1)] * 6, [(2, 2), (1, 1), (1, 1), (1, 1), (2, 1), (1, 6)]]


@pytest.mark.parametrize("second", [False, True])
@pytest.mark.parametrize("units", UNITS)
def test_no_order_of_steps_gets_stuck_or_overtakes_a_half(walk, second, units):
    result, states = walk(second, units)
    assert result == FINE and states > 20


@pytest.mark.parametrize("second", [False, True])
def test_units_of_all_kinds(walk, second):
    rng = random.Random(5)
    for _ in range(60):
        assert walk(second, [(rng.randint(1, 2), rng.choice([1, 1, 2, 3, 5, 9])) for _ in range(rng.randint(2, 7))])[0] == FINE


@pytest.mark.parametrize("second, units", [(False, [(2, 1), (1, 16)]), (False, [(2, 2), (1, 16), (2, 3)]), (True, [(2, 1), (1, 1), (1, 1), (1, 1), (2, 1)])])
def test_units_that_did_not_wait_for_the_second_half_would(walk, second, units):
    """The model sees the second half fall behind units that have none, until another tile is in its place."""
    assert walk(second, units, rule=False)[0] == OVERWRITTEN
    assert walk(second, units)[0] == FINE


def test_the_kernel_goes_by_this_arithmetic():
    """Places, barriers and waits of the kernel come from the header that is walked through here."""
    text = (CSRC / "kv_weights_prompt.cu").read_text()
    assert text.count("sh.info[info_place(SUMS, ") == text.count("sh.info[") == 2
    assert text.count("before_unit(halves, steps, read_out)") == 1 and text.count("before_step(half, steps, read_out)") == 1
