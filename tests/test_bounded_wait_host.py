"""The kernels' bounded wait as a program on the host, with a clock and a test of its own: what a context that is switched out for longer than the
limit must not lose, and that a wait on what never comes ends."""
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2412_16602_gb300", "csrc")
PROGRAM = r"""
#include <stdio.h>
#include "bounded_wait.h"
// argv-less: prints one line for each story
static uint64_t now, tests, done_at_test, done_at_time, jump_after, jump;
static bool test() { ++tests; return tests >= done_at_test || now >= done_at_time; }
static uint64_t clock_() { now += 1; if (tests == jump_after && jump) { now += jump; jump = 0; } return now; }
static void story(const char* name, uint64_t dt, uint64_t dn, uint64_t ja, uint64_t j) {
    now = 1000, tests = 0, done_at_test = dt, done_at_time = dn, jump_after = ja, jump = j;
    const bool ok = vmb::bounded_wait(test, clock_, 100);
    printf("%s %d %llu\n", name, ok, (unsigned long long)(now - 1000));
}
int main() {
    const uint64_t never = ~0ull;
    story("at_once", 1, never, 0, 0);
    story("soon", 5, never, 0, 0);
    story("never", never, never, 0, 0);
    // switched out for ten times the limit between a test and the look at the clock; what was waited for came meanwhile
    story("done_while_away", never, 1500, 4, 1000);
    // the same in the second half
    story("done_while_away_late", never, 1500, 60, 1000);
    // who should do it was switched out as well, and needs 20 more tests
    story("held_up_too", 25, never, 4, 1000);
}
"""


@pytest.fixture(scope="module")
def stories(tmp_path_factory):
    d = tmp_path_factory.mktemp("wait")
    (d / "wait.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", CSRC, str(d / "wait.cpp"), "-o", str(d / "wait")], check=True)
    lines = subprocess.run([str(d / "wait")], check=True, capture_output=True, text=True, timeout=60).stdout.split("\n")
    return {n: (ok == "1", int(t)) for n, ok, t in (line.split() for line in lines if line)}


@pytest.mark.parametrize("name", ["at_once", "soon", "done_while_away", "done_while_away_late", "held_up_too"])
def test_what_is_done_is_not_given_up(stories, name):
    assert stories[name][0]


def test_a_wait_on_nothing_ends_at_the_limit(stories):
    ok, waited = stories["never"]
    assert not ok and 100 <= waited <= 106  # two halves of 50, and the looks at the clock that begin and end them
