"""How shared and cross attention number their work, on the host: the kernels' own arithmetic on offsets, lengths and groups that come from device memory,
also on those that no careful caller has.  No GPU is touched."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

BEGIN = r"""
#include <stdio.h>
#include <stdlib.h>
#include <vector>
#include "rows_numbering.h"
using namespace specvlm;

#define REQUIRE(x, ...) do { if (!(x)) { printf("%d: " #x, __LINE__); printf(" " __VA_ARGS__); puts(""); return 1; } } while (0)
"""

# The kernel's loop over entries of so much work each, with what it does at each one counted.
WALK = r"""
static int walk(const std::vector<int>& work)
{
    const int entries = (int)work.size();
    RowsParams p = {};
    p.workgroups = 256;
    const auto look_at = [&](int c0) {
        Numbers n = {0, 0};
        for (int e = c0; e < c0 + kRowsThreads && e < entries; ++e) n.work += work[e], n.rows += 32 * (work[e] > 0);
        return n;
    };
    int total = 0;
    for (int w : work) total += w;
    const Shares shares = shares_of(p, total);
    std::vector<int> told(entries, 0), taken(entries, 0);
    for (int j = 0; j < shares.n; ++j) {
        int x = shares.begin(j), steps = 0;
        const int x_end = shares.begin(j + 1);
        Walk at_hand = {{0, 0}, 0, entries <= kRowsThreads || j > 0};
        Numbers here = look_at(0);
        const auto tell = [&] { for (int e = at_hand.c0; e < at_hand.c0 + kRowsThreads && e < entries; ++e) ++told[e]; };
        if (j == 0) tell();
        while (x < x_end || !at_hand.told) {
            while (at_hand.goes_on(x, x_end, here.work)) {
                REQUIRE(++steps <= 2 * (entries / kRowsThreads + 1), "workgroup %d goes on for ever: %d entries, %d units", j, entries, total);
                at_hand.step(here, entries);
                here = look_at(at_hand.c0);
                if (!at_hand.told) tell();
            }
            if (x >= x_end) break;
            int e = at_hand.c0, front = at_hand.base.work;
            while (x >= front + work[e]) front += work[e++];
            const int end = x_end < front + work[e] ? x_end : front + work[e];
            taken[e] += end - x;
            x = end;
        }
    }
    for (int e = 0; e < entries; ++e) REQUIRE(told[e] == 1 && taken[e] == work[e], "entry %d of %d", e, entries);
    return 0;
}

int main()
{
    srand(1);
    for (int entries : {1, 2, 511, 512, 513, 514, 1000, 1024, 1025, 1200, 5000}) {
        std::vector<int> work(entries, 0);
        if (walk(work)) return 1;                            // all are skipped
        for (int at : {0, entries / 2, entries - 1}) {       // all but one
            work.assign(entries, 0);
            work[at] = 1 + rand() % 100000;
            if (walk(work)) return 1;
        }
        for (int some : {2, 50}) {
            for (int& w : work) w = rand() % some ? 0 : 28 + rand() % 3000;
            if (walk(work)) return 1;
        }
        for (int& w : work) w = 28 + rand() % 100;
        if (walk(work)) return 1;
    }
    puts("ok");
}
"""

PROGRAMS = {"a workgroup's way through the entries": WALK}


@pytest.mark.parametrize("what", PROGRAMS)
def test_numbering(tmp_path, what):
    source, program = tmp_path / "numbering.hip", tmp_path / "numbering"
    source.write_text(BEGIN + PROGRAMS[what])
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    subprocess.run([hipcc, "--offload-host-only", "-O1", "-std=c++17", "-w", "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(ROOT, "paper_2508_16201_amd", "csrc"), "-o", str(program), str(source)], check=True)
    res = subprocess.run([str(program)], capture_output=True, text=True, timeout=60)
    assert res.returncode == 0 and res.stdout == "ok\n", res.stdout + res.stderr
