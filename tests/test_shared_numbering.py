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

# Requests and groups of every kind: who is taken with a group has its queries among those of the group's entry, before its block and behind the shared
# keys; everyone whose own words fit together is taken, once.
GROUPS = r"""
struct Call {
    std::vector<int> cu_q, kv_lens, groups;
    int n_queries, q_len, kv_len;
};

static int check(const Call& c, const std::vector<int>& with)       // with: who has to be taken with a group (empty: anyone)
{
    RowsParams p = {};
    const int batch = (int)c.kv_lens.size();
    p.cu_q = c.cu_q.data(); p.kv_lens = c.kv_lens.data(); p.groups = c.groups.data();
    p.batch = batch; p.entries = 2 * batch; p.n_queries = c.n_queries; p.q_len = c.q_len; p.kv_len = c.kv_len;
    for (int b = 0; b < batch; ++b) {
        const Entry all = entry_of<true>(p, b, true), own = entry_of<true>(p, batch + b, true), alone = entry_of<true>(p, batch + b, false);
        if (all.n_q > 0) REQUIRE(all.q0 >= 0 && all.n_q <= c.n_queries - all.q0 && all.key0 == 0 && all.key1 > 0 && all.key1 <= c.kv_len && all.key1 % 16 == 0, "%d", b);
        const int64_t from = c.cu_q[b], to = c.cu_q[b + 1], n = to - from, kvl = c.kv_lens[b];
        const bool fits = from >= 0 && n > 0 && n <= c.q_len && to <= c.n_queries && kvl >= n && kvl <= c.kv_len;
        REQUIRE((own.n_q > 0) == fits && (alone.n_q > 0) == fits, "%d", b);
        if (!fits) continue;
        REQUIRE(own.q0 == from && own.n_q == n && own.key1 == kvl && alone.key0 == 0 && alone.key1 == kvl && alone.first == -1, "%d", b);
        REQUIRE((own.first >= 0) == (own.key0 > 0) && own.first <= b, "%d", b);
        if (own.key0 > 0) {
            const Entry first = entry_of<true>(p, own.first, true);
            REQUIRE(first.n_q > 0 && first.key1 == own.key0 && own.key0 <= kvl - n, "%d", b);
            REQUIRE(first.q0 <= from && to <= first.q0 + first.n_q, "the queries of %d, %d to %d, are not among those of %d: %d to %d", b, (int)from, (int)to, own.first,
                    first.q0, first.q0 + first.n_q);
        }
        if (!with.empty()) REQUIRE(own.first == with[b], "%d is with %d, not %d", b, own.first, with[b]);
    }
    return 0;
}

static int group_of(std::vector<int>& groups, int batch, int first, int members, int shared)
{
    for (int b = first; b < first + members; ++b) groups[b] = first, groups[batch + b] = b == first ? members : 0, groups[2 * batch + b] = shared;
    return 0;
}

int main()
{
    const auto one_group = [](std::vector<int> cu_q, int n_queries, int q_len) {
        const int batch = (int)cu_q.size() - 1;
        Call c = {cu_q, std::vector<int>(batch, 500), std::vector<int>(3 * batch, 0), n_queries, q_len, 500};
        group_of(c.groups, batch, 0, batch, 64);
        return c;
    };
    if (check(one_group({0, 5, 9, 20}, 20, 11), {0, 0, 0})) return 1;
    if (check(one_group({0, 5, 100, 20}, 100, 95), {0, -1, -1})) return 1;              // (the second ends behind the last one's end)
    if (check(one_group({50, 60, 10, 40, 90}, 100, 50), {0, -1, -1, -1})) return 1;     // (the third lies in front of the first)
    if (check(one_group({10, 12, 0, 8, -5, 14}, 20, 20), {0, -1, -1, -1, -1})) return 1;
    if (check(one_group({0, 5, 300, 9, 20}, 20, 20), {0, -1, -1, 0})) return 1;         // (skipped ones in between change no other)
    srand(1);
    for (int i = 0; i < 300000; ++i) {
        const int batch = 1 + rand() % 7, n_queries = 1 + rand() % 60;
        Call c = {std::vector<int>(batch + 1), std::vector<int>(batch), std::vector<int>(3 * batch, 0), n_queries, 1 + rand() % 60, 40 + rand() % 100};
        int at = rand() % 8;
        for (int& x : c.cu_q) {
            x = rand() % 6 ? at : rand() % (n_queries + 20) - 10;
            at += rand() % 12;
        }
        for (int& x : c.kv_lens) x = rand() % 8 ? 30 + rand() % 110 : rand() % 20 - 5;
        for (int b = 0; b < batch; ++b) {
            if (rand() % 3 == 0) group_of(c.groups, batch, b, 1 + rand() % (batch - b), 16 * (rand() % 6));
            if (rand() % 9 == 0) c.groups[rand() % (3 * batch)] = rand() % 40 - 5;
        }
        if (check(c, {})) return 1;
    }
    puts("ok");
}
"""

# The same where lengths and offsets are any numbers at all.
ANYTHING = GROUPS[:GROUPS.index("int main()")] + r"""
int main()
{
    const int ends[] = {INT32_MIN, INT32_MIN + 1, INT32_MIN + 5, -1, 0, 1, 5, 40, INT32_MAX - 4, INT32_MAX};
    srand(2);
    for (int i = 0; i < 300000; ++i) {
        const int batch = 1 + rand() % 5, n_queries = 1 + rand() % 60;
        Call c = {std::vector<int>(batch + 1), std::vector<int>(batch), std::vector<int>(3 * batch, 0), n_queries, 1 + rand() % 60, 40 + rand() % 100};
        int at = 0;
        for (int& x : c.cu_q) {
            x = rand() % 4 ? at : ends[rand() % 10];
            at += rand() % 12;
        }
        for (int& x : c.kv_lens) x = rand() % 2 ? 30 + rand() % 110 : ends[rand() % 10];
        for (int b = 0; b < batch; ++b)
            if (rand() % 2 == 0) group_of(c.groups, batch, b, 1 + rand() % (batch - b), rand() % 2 ? 16 * (rand() % 6) : (ends[rand() % 10] & ~15));
        if (check(c, {})) return 1;
    }
    puts("ok");
}
"""

# Shares of entries whose queries lie in any order: every one has a number of its own.
SHARES = r"""
static int check(const std::vector<int>& cu_q, int n_queries, int span, bool required)
{
    RowsParams p = {};
    p.cu_q = cu_q.data(); p.batch = (int)cu_q.size() - 1; p.n_queries = p.q_len = n_queries; p.span = span; p.inv_span = reciprocal(span);
    const int entries = p.batch + n_queries / span + 1;
    std::vector<int> in(n_queries, 0);
    int number = 0, queries = 0;
    for (int b = 0; b < p.batch; ++b) {
        const int n = shares_of_entry(p, b), q0 = cu_q[b], of = has_queries(p, b) ? cu_q[b + 1] - q0 : 0;
        REQUIRE(n * span >= of && (n - 1) * span < of, "%d", b);
        for (int i = 0; i < of; ++i) {
            if (in[q0 + i]++) return required;               // (a query in two entries)
            ++queries;
        }
        number += n;
    }
    REQUIRE(number <= entries, "%d shares of %d queries, %d numbers", number, queries, entries);
    REQUIRE(shares_of_entry(p, p.batch) == 0);
    return 0;
}

int main()
{
    if (check({32, 96, 0, 32}, 96, 32, true) || check({0, 40, 999, 40, 70}, 70, 36, true) || check({64, 96, 32, 64, 0, 32}, 96, 32, true)) return 1;
    srand(3);
    for (int i = 0; i < 300000; ++i) {
        const int n_queries = 1 + rand() % 200, span = 1 + rand() % 70;
        std::vector<int> cu_q(2 + rand() % 8);
        int at = rand() % 20;
        for (int& x : cu_q) {
            x = rand() % 3 ? at : rand() % (n_queries + 20) - 10;
            at += rand() % 40;
        }
        if (check(cu_q, n_queries, span, false)) return 1;
    }
    puts("ok");
}
"""

PROGRAMS = {"a workgroup's way through the entries": WALK, "who is taken with a group": GROUPS,
            "groups of requests of which anything is said": ANYTHING, "shares of entries in any order": SHARES}


@pytest.mark.parametrize("what", PROGRAMS)
def test_numbering(tmp_path, what):
    source, program = tmp_path / "numbering.hip", tmp_path / "numbering"
    source.write_text(BEGIN + PROGRAMS[what])
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    subprocess.run([hipcc, "--offload-host-only", "-O1", "-std=c++17", "-w", "-I", os.path.join(ROOT, "include"), "-I",
                    os.path.join(ROOT, "paper_2508_16201_amd", "csrc"), "-o", str(program), str(source)], check=True)
    res = subprocess.run([str(program)], capture_output=True, text=True, timeout=60)
    assert res.returncode == 0 and res.stdout == "ok\n", res.stdout + res.stderr
