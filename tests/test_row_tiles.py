"""Which rows and columns a workgroup takes (csrc/rowtiles.h), on the CPU: the header is compiled for the host with the
64 lanes of a wavefront as fibers that meet at every cross-lane operation.  Rising offsets: every row of every
panel is taken exactly once.  Offsets of any values: whatever is taken lies inside the rows, the experts and the panels,
also where the falling offsets' tiles are more than 32 bits count."""
import os
import shutil
import subprocess

import pytest

from paper_2606_00395_amd import build as BLD

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")

COMMON = r"""
#pragma once
#include <ucontext.h>
#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>
#define __device__
#define __forceinline__ inline
using std::max;
using std::min;
struct Lane { unsigned x; };
inline Lane ids[64];
inline int current = 0, turn[64];
inline int64_t slots[2][64];
inline ucontext_t main_context, lanes[64];
#define threadIdx ids[current]
// every lane's value of an operation that all of them reach
inline const int64_t* meet(int64_t v) {
    const int me = current, t = turn[me];
    turn[me] ^= 1;
    slots[t][me] = v;
    swapcontext(&lanes[me], &main_context);
    return slots[t];
}
inline int wave_readlane(int v, int lane) { return (int)meet(v)[lane]; }
inline uint64_t wave_ballot(bool v) {
    const int64_t* all = meet(v);
    uint64_t m = 0;
    for (int l = 0; l < 64; ++l) m |= (uint64_t)(all[l] != 0) << l;
    return m;
}
inline int wave_dpp(int old, int v, int ctrl, int row_mask, int, bool) {
    const int64_t* all = meet(v);
    const int me = current, row = me / 16;
    if (!(row_mask >> row & 1)) return old;
    if (ctrl > 0x110 && ctrl < 0x120) return me % 16 < ctrl - 0x110 ? old : (int)all[me - (ctrl - 0x110)];   // row_shr
    if (ctrl == 0x142) return row ? (int)all[row * 16 - 1] : old;       // row_bcast:15
    if (ctrl == 0x143) return row > 1 ? (int)all[31] : old;             // row_bcast:31
    abort();
}
#define __builtin_amdgcn_readlane wave_readlane
#define __builtin_amdgcn_update_dpp wave_dpp
#define __ballot wave_ballot
"""

MAIN = r"""
#include "rowtiles.h"
using namespace pr2;
struct Call { const int* offsets; int N, R, rows, panels; uint32_t block; bool by_panel; };
Call call;
bool got[64];
RowTile tiles[64];
char stacks[64][16384];
void lane_main(int l) {
    RowTile t{};
    got[l] = call.by_panel ? find_tile<true>(call.offsets, call.N, call.R, call.rows, call.panels, call.block, &t)
                           : find_tile<false>(call.offsets, call.N, call.R, call.rows, call.panels, call.block, &t);
    tiles[l] = t;
    for (;;) { turn[l] = 2; swapcontext(&lanes[l], &main_context); }
}
bool find(RowTile* t) {
    for (int l = 0; l < 64; ++l) {
        ids[l].x = l;
        turn[l] = 0;
        getcontext(&lanes[l]);
        lanes[l].uc_stack.ss_sp = stacks[l];
        lanes[l].uc_stack.ss_size = sizeof stacks[l];
        lanes[l].uc_link = nullptr;
        makecontext(&lanes[l], (void (*)())lane_main, 1, l);
    }
    for (bool on = true; on;) {
        on = false;
        for (current = 0; current < 64; ++current) {
            if (turn[current] == 2) continue;
            swapcontext(&main_context, &lanes[current]);
            on |= turn[current] != 2;
        }
    }
    for (int l = 1; l < 64; ++l)
        if (got[l] != got[0]) { printf("lanes differ\n"); exit(1); }
    *t = tiles[0];
    return got[0];
}
std::mt19937_64 rng(7);
int pick(int n) { return (int)(rng() % n); }
void wrong(const char* what, const RowTile& t) {
    printf("%s: R %d N %d rows %d panels %d by_panel %d block %u -> expert %d row0 %d rows %d panel %d\n", what, call.R, call.N,
           call.rows, call.panels, call.by_panel, call.block, t.expert, t.row0, t.rows, t.panel);
    exit(1);
}
void inside(const RowTile& t) {
    if (t.expert < 0 || t.expert > call.N || t.row0 < 0 || t.rows < 1 || t.rows > call.rows ||
        (int64_t)t.row0 + t.rows > call.R || t.panel < 0 || t.panel >= call.panels) wrong("outside", t);
}
int main(int argc, char** argv) {
    if (argc > 1) {     // rising offsets, every workgroup
        for (int round = 0; round < 60; ++round) {
            const int few[] = {1, 2, 5, 63, 64, 130, 300, 1024};
            const int N = few[pick(8)], R = 1 + pick(round % 3 ? 900 : 90), tail = pick(3) ? 0 : pick(R);
            std::vector<int> o(N + 1, 0);
            for (int e = 1; e < N; ++e) o[e] = pick(R - tail + 1);
            o[N] = R - tail;
            std::sort(o.begin(), o.end());
            const bool none = N == 1 && pick(2);
            call = Call{none ? nullptr : o.data(), N, R, 16 << pick(5), 1 + pick(7), 0, pick(2) == 1};
            std::vector<int> seen((size_t)R * call.panels, 0);
            const int64_t groups = tile_groups(R, N, call.rows, call.panels);
            for (int64_t b = 0; b < groups; ++b) {
                call.block = (uint32_t)b;
                RowTile t;
                if (!find(&t)) continue;
                inside(t);
                const int first = none ? 0 : t.expert < N ? o[t.expert] : o[N], last = none || t.expert == N ? R : o[t.expert + 1];
                if (t.row0 < first || t.row0 + t.rows > last) wrong("another expert's rows", t);
                for (int r = t.row0; r < t.row0 + t.rows; ++r) ++seen[(size_t)r * call.panels + t.panel];
            }
            for (int v : seen)
                if (v != 1) wrong("rows not taken once", RowTile{});
        }
    } else {            // any offsets
        int taken = 0;
        for (int round = 0; round < 400; ++round) {
            const int rows = 16 << pick(5), kind = pick(5);
            int R = round % 4 == 0 ? 1 + pick(5000) : (int)std::min<int64_t>(0x7fffffff - 1024, ((int64_t)1 << (22 + pick(10))) - 1 + pick(9));
            const int N = round % 2 ? 1024 - pick(4) : 1 + pick(1024);
            if (kind == 3) R = std::min(rows * ((1 << 23) - pick(9)), 0x7fffffff - 1024);    // nearly 2^32 tiles
            std::vector<int> o(N + 1);
            for (int e = 0; e <= N; ++e) {
                const int some[] = {0, 1, R, R - 1, R / 2, -5, 0x7fffffff, pick(R)};
                o[e] = kind == 0 ? (e & 1 ? R : 0) : kind == 1 ? some[pick(8)] : kind == 2 ? (e % 16 == 15 ? 1 : e & 1 ? R : 0)
                     : kind == 3 ? (e < 2 ? e : e & 1 ? 0 : R) : (int)rng();
            }
            call = Call{o.data(), N, R, rows, round % 3 ? 1 + pick(3) : 1 + pick(40), 0, pick(2) == 1};
            const int64_t groups = std::min<int64_t>(tile_groups(R, N, call.rows, call.panels), 0x7fffffff);
            for (int i = 0; i < 16; ++i) {
                call.block = (uint32_t)(i < 8 ? i : i == 8 ? groups - 1 : (int64_t)(rng() % (uint64_t)groups));
                RowTile t;
                if (!find(&t)) continue;
                ++taken;
                inside(t);
            }
        }
        if (taken < 500) { printf("only %d workgroups took rows\n", taken); return 1; }
    }
    return 0;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    d = tmp_path_factory.mktemp("row_tiles")
    (d / "common.h").write_text(COMMON)
    (d / "main.cpp").write_text(MAIN)
    shutil.copy(os.path.join(BLD.CSRC, "rowtiles.h"), d / "rowtiles.h")
    # (sums of tiles that pass 32 bits wrap on the device)
    subprocess.run(["g++", "-std=c++17", "-O1", "-fwrapv", "-o", str(d / "main"), str(d / "main.cpp")], check=True)
    return str(d / "main")


@pytest.mark.parametrize("args", [["rising"], []], ids=["rising", "any"])
def test_what_a_workgroup_takes(program, args):
    p = subprocess.run([program, *args], stdout=subprocess.PIPE, text=True, timeout=120)
    assert p.returncode == 0, p.stdout
