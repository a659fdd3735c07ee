// The tile lookup of the products whose rows choose their weights
// (igemm_rows_find.h) on the host: a wave's 64 lanes are fibers that run in turn up
// to the next exchange. Built with the undefined-behaviour sanitizer and run by
// tests/test_rows_find.py.
//
//   legal    random ascending offsets: every tile is found, once
//   hostile  offsets that do not ascend: whatever a workgroup finds lies inside
#include <ucontext.h>

#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <tuple>
#include <vector>

using std::max;
using std::min;
#define __device__
#define __forceinline__ inline

static ucontext_t lanes[64], back;
static char stacks[64][64 * 1024];
static int now;
static int32_t slot[64], result[64];
static uint64_t mask;
static void yield() { swapcontext(&lanes[now], &back); }
// Every lane puts its value down, then every lane looks.
static int exchange(int x, int from) {
    slot[now] = x;
    yield();
    const int y = slot[from];
    yield();
    return y;
}
static int __shfl_up(int x, int d) { return exchange(x, now >= d ? now - d : now); }
static int __shfl_down(int x, int d) { return exchange(x, now + d < 64 ? now + d : now); }
static int __builtin_amdgcn_readlane(int x, int l) { return exchange(x, l & 63); }
static int __builtin_amdgcn_readfirstlane(int x) { return exchange(x, 0); }
static uint64_t __ballot(bool b) {
    const int mine = exchange(b, now);
    if (now == 0) {
        mask = 0;
        for (int l = 0; l < 64; ++l) mask |= (uint64_t)slot[l] << l;
    }
    (void)mine;
    yield();
    const uint64_t m = mask;
    yield();
    return m;
}
static int __ffsll(unsigned long long x) { return __builtin_ffsll((long long)x); }

#include "igemm_rows_find.h"

using namespace igemm::rows;

static Product prod;
static int g_bm, g_bn, g_slices, g_block;
static Place places[64];
static bool done[64];
static void lane_main() {
    places[now] = place_of(prod, g_bm, g_bn, g_slices, now, g_block);
    done[now] = true;
    swapcontext(&lanes[now], &back);
}
static Place find(int bm, int bn, int slices, int block) {
    g_bm = bm, g_bn = bn, g_slices = slices, g_block = block;
    for (int l = 0; l < 64; ++l) {
        getcontext(&lanes[l]);
        lanes[l].uc_stack.ss_sp = stacks[l];
        lanes[l].uc_stack.ss_size = sizeof stacks[l];
        lanes[l].uc_link = nullptr;
        makecontext(&lanes[l], lane_main, 0);
        done[l] = false;
    }
    for (bool any = true; any;) {
        any = false;
        for (now = 0; now < 64; ++now)
            if (!done[now]) {
                swapcontext(&back, &lanes[now]);
                any = true;
            }
    }
    for (int l = 1; l < 64; ++l) {
        const Place &a = places[0], &b = places[l];
        if (a.f.cnt != b.f.cnt ||
            (a.f.cnt && (a.f.group != b.f.group || a.f.lo != b.f.lo || a.m0 != b.m0 ||
                         a.n0 != b.n0 || a.z != b.z))) {
            std::printf("lanes differ\n");
            std::exit(1);
        }
    }
    return places[0];
}
static bool inside(const Place &w, int slices) {
    return w.f.cnt == 0 ||
           (w.f.group >= 0 && w.f.group < prod.groups && w.f.lo >= 0 && w.f.cnt > 0 &&
            w.f.cnt <= prod.rows - w.f.lo && w.m0 >= 0 && w.m0 < w.f.cnt && w.n0 >= 0 &&
            w.n0 < prod.n && w.z >= 0 && w.z < slices);
}
static void show(const Place &w, int block) {
    std::printf("block %d: group %d lo %d cnt %d m0 %d n0 %d z %d\n", block, w.f.group, w.f.lo,
                w.f.cnt, w.m0, w.n0, w.z);
}

static int legal() {
    std::mt19937 rng(1);
    const int tiles[][2] = {{32, 128}, {32, 256}, {64, 128}, {128, 128}, {256, 256}};
    int found = 0;
    for (int it = 0; it < 40; ++it) {
        const int *bt = tiles[it % 5], bm = bt[0], bn = bt[1];
        prod = {};
        prod.rows = 1 + rng() % (it % 3 ? 3000 : 100);
        prod.groups = 1 + rng() % (it % 4 ? 12 : 200);
        prod.n = 1 + rng() % 1300;
        const int slices = bm <= 64 && bn == 128 ? 1 + rng() % 3 : 1;
        std::vector<int32_t> off(prod.groups + 1);
        for (auto &o : off) o = (int)(rng() % (prod.rows + 20)) - 10;
        std::sort(off.begin(), off.end());
        prod.offsets = it % 7 ? off.data() : nullptr;
        if (!prod.offsets) prod.groups = 1;
        const int64_t grid =
            most_tiles(prod.rows, prod.groups, bm) * ((prod.n + bn - 1) / bn) * slices;
        std::map<std::tuple<int, int, int, int>, int> seen;
        for (int b = 0; b < grid; ++b) {
            const Place w = find(bm, bn, slices, b);
            if (!inside(w, slices)) return show(w, b), 1;
            if (w.f.cnt) ++seen[{w.f.group, w.m0, w.n0, w.z}];
        }
        size_t want = 0;
        for (int g = 0; g < prod.groups; ++g) {
            const int lo = prod.offsets ? min(max(off[g], 0), prod.rows) : 0;
            const int hi = prod.offsets ? min(max(off[g + 1], 0), prod.rows) : prod.rows;
            for (int m0 = 0; m0 < hi - lo; m0 += bm)
                for (int n0 = 0; n0 < prod.n; n0 += bn)
                    for (int z = 0; z < slices; ++z, ++want)
                        if (seen[{g, m0, n0, z}] != 1) {
                            std::printf("group %d m0 %d n0 %d z %d: %d times\n", g, m0, n0, z,
                                        seen[{g, m0, n0, z}]);
                            return 1;
                        }
        }
        if (seen.size() != want) return std::printf("tiles that are none\n"), 1;
        found += (int)want;
    }
    std::printf("ok %d\n", found);
    return 0;
}

static int hostile() {
    std::mt19937_64 rng(2);
    struct Case {
        int rows, groups, n, bm, bn, slices, kind;
    };
    const Case cases[] = {
        {131072, 65536, 8192, 32, 256, 1, 0},
        {1 << 22, 65536, 4096, 64, 128, 1, 0},
        {1 << 22, 65536, 2432, 64, 128, 1, 0},
        {1 << 20, 65536, 4096, 32, 128, 1, 1},
        {4096, 60000, 4 << 20, 32, 128, 16, 0},
        {100000, 64, 1 << 20, 256, 256, 1, 0},
        {100000, 63, 70000, 128, 128, 1, 2},
        {2147483136, 65536, 1, 256, 256, 1, 0},
        {2147483136, 65536, 1, 128, 128, 1, 2},
        {50000, 1000, 100000, 64, 128, 16, 1},
    };
    int some = 0;
    for (const Case &c : cases) {
        prod = {};
        prod.rows = c.rows, prod.groups = c.groups, prod.n = c.n;
        std::vector<int32_t> off(c.groups + 1);
        for (int g = 0; g <= c.groups; ++g)
            off[g] = c.kind == 0   ? (g & 1 ? c.rows : 0)
                     : c.kind == 1 ? (int32_t)rng()
                                   : (g & 1 ? 0x7fffffff : (int)(rng() % 1000) - 500);
        prod.offsets = off.data();
        const int64_t grid = min(most_tiles(c.rows, c.groups, c.bm) * ((c.n + c.bn - 1) / c.bn) *
                                     c.slices,
                                 (int64_t)0xffffff);
        for (int s = 0; s < 600; ++s) {
            const int b = s < 40 ? min((int64_t)s, grid - 1)
                          : s < 80 ? max(grid - 1 - (s - 40), (int64_t)0)
                                   : (int)(rng() % grid);
            const Place w = find(c.bm, c.bn, c.slices, b);
            if (!inside(w, c.slices)) return show(w, b), 1;
            some += w.f.cnt > 0;
        }
    }
    std::printf("ok %d\n", some);
    return some > 0 ? 0 : 1;
}

int main(int argc, char **argv) { return argc > 1 && argv[1][0] == 'h' ? hostile() : legal(); }
