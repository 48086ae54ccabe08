// The experts' tile search (block_row_tiles.h) on the host: its 64 lanes run as
// fibers that wait for each other at every wave function, and every tile
// number's answer is compared with a plain walk over the experts.
#include <ucontext.h>

#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <functional>
#include <random>
#include <vector>

// ---- a wave of 64 lanes ----
constexpr int kLanes = 64;
static ucontext_t g_main, g_lane[kLanes];
static std::vector<char> g_stack[kLanes];
static int g_now;          // the lane that runs
static int g_values[2][kLanes];  // what the lanes gave to this wave function and to the one before
static int g_turn[kLanes];
static std::function<void(int)> g_body;

struct Index {
  struct X {
    operator int() const { return g_now; }
  } x;
};
static Index threadIdx;

static const int* exchange(int v) {
  const int lane = g_now, turn = g_turn[lane]++ & 1;
  g_values[turn][lane] = v;
  swapcontext(&g_lane[lane], &g_main);  // until every lane is here
  return g_values[turn];
}
static int __shfl_up(int v, int d) {
  const int* all = exchange(v);
  return g_now >= d ? all[g_now - d] : v;
}
static int readlane(int v, int l) { return exchange(v)[l]; }
static uint64_t __ballot(bool p) {
  const int* all = exchange(p);
  uint64_t m = 0;
  for (int l = 0; l < kLanes; ++l) m |= (uint64_t)(all[l] != 0) << l;
  return m;
}
static bool g_done[kLanes];
static void lane_main() {
  g_body(g_now);
  g_done[g_now] = true;
}
static void run_wave(std::function<void(int)> body) {
  g_body = std::move(body);
  for (int l = 0; l < kLanes; ++l) {
    g_stack[l].resize(1 << 16);
    g_done[l] = false;
    g_turn[l] = 0;
    getcontext(&g_lane[l]);
    g_lane[l].uc_stack.ss_sp = g_stack[l].data();
    g_lane[l].uc_stack.ss_size = g_stack[l].size();
    g_lane[l].uc_link = &g_main;
    makecontext(&g_lane[l], lane_main, 0);
  }
  for (bool any = true; any;) {
    any = false;
    for (int l = 0; l < kLanes; ++l)
      if (!g_done[l]) {
        g_now = l;
        swapcontext(&g_main, &g_lane[l]);
        any = true;
      }
  }
}

using std::max;
using std::min;
#define __device__
#define __forceinline__ inline
#define __builtin_amdgcn_readlane readlane
#include "block_row_tiles.h"

struct Args {
  const int32_t* offsets;
  int rows, experts;
};

static int failures = 0;

static void check(const std::vector<int32_t>& offsets, int rows, int TR) {
  const Args g{offsets.data(), rows, (int)offsets.size() - 1};
  std::vector<agn::RowTile> want;
  for (int e = 0; e < g.experts; ++e) {
    const int b = min(max(offsets[e], 0), rows), end = max(b, min(max(offsets[e + 1], 0), rows));
    const int n = (end - b + TR - 1) / TR;
    for (int i = 0; i < n; ++i) want.push_back({e, b + i * TR, end, i, n});
  }
  const int numbers = (int)want.size() + 40;  // the tiles, and numbers past them
  std::vector<std::vector<agn::RowTile>> got(kLanes, std::vector<agn::RowTile>(numbers));
  std::vector<int> total(kLanes);
  run_wave([&](int lane) {
    agn::RowTiles t;
    t.init(g, TR);
    total[lane] = t.total;
    for (int i = 0; i < numbers; ++i) got[lane][i] = t.find(g, i);
  });
  for (int l = 0; l < kLanes; ++l) {
    bool ok = total[l] == (int)want.size();
    for (int i = 0; i < numbers; ++i) {
      const agn::RowTile& a = got[l][i];
      if (i >= (int)want.size()) {
        ok = ok && a.e == -1;
      } else {
        const agn::RowTile& b = want[i];
        ok = ok && a.e == b.e && a.r0 == b.r0 && a.rend == b.rend && a.of == b.of && a.of_expert == b.of_expert;
      }
    }
    if (!ok) {
      if (l == 0) std::fprintf(stderr, "FAIL: %d experts, %d rows, tiles of %d\n", g.experts, rows, TR);
      ++failures;
      break;
    }
  }
}

int main() {
  std::mt19937 rng(7);
  int checked = 0;
  for (int experts : {1, 7, 63, 64, 65, 128, 130, 200, 1024})
    for (int TR : {16, 128})
      for (int kind = 0; kind < 4; ++kind) {
        std::vector<int32_t> o(experts + 1, 0);
        for (int e = 0; e < experts; ++e) {
          int n = 0;
          if (kind == 0) n = experts > 200 ? rng() % 9 == 0 : rng() % 3;  // a few rows each
          if (kind == 1) n = rng() % (1 + experts / 8) == 0 ? rng() % 200 : 0;  // some experts only
          if (kind == 2) n = e >= experts - 3 ? 1 + (int)(rng() % 70) : 0;   // the last ones only
          if (kind == 3) n = e < 2 ? 40 : 0;                              // the first ones only
          o[e + 1] = o[e] + n;
        }
        const int rows = o[experts] + (int)(rng() % 20);
        check(o, rows, TR);
        if (kind == 1) {  // offsets that do not rise, or leave the matrix: tiles stay in it
          for (int i = 0; i < 3; ++i) o[rng() % (experts + 1)] = (int32_t)(rng() % (2 * rows + 9)) - 5;
          check(o, rows, TR);
        }
        ++checked;
      }
  std::printf("%d plans, %d failure(s)\n", checked, failures);
  return failures != 0;
}
