// Host-side harness for tests/test_window_host.py: the key lists and tile numbers of the windowed attention, with the
// library's own functions, checked against the definition by enumeration.  Compiled by the test with hipcc as host
// code; nothing runs on a GPU.  Prints "ok lists tiles" or the first case that is wrong.
#include "window_common.h"

#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

using namespace nexus;

static bool sees(int p, int k, int window, int sinks) { return k <= p && (k > p - window || k < sinks); }

static long check_list(int window, int sinks, int p0, int p1) {
  const KeyList l = key_list(window, sinks, p0, p1);
  std::vector<char> listed((p1 >> 4) + 1, 0);
  int last = -1;
  for (int e = 0; e < l.n; ++e) {
    const int p = l.page(e);
    if (p <= last || p > p1 >> 4) return 1;            // pages increase, none behind the last key's
    last = p;
    listed[p] = 1;
    int n = 0;
    for (int s = 0; s < 16; ++s) {
      const int k = 16 * p + s, in = l.stand_in(k);
      if (in >> 4 != p || !l.seen(in) || (l.seen(k) && in != k)) return 2;
      n += l.seen(k);
    }
    if (n == 0) return 3;
  }
  for (int k = 0; k <= p1; ++k) {
    bool any = false;
    for (int p = p0 < 0 ? 0 : p0; p <= p1 && !any; ++p) any = sees(p, k, window, sinks);
    if (any && (!listed[k >> 4] || !l.seen(k))) return 4;          // every key that a row sees is listed
    if (p0 >= 0 && !any && l.seen(k) && l.lo > 0) return 5;        // and none that no row does, where they part
  }
  return 0;
}

// The splits' steps go through every tile of a list once.
template <int PT>
static bool check_order(int window, int sinks, int p0, int p1, int period) {
  const KeyList l = key_list(window, sinks, p0, p1);
  for (int n_splits : {1, 2, 3, 7}) {
    const int all = (l.n + PT - 1) / PT;
    std::vector<int> taken(all, 0);
    for (int s = 0; s < n_splits; ++s) {
      const TileOrder<PT> o = tile_order<PT>(l, period, s, n_splits);
      for (int t = 0; t < o.t1 - o.t0; ++t) {
        const int x = o.tile(t);
        if (x < 0 || x >= all || taken[x]++) return false;
        for (int g = 0; g < PT; ++g)
          if (o.entry(PT * t + g) != PT * x + g) return false;
      }
    }
    for (int x : taken)
      if (x != 1) return false;
  }
  return true;
}

template <int R>
static bool check_tiles(std::mt19937 &rng) {
  const int n_seqs = 1 + rng() % 70, group = 1 + rng() % 40;
  std::vector<int> start(1, rng() % 3 == 0 ? rng() % 50 : 0);
  for (int b = 0; b < n_seqs; ++b) start.push_back(start.back() + (rng() % 3 ? rng() % 5 : rng() % 300));
  const int n_rows = start.back() + rng() % 4;
  const uint32_t bound = (uint32_t)((int64_t)n_rows * group / R + n_seqs);
  for (int b = 0; b < n_seqs; ++b) {
    const uint32_t first = first_tile<R>(start[b], group, b), next = first_tile<R>(start[b + 1], group, b + 1);
    const uint32_t need = ((uint32_t)(start[b + 1] - start[b]) * group + R - 1) / R;
    if (next <= first || next - first < need) return false;        // numbers increase and suffice
    if (first + need > bound) return false;                        // within the launch
  }
  return true;
}

int main() {
  long lists = 0, tiles = 0;
  for (int window : {1, 2, 3, 15, 16, 17, 31, 33, 64, 200})
    for (int sinks : {0, 1, 4, 15, 16, 17, 40, 128})
      for (int p0 = -3; p0 < 150; p0 += 1 + (p0 > 70) * 6)
        for (int p1 : {p0, p0 + 1, p0 + 7, p0 + 25, p0 + 64, p0 + 127}) {
          if (p1 < 0) continue;
          const long e = check_list(window, sinks, p0, p1);
          if (e) {
            printf("list %ld: window %d sinks %d rows %d..%d\n", e, window, sinks, p0, p1);
            return 0;
          }
          for (int period : {1, 2, 5, 9, 1000})
            if (!check_order<4>(window, sinks, p0, p1, period) || !check_order<2>(window, sinks, p0, p1, period)) {
              printf("order: window %d sinks %d rows %d..%d period %d\n", window, sinks, p0, p1, period);
              return 0;
            }
          ++lists;
        }
  std::mt19937 rng(7);
  for (int i = 0; i < 20000; ++i, ++tiles)
    if (!check_tiles<128>(rng) || !check_tiles<256>(rng) || !check_tiles<16>(rng)) {
      printf("tiles %d\n", i);
      return 0;
    }
  printf("ok %ld %ld\n", lists, tiles);
  return 0;
}
