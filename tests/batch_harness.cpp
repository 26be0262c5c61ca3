// Host-side harness for tests/test_batch_host.py: what the sequences of a layout ask for and which of them are refused,
// with the library's own functions, walked in the order of the sequences and checked against the definition token by
// token.  Compiled by the test with hipcc as host code; nothing runs on a GPU.  Prints "ok batches" or the first that
// is wrong.
#include "launch_batch.h"

#include <cstdio>
#include <random>
#include <vector>

using namespace nexus;

// The definition: pages a token at a time, rows within the launch.
static bool wanted(int64_t cached, int64_t fresh, int64_t stride, int64_t before, int64_t max_tokens, int64_t &pages) {
  pages = 0;
  if (cached < 0 || fresh < 0 || cached + fresh > 16 * stride) return false;
  if (fresh > 0 && before + fresh > max_tokens) return false;
  for (int64_t t = cached; t < cached + fresh; ++t) pages += t % 16 == 0;
  return true;
}

static bool check(const std::vector<int> &cached, const std::vector<int> &fresh, int n_free, int max_tokens,
                  int stride) {
  int64_t rows = 0, pages = 0, before = 0, used = 0;
  for (size_t b = 0; b < cached.size(); ++b) {
    const BatchAsk a = batch_ask(cached[b], fresh[b], (int64_t)stride * 16);
    const bool ok = batch_grants(a, rows, pages, max_tokens, n_free);
    rows += a.rows;
    pages += a.pages > 0 ? a.pages : 0;
    int64_t need;
    bool want = wanted(cached[b], fresh[b], stride, before, max_tokens, need);
    used += need;
    if (want && need > 0 && used > n_free) want = false;
    if (fresh[b] > 0) before += fresh[b];
    if (ok != want || (ok && a.pages != need)) return false;
  }
  return true;
}

int main() {
  std::mt19937 rng(3);
  auto one_of = [&](std::initializer_list<int> x) { return x.begin()[rng() % x.size()]; };
  long n = 0;
  for (; n < 200000; ++n) {
    const int max_tokens = one_of({1, 2, 15, 16, 17, 32, 50, 100}), stride = 1 + rng() % 9, n_free = rng() % 12;
    std::vector<int> cached, fresh;
    for (int b = 1 + rng() % 6; b > 0; --b) {
      cached.push_back(one_of({0, 0, 1, 15, 16, 17, 40, -1, INT32_MAX}));
      fresh.push_back(one_of({0, 0, 1, 1, 2, 16, 17, 33, max_tokens - 1, max_tokens, max_tokens + 1, 2 * max_tokens, -3,
                              INT32_MAX, INT32_MIN}));
    }
    if (!check(cached, fresh, n_free, max_tokens, stride)) {
      printf("free %d rows %d stride %d:", n_free, max_tokens, stride);
      for (size_t b = 0; b < cached.size(); ++b) printf(" %d+%d", cached[b], fresh[b]);
      printf("\n");
      return 0;
    }
  }
  printf("ok %ld\n", n);
  return 0;
}
