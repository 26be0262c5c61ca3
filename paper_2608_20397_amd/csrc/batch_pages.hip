// A ragged batch laid out on the device: from every sequence's cached and fresh tokens, the rows of each (q_start),
// its new length, pages out of the free list for the tokens that need them, and position and cache slot of every row.
//
//   need[b]    = ceil((cached + fresh) / 16) - ceil(cached / 16)
//   q_start[b] = fresh[0] + .. + fresh[b - 1];  the pages of b are the free list's entries n_free - 1 - (need[0] + ..
//                + need[b - 1]) downwards
//
// Latency-bound: a few words a row.  Every workgroup forms both sums over all sequences for itself (one pass, kept in
// LDS; the lengths of a batch are some KB and come from the L2), then takes its share of the rows, whose sequence it
// finds by bisection; so the launch is one kernel without a word exchanged between workgroups.  A new page's map entry
// is written by the row that fills its first slot: a page behind the cached tokens starts with a fresh one.
#include "device_common.h"
#include "launch_batch.h"

#include <algorithm>

namespace nexus {

namespace {

constexpr int kThreads = 1024;

struct Two {
  int64_t rows, pages;
};

}  // namespace

__global__ __launch_bounds__(kThreads) void batch_pages_kernel(const BatchPagesLaunch p, int rows_per_wg) {
  extern __shared__ int32_t sums[];           // [n_seqs] rows up to and with b, [n_seqs] pages before b (-1: refused)
  __shared__ Two waves[kThreads / 64];
  __shared__ int32_t granted;
  int32_t *upto = sums, *before = sums + p.n_seqs;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n_free = min(max(p.n_free[0], 0), p.free_capacity);
  if (tid == 0) granted = 0;

  // rows and pages that sequence b asks for; pages -1: its lengths are not valid
  const int64_t capacity = (int64_t)p.map_stride * kPage;
  auto ask = [&](int b, int &rows, int &pages) {
    const int c = p.cached[b], f = p.fresh[b];
    rows = min(max(f, 0), p.max_tokens);
    const int64_t n = (int64_t)c + f;
    pages = c < 0 || f < 0 || n > capacity ? -1 : (int)((n + kPage - 1) / kPage - ((int64_t)c + kPage - 1) / kPage);
  };
  // a thread sums a run of neighbouring sequences, the workgroup the runs
  const int run = (p.n_seqs + kThreads - 1) / kThreads;
  const int b0 = min(tid * run, p.n_seqs), b1 = min(b0 + run, p.n_seqs);
  // (a sequence whose rows go past max_tokens asks for no pages either; the sum of rows decides, so it comes first)
  int64_t rows = 0;
  for (int b = b0; b < b1; ++b) {
    int r, g;
    ask(b, r, g);
    rows += r;
  }
  auto scan = [&](int64_t x) {                // sum over the threads before this one
    int64_t s = x;
    for (int off = 1; off < 64; off <<= 1) {
      const int64_t y = __shfl_up(s, off);
      if (lane >= off) s += y;
    }
    if (lane == 63) waves[wave].rows = s;
    __syncthreads();
    int64_t base = 0;
    for (int w = 0; w < wave; ++w) base += waves[w].rows;
    __syncthreads();
    return base + s - x;
  };
  int64_t r0 = scan(rows);
  int64_t pages = 0;
  {
    int64_t at = r0;
    for (int b = b0; b < b1; ++b) {
      int r, g;
      ask(b, r, g);
      at += r;
      upto[b] = (int32_t)min(at, (int64_t)p.max_tokens);
      pages += g > 0 && at <= p.max_tokens ? g : 0;     // (g > 0: it has rows)
    }
  }
  int64_t g0 = scan(pages);
  {
    int64_t at = r0;
    int most = 0;
    for (int b = b0; b < b1; ++b) {
      int r, g;
      ask(b, r, g);
      at += r;
      bool ok = g >= 0 && (r == 0 || at <= p.max_tokens);
      if (ok && g > 0) {
        ok = g0 + g <= n_free;
        if (ok) most = (int)(g0 + g);
        g0 += g;
      }
      before[b] = ok ? (int32_t)(g > 0 ? g0 - g : 0) : -1;
      if (blockIdx.x == 0) {
        p.seq_len[b] = ok ? p.cached[b] + p.fresh[b] : 0;
        p.q_start[b + 1] = upto[b];
      }
    }
    if (most > 0) atomicMax(&granted, most);
  }
  __syncthreads();
  if (blockIdx.x == 0 && tid == 0) {
    p.q_start[0] = 0;
    p.n_left[0] = n_free - granted;
  }
  const int64_t t0 = (int64_t)blockIdx.x * rows_per_wg;
  const int t1 = (int)min(t0 + rows_per_wg, (int64_t)p.max_tokens);
  for (int t = (int)t0 + tid; t < t1; t += kThreads) {
    // the first sequence whose rows reach past t
    int lo = 0, hi = p.n_seqs;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (upto[mid] > t) hi = mid;
      else lo = mid + 1;
    }
    int pos = -1, slot = -1;
    if (lo < p.n_seqs && before[lo] >= 0) {
      const int c = p.cached[lo];
      pos = c + t - (lo > 0 ? upto[lo - 1] : 0);
      const int page = pos >> kPageShift, held = (int)(((int64_t)c + kPage - 1) >> kPageShift);
      int32_t *entry = p.maps + (size_t)lo * p.map_stride + page;
      int32_t phys;
      if (page < held) {
        phys = *entry;
      } else {
        phys = p.free_pages[n_free - 1 - (before[lo] + page - held)];
        if ((pos & (kPage - 1)) == 0) *entry = phys;
      }
      slot = phys * kPage + (pos & (kPage - 1));
    }
    p.pos[t] = pos;
    p.slot[t] = slot;
  }
}

hipError_t launch_batch_pages(const BatchPagesLaunch &p, hipStream_t stream) {
  const size_t lds = (size_t)p.n_seqs * 2 * sizeof(int32_t);
  // two rows a thread, at most two workgroups a CU
  const int64_t per = std::max<int64_t>(2 * kThreads, ((int64_t)p.max_tokens + 511) / 512);
  const int rows_per_wg = (int)std::min<int64_t>(per, p.max_tokens);
  const dim3 grid((p.max_tokens + rows_per_wg - 1) / rows_per_wg);
  if (lds > 48 * 1024) {
    const hipError_t e = hipFuncSetAttribute((const void *)batch_pages_kernel,
                                             hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(batch_pages_kernel, grid, dim3(kThreads), lds, stream, p, rows_per_wg);
  return hipGetLastError();
}

}  // namespace nexus
