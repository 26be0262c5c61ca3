// A ragged batch laid out on the device: from every sequence's cached and fresh tokens, the rows of each (q_start),
// its new length, pages out of the free list for the tokens that need them, and position and cache slot of every row.
//
//   need[b]    = ceil((cached + fresh) / 16) - ceil(cached / 16)
//   q_start[b] = fresh[0] + .. + fresh[b - 1];  the pages of b are the free list's entries n_free - 1 - (need[0] + ..
//                + need[b - 1]) downwards
//
// Latency-bound: a few words a row.  Every workgroup forms both sums over all sequences for itself (one scan; the
// lengths of a batch are some KB and come from the L2), keeps what a row needs of its sequence in LDS, then takes its
// share of the rows, whose sequence it finds by bisection; so the launch is one kernel without a word exchanged between
// workgroups, and a row's only load is that of its page.  A new page's map entry is written by the row that fills its
// first slot: a page behind the cached tokens starts with a fresh one.
// A step of 32 sequences 4.1 us; 65 thousand rows of 256 sequences 6.6 (0.6 MB; three passes over the lengths, two rows a
// thread: 10.4).
#include "device_common.h"
#include "launch_batch.h"

#include <algorithm>

namespace nexus {

namespace {

constexpr int kThreads = 1024;
constexpr int kRefused = INT32_MIN;

}  // namespace

__global__ __launch_bounds__(kThreads) void batch_pages_kernel(const BatchPagesLaunch p, int rows_per_wg) {
  // per sequence: rows up to and with it; cached tokens minus rows before it, or kRefused; pages before it minus pages
  // that it holds
  extern __shared__ int32_t sums[];
  __shared__ int64_t wave_rows[kThreads / 64], wave_pages[kThreads / 64];
  __shared__ int32_t granted;
  int32_t *upto = sums, *shift = sums + p.n_seqs, *ahead = sums + 2 * p.n_seqs;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n_free = min(max(p.n_free[0], 0), p.free_capacity);
  if (tid == 0) granted = 0;

  const int64_t capacity = (int64_t)p.map_stride * kPage;
  // a thread sums a run of neighbouring sequences (one, in batches of up to 1024), the workgroup the runs.  Sequences
  // whose rows pass max_tokens may count in the sum of pages: all that come after them are refused or need none.
  const int run = (p.n_seqs + kThreads - 1) / kThreads;
  const int b0 = min(tid * run, p.n_seqs), b1 = min(b0 + run, p.n_seqs);
  int c0 = 0, f0 = 0;
  int64_t rows = 0, pages = 0;
  for (int b = b0; b < b1; ++b) {
    c0 = p.cached[b];
    f0 = p.fresh[b];
    const BatchAsk a = batch_ask(c0, f0, capacity);
    rows += a.rows;
    pages += max(a.pages, 0);
  }
  int64_t r0 = rows, g0 = pages;
  for (int off = 1; off < 64; off <<= 1) {
    const int64_t x = __shfl_up(r0, off), y = __shfl_up(g0, off);
    if (lane >= off) {
      r0 += x;
      g0 += y;
    }
  }
  if (lane == 63) {
    wave_rows[wave] = r0;
    wave_pages[wave] = g0;
  }
  __syncthreads();
  r0 -= rows;
  g0 -= pages;
  for (int w = 0; w < wave; ++w) {
    r0 += wave_rows[w];
    g0 += wave_pages[w];
  }
  int most = 0;
  for (int b = b0; b < b1; ++b) {
    if (run > 1) {
      c0 = p.cached[b];
      f0 = p.fresh[b];
    }
    const BatchAsk a = batch_ask(c0, f0, capacity);
    const bool ok = batch_grants(a, r0, g0, p.max_tokens, n_free);
    if (ok && a.pages > 0) most = (int)(g0 + a.pages);
    // (of a sequence without rows neither is looked up)
    shift[b] = ok ? (int32_t)(c0 - min(r0, (int64_t)p.max_tokens)) : kRefused;
    ahead[b] = ok && a.pages > 0 ? (int32_t)(g0 - batch_pages_of(c0)) : 0;
    r0 += a.rows;
    g0 += max(a.pages, 0);
    upto[b] = (int32_t)min(r0, (int64_t)p.max_tokens);
    if (blockIdx.x == 0) {
      p.seq_len[b] = ok ? c0 + f0 : 0;
      p.q_start[b + 1] = upto[b];
    }
  }
  if (most > 0) atomicMax(&granted, most);
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
    if (lo < p.n_seqs && shift[lo] != kRefused) {
      const int c = shift[lo] + (lo > 0 ? upto[lo - 1] : 0);
      pos = shift[lo] + t;
      const int page = pos >> kPageShift;
      int32_t *entry = p.maps + (size_t)lo * p.map_stride + page;
      int32_t phys;
      if (page < batch_pages_of(c)) {
        phys = *entry;
      } else {
        phys = p.free_pages[n_free - 1 - (ahead[lo] + page)];
        if ((pos & (kPage - 1)) == 0) *entry = phys;
      }
      if ((uint32_t)phys < (1u << 27)) slot = phys * kPage + (pos & (kPage - 1));      // (no page's number: no slot)
    }
    p.pos[t] = pos;
    p.slot[t] = slot;
  }
}

hipError_t launch_batch_pages(const BatchPagesLaunch &p, hipStream_t stream) {
  const size_t lds = (size_t)p.n_seqs * 3 * sizeof(int32_t);
  // a row a thread, at most two workgroups a CU
  const int64_t per = std::max<int64_t>(kThreads, ((int64_t)p.max_tokens + 511) / 512);
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
