// Block tables and slot maps of a serving step, from request lengths on the GPU.
//
// With held_b = ceil(Lp_b / P) and need_b = ceil((Lp_b + Ls_b) / P) (both at most the
// table's row), sequence b takes need_b - held_b pages of the free list, those from F_b
// on, F the exclusive sum of need - held; its packed rows start at cu_b, the exclusive sum
// of Ls.  Token t belongs to the last sequence with cu_b <= t (one that has new tokens).
//
// Bound by latency: the smallest steps write a few hundred bytes, the largest a few MB.
// So there is one launch where possible: with at most kLdsSeqs sequences every workgroup
// sums all lengths itself into its LDS (28 KB of cached reads at 3500 sequences), which
// needs no wait between workgroups, and then takes its share of the tokens and pages,
// each thread searching its sequence in LDS.  Longer lists are summed by one workgroup
// into the workspace first.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>

#include "../cw_internal.h"

namespace cw {
namespace {

constexpr int kThreads = 256;
constexpr int kScanThreads = 1024;
constexpr int kTokensPerThread = 4;
constexpr int kMaxBlocks = 1024;

__device__ __forceinline__ int32_t clip(int64_t x) { return x > INT32_MAX ? INT32_MAX : static_cast<int32_t>(x); }

// What a sequence's lengths ask for; negative lengths count as none.
struct Want {
  int32_t lp, ls, held, need;
  bool over;  // more pages than a row of the table holds
};
__device__ __forceinline__ Want want_of(const StepTablesParams& p, int b) {
  Want w;
  w.lp = max(p.prefix_lens[b], 0);
  w.ls = max(p.suffix_lens[b], 0);
  const int64_t held = (int64_t(w.lp) + p.page_size - 1) / p.page_size;
  const int64_t need = (int64_t(w.lp) + w.ls + p.page_size - 1) / p.page_size;
  w.over = need > p.bt_stride;
  w.held = static_cast<int32_t>(min(held, int64_t(p.bt_stride)));
  w.need = static_cast<int32_t>(min(need, int64_t(p.bt_stride)));
  return w;
}

struct Sums {
  int64_t tokens, pages, over;
};
__device__ __forceinline__ Sums operator+(Sums a, Sums b) {
  return Sums{a.tokens + b.tokens, a.pages + b.pages, a.over + b.over};
}

// Exclusive sums of `mine` over the workgroup's threads; *all: over all of them.
template <int N>
__device__ __forceinline__ Sums block_exclusive(Sums mine, Sums* all) {
  __shared__ Sums waves[N / 64];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  Sums inc = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const Sums up{__shfl_up(inc.tokens, d), __shfl_up(inc.pages, d), __shfl_up(inc.over, d)};
    if (lane >= d) inc = inc + up;
  }
  if (lane == 63) waves[wave] = inc;
  __syncthreads();
  Sums before{0, 0, 0}, total{0, 0, 0};
#pragma unroll
  for (int w = 0; w < N / 64; ++w) {
    if (w < wave) before = before + waves[w];
    total = total + waves[w];
  }
  __syncthreads();  // `waves` may be written again
  *all = total;
  return before + Sums{inc.tokens - mine.tokens, inc.pages - mine.pages, inc.over - mine.over};
}

// First new-token row and first free-list entry of every sequence (and the totals at
// index n), clipped to int32: rows and entries past INT32_MAX exist nowhere.
template <int N, class Rows, class Pages>
__device__ __forceinline__ Sums sum_lengths(const StepTablesParams& p, Rows rows, Pages pages) {
  const int per = (p.num_seqs + N - 1) / N;
  const int b0 = min(int(threadIdx.x) * per, p.num_seqs), b1 = min(b0 + per, p.num_seqs);
  Sums mine{0, 0, 0};
  for (int b = b0; b < b1; ++b) {
    const Want w = want_of(p, b);
    mine = mine + Sums{w.ls, w.need - w.held, w.over ? 1 : 0};
  }
  Sums all;
  Sums at = block_exclusive<N>(mine, &all);
  for (int b = b0; b < b1; ++b) {
    const Want w = want_of(p, b);
    rows[b] = clip(at.tokens);
    pages[b] = clip(at.pages);
    at = at + Sums{w.ls, w.need - w.held, 0};
  }
  if (threadIdx.x == 0) {
    rows[p.num_seqs] = clip(all.tokens);
    pages[p.num_seqs] = clip(all.pages);
  }
  return all;
}

__device__ __forceinline__ void put_info(const StepTablesParams& p, Sums all) {
  if (p.info != nullptr && threadIdx.x == 0) {
    p.info[0] = all.pages;
    p.info[1] = all.tokens;
    p.info[2] = all.over;
  }
}

// The number of entries of first[0 .. n) that are <= x, less one (first[0] = 0, x >= 0).
template <class T>
__device__ __forceinline__ int last_at_most(const T* first, int n, int32_t x) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (first[mid] <= x) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// This workgroup's share of the tokens and of the new pages, and workgroup 0's cu_rows.
__device__ __forceinline__ void fill(const StepTablesParams& p, const int32_t* rows, const int32_t* pages) {
  const int n = p.num_seqs;
  const int total_rows = rows[n], total_pages = pages[n];
  const int64_t stride = int64_t(gridDim.x) * kThreads, first = int64_t(blockIdx.x) * kThreads + threadIdx.x;
  auto free_page = [&](int64_t f) -> int32_t { return f < p.num_free ? p.free_pages[f] : -1; };
  for (int64_t f = first; f < total_pages; f += stride) {
    const int b = last_at_most(pages, n, static_cast<int32_t>(f));
    const int col = want_of(p, b).held + static_cast<int32_t>(f - pages[b]);
    p.block_table[int64_t(b) * p.bt_stride + col] = free_page(f);
  }
  for (int64_t t = first; t < p.max_tokens; t += stride) {
    int32_t seq = -1, pos = -1;
    int64_t slot = -1;
    if (t < total_rows) {
      seq = last_at_most(rows, n, static_cast<int32_t>(t));
      const Want w = want_of(p, seq);
      const int64_t at = int64_t(w.lp) + (t - rows[seq]);
      const int64_t col = at / p.page_size;
      pos = clip(at);
      if (col < p.bt_stride && p.slots != nullptr) {
        // a page of this step is read from the free list: another workgroup writes the table
        const int32_t pg = col < w.held ? p.block_table[int64_t(seq) * p.bt_stride + col]
                                        : free_page(int64_t(pages[seq]) + (col - w.held));
        if (pg >= 0) slot = int64_t(pg) * p.page_size + at % p.page_size;
      }
    }
    if (p.seq_ids != nullptr) p.seq_ids[t] = seq;
    if (p.positions != nullptr) p.positions[t] = pos;
    if (p.slots != nullptr) p.slots[t] = slot;
  }
  if (p.cu_rows != nullptr)
    for (int64_t b = first; b <= n; b += stride) p.cu_rows[b] = rows[b];
}

__global__ __launch_bounds__(kThreads) void step_tables_kernel(StepTablesParams p) {
  __shared__ int32_t rows[kStepTablesLdsSeqs + 1], pages[kStepTablesLdsSeqs + 1];
  const Sums all = sum_lengths<kThreads>(p, rows, pages);
  if (blockIdx.x == 0) put_info(p, all);
  __syncthreads();
  fill(p, rows, pages);
}

__global__ __launch_bounds__(kScanThreads) void step_tables_sum_kernel(StepTablesParams p) {
  put_info(p, sum_lengths<kScanThreads>(p, p.sums, p.sums + p.num_seqs + 1));
}

__global__ __launch_bounds__(kThreads) void step_tables_fill_kernel(StepTablesParams p) {
  fill(p, p.sums, p.sums + p.num_seqs + 1);
}

}  // namespace

hipError_t launch_step_tables(const StepTablesParams& p, hipStream_t stream) {
  // (a step has at most as many new pages as new tokens)
  const int64_t work = std::max<int64_t>(p.max_tokens, p.num_seqs + 1);
  constexpr int64_t kPerBlock = int64_t(kThreads) * kTokensPerThread;
  const dim3 grid(static_cast<unsigned>(std::min<int64_t>((work + kPerBlock - 1) / kPerBlock, kMaxBlocks)));
  if (p.num_seqs <= kStepTablesLdsSeqs) {
    hipLaunchKernelGGL(step_tables_kernel, grid, dim3(kThreads), 0, stream, p);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(step_tables_sum_kernel, dim3(1), dim3(kScanThreads), 0, stream, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(step_tables_fill_kernel, grid, dim3(kThreads), 0, stream, p);
  return hipGetLastError();
}

}  // namespace cw
