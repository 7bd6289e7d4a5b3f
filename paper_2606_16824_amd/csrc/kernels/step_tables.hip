// Block tables and slot maps of a serving step, from request lengths on the GPU.
//
// With held_b = ceil(Lp_b / P) and need_b = ceil((Lp_b + Ls_b) / P) (both at most the
// table's row), sequence b takes need_b - held_b pages of the free list, those from F_b
// on, F the exclusive sum of need - held; its packed rows start at cu_b, the exclusive sum
// of Ls.  Token t belongs to the last sequence with cu_b <= t (one that has new tokens).
//
// Bound by latency: the smallest steps write a few hundred bytes, the largest a few MB.
// So there is one launch where possible: with at most kStepTablesLdsSeqs sequences every
// workgroup sums all lengths itself into its LDS (28 KB of cached reads at 3500
// sequences), which needs no wait between workgroups, and then takes its share of the
// tokens and pages, each thread searching its sequence in LDS.  A thread reads the lengths
// of its (at most four) sequences at once.  Longer lists are summed by one workgroup into
// the workspace first.  All arithmetic on lengths is in 32 bits, clipped, with shifts for the
// page size: in 64 bits with divisions the largest steps were bound by it.  A page's and a
// token's loads go out together, and a workgroup of its own sums `info`.  Time in a graph of 8
// sequences 2.8-3.0 us (3.8 with `info` by the last workgroup and pages before tokens), of 200
// with 25k tokens 4.2-4.5, of 3500 with 304k tokens 9.7-9.8 us (20.7 in 64 bits), of 9000 with 798k
// tokens, in two launches, 36 us.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>

#include "../cw_internal.h"

namespace cw {
namespace {

constexpr int kScanThreads = 1024;
constexpr int kPer = 4;  // sequences per thread of the one-launch form
constexpr int kMaxBlocks = 1024;
// Of 1024 threads, which all sum the lengths (2.5 us of vector work at four waves per SIMD): one
// to a CU, and info's. 3500 sequences with 304k tokens: 298 workgroups 11.0 us, 255 9.7.
constexpr int kMaxWideBlocks = 255;

// Sums of lengths are clipped at INT32_MAX (rows and entries past it exist nowhere); both
// terms are at most that, so their sum fits uint32.
__device__ __forceinline__ uint32_t clip_add(uint32_t a, uint32_t b) { return min(a + b, uint32_t(INT32_MAX)); }

// What a sequence's lengths ask for, in at most bt_stride pages; negative lengths count as none.
struct Want {
  uint32_t lp, ls;
  int32_t held, fresh;
  bool over;  // more pages than a row of the table holds
};
__device__ __forceinline__ int32_t pages_of(const StepTablesParams& p, uint32_t n) {
  return static_cast<int32_t>((n + (1u << p.page_shift) - 1u) >> p.page_shift);  // (n at most INT32_MAX)
}
__device__ __forceinline__ Want want_of(const StepTablesParams& p, int32_t lp, int32_t ls) {
  Want w;
  w.lp = static_cast<uint32_t>(max(lp, 0));
  w.ls = static_cast<uint32_t>(max(ls, 0));
  // (two lengths, rounded up, may pass 32 bits: their pages are counted without that sum)
  const uint32_t n = w.lp + w.ls;
  const int32_t need = static_cast<int32_t>((n >> p.page_shift) + ((n & ((1u << p.page_shift) - 1u)) != 0u ? 1u : 0u));
  w.over = need > p.bt_stride;
  w.held = min(pages_of(p, w.lp), p.bt_stride);
  w.fresh = min(need, p.bt_stride) - w.held;
  return w;
}
__device__ __forceinline__ Want want_of(const StepTablesParams& p, int b) {
  return want_of(p, p.prefix_lens[b], p.suffix_lens[b]);
}

struct Sums {
  uint32_t tokens, pages;
};
__device__ __forceinline__ Sums operator+(Sums a, Sums b) {
  return Sums{clip_add(a.tokens, b.tokens), clip_add(a.pages, b.pages)};
}

// Exclusive sums of `mine` over the workgroup's threads; *all: over all of them.
template <int N>
__device__ __forceinline__ Sums block_exclusive(Sums mine, Sums* all) {
  __shared__ Sums waves[N / 64];
  const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  Sums inc = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const Sums up{__shfl_up(inc.tokens, d), __shfl_up(inc.pages, d)};
    if (lane >= d) inc = inc + up;
  }
  if (lane == 63) waves[wave] = inc;
  const Sums left{__shfl_up(inc.tokens, 1), __shfl_up(inc.pages, 1)};
  __syncthreads();
  Sums before{0, 0}, total{0, 0};
#pragma unroll
  for (int w = 0; w < N / 64; ++w) {
    if (w < wave) before = before + waves[w];
    total = total + waves[w];
  }
  __syncthreads();  // `waves` may be written again
  *all = total;
  return lane == 0 ? before : before + left;
}

// First new-token row and first free-list entry of every sequence (and the totals at
// index n).  A thread's sequences are consecutive; with PER > 0 at most PER, their lengths
// read at once (and their prefix lengths kept in lens).
template <int N, int PER>
__device__ __forceinline__ void sum_lengths(const StepTablesParams& p, int32_t* rows, int32_t* pages, int32_t* lens) {
  const int per = PER > 0 ? PER : (p.num_seqs + N - 1) / N;
  const int b0 = min(int(threadIdx.x) * per, p.num_seqs), b1 = min(b0 + per, p.num_seqs);
  Sums mine{0, 0}, all;
  auto put = [&](int b, Sums at) {
    rows[b] = static_cast<int32_t>(at.tokens);
    pages[b] = static_cast<int32_t>(at.pages);
  };
  if constexpr (PER > 0) {
    int32_t lp[PER], ls[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      lp[i] = b0 + i < b1 ? p.prefix_lens[b0 + i] : 0;
      ls[i] = b0 + i < b1 ? p.suffix_lens[b0 + i] : 0;
    }
    Sums own[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const Want w = want_of(p, lp[i], ls[i]);
      own[i] = Sums{w.ls, static_cast<uint32_t>(w.fresh)};
      mine = mine + own[i];
    }
    Sums at = block_exclusive<N>(mine, &all);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (b0 + i < b1) {
        put(b0 + i, at);
        lens[b0 + i] = lp[i];
      }
      at = at + own[i];
    }
  } else {
    for (int b = b0; b < b1; ++b) {
      const Want w = want_of(p, b);
      mine = mine + Sums{w.ls, static_cast<uint32_t>(w.fresh)};
    }
    Sums at = block_exclusive<N>(mine, &all);
    for (int b = b0; b < b1; ++b) {
      const Want w = want_of(p, b);
      put(b, at);
      at = at + Sums{w.ls, static_cast<uint32_t>(w.fresh)};
    }
  }
  if (threadIdx.x == 0) put(p.num_seqs, all);
}

// The step's totals, unclipped (one workgroup).
template <int N>
__device__ __forceinline__ void put_info(const StepTablesParams& p) {
  __shared__ int64_t parts[N / 64][3];
  int64_t x[3] = {0, 0, 0};
  for (int b = threadIdx.x; b < p.num_seqs; b += N) {
    const Want w = want_of(p, b);
    x[0] += w.fresh;
    x[1] += w.ls;
    x[2] += w.over ? 1 : 0;
  }
#pragma unroll
  for (int k = 0; k < 3; ++k) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) x[k] += __shfl_xor(x[k], d);
    if (threadIdx.x % 64 == 0) parts[threadIdx.x / 64][k] = x[k];
  }
  __syncthreads();
  if (threadIdx.x < 3) {
    int64_t sum = 0;
    for (int w = 0; w < N / 64; ++w) sum += parts[w][threadIdx.x];
    p.info[threadIdx.x] = sum;
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

// The share of `me` among `of` workgroups of the tokens, of the new pages and of cu_rows;
// `lens`: the prefix lengths as given.
__device__ __forceinline__ void fill(const StepTablesParams& p, const int32_t* rows, const int32_t* pages,
                                     const int32_t* lens, int me, int of) {
  const int n = p.num_seqs;
  const int total_rows = rows[n], total_pages = pages[n];
  const int64_t stride = int64_t(of) * blockDim.x, first = int64_t(me) * blockDim.x + threadIdx.x;
  auto free_page = [&](uint32_t f) -> int32_t { return f < uint32_t(p.num_free) ? p.free_pages[f] : -1; };
  auto held_of = [&](uint32_t lp) -> int32_t { return min(pages_of(p, lp), p.bt_stride); };
  const int64_t last = max(int64_t(total_pages), max(int64_t(p.max_tokens), int64_t(n) + 1));
  for (int64_t i = first; i < last; i += stride) {
    // new page i and token i: their loads go out before either is stored
    const bool page = i < total_pages, token = i < p.max_tokens;
    int32_t new_page = -1;
    int64_t entry = 0;
    if (page) {
      const int b = last_at_most(pages, n, static_cast<int32_t>(i));
      entry = int64_t(b) * p.bt_stride + held_of(max(lens[b], 0)) + (static_cast<int32_t>(i) - pages[b]);
      new_page = free_page(static_cast<uint32_t>(i));
    }
    int32_t seq = -1, pos = -1, pg = -1, in_page = 0;
    if (token && i < total_rows) {
      seq = last_at_most(rows, n, static_cast<int32_t>(i));
      const uint32_t lp = max(lens[seq], 0);
      const int32_t held = held_of(lp);
      const uint32_t at = lp + static_cast<uint32_t>(i - rows[seq]);
      const int32_t col = static_cast<int32_t>(at >> p.page_shift);
      pos = static_cast<int32_t>(min(at, uint32_t(INT32_MAX)));
      in_page = static_cast<int32_t>(at & ((1u << p.page_shift) - 1u));
      if (col < p.bt_stride && p.slots != nullptr)
        // a page of this step is read from the free list: another workgroup writes the table
        pg = col < held ? p.block_table[int64_t(seq) * p.bt_stride + col]
                        : free_page(static_cast<uint32_t>(pages[seq]) + static_cast<uint32_t>(col - held));
    }
    if (i <= n && p.cu_rows != nullptr) p.cu_rows[i] = rows[i];
    if (page) p.block_table[entry] = new_page;
    if (token) {
      if (p.seq_ids != nullptr) p.seq_ids[i] = seq;
      if (p.positions != nullptr) p.positions[i] = pos;
      if (p.slots != nullptr) p.slots[i] = pg >= 0 ? (int64_t(pg) << p.page_shift) + in_page : -1;
    }
  }
}

template <int N>
__global__ __launch_bounds__(N) void step_tables_kernel(StepTablesParams p) {
  __shared__ int32_t rows[N * kPer + 1], pages[N * kPer + 1], lens[N * kPer];
  const int fills = static_cast<int>(gridDim.x) - (p.info != nullptr ? 1 : 0);
  if (static_cast<int>(blockIdx.x) == fills) {  // the last workgroup, besides the others
    put_info<N>(p);
    return;
  }
  sum_lengths<N, kPer>(p, rows, pages, lens);
  __syncthreads();
  fill(p, rows, pages, lens, static_cast<int>(blockIdx.x), fills);
}

__global__ __launch_bounds__(kScanThreads) void step_tables_sum_kernel(StepTablesParams p) {
  sum_lengths<kScanThreads, 0>(p, p.sums, p.sums + p.num_seqs + 1, nullptr);
  if (p.info != nullptr) put_info<kScanThreads>(p);
}

__global__ __launch_bounds__(256) void step_tables_fill_kernel(StepTablesParams p) {
  fill(p, p.sums, p.sums + p.num_seqs + 1, p.prefix_lens, static_cast<int>(blockIdx.x), static_cast<int>(gridDim.x));
}

}  // namespace

hipError_t launch_step_tables(const StepTablesParams& p, hipStream_t stream) {
  // a token (or entry of cu_rows) per thread; a step has at most as many new pages as new tokens
  const int64_t work = std::max<int64_t>(p.max_tokens, p.num_seqs + 1);
  auto grid = [&](int64_t threads, int more) {
    return dim3(static_cast<unsigned>(std::min<int64_t>((work + threads - 1) / threads, threads == kScanThreads ? kMaxWideBlocks : kMaxBlocks) + more));
  };
  const int info = p.info != nullptr ? 1 : 0;  // a workgroup of its own in the one-launch form
  static_assert(1024 * kPer == kStepTablesLdsSeqs, "the largest one-launch form");
  if (p.num_seqs <= 64 * kPer) {
    hipLaunchKernelGGL((step_tables_kernel<64>), grid(64, info), dim3(64), 0, stream, p);
    return hipGetLastError();
  }
  if (p.num_seqs <= kStepTablesLdsSeqs) {
    hipLaunchKernelGGL((step_tables_kernel<1024>), grid(kScanThreads, info), dim3(kScanThreads), 0, stream, p);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(step_tables_sum_kernel, dim3(1), dim3(kScanThreads), 0, stream, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(step_tables_fill_kernel, grid(256, 0), dim3(256), 0, stream, p);
  return hipGetLastError();
}

}  // namespace cw
