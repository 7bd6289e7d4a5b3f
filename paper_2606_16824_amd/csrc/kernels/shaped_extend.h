// Attention with shaped scores for chunks of new tokens over a paged cache (the kernel; its
// instances are compiled by shaped_extend_d64.hip and shaped_extend_d128.hip).
//
// A workgroup of eight waves owns 256 packed query rows (token x query head of one kv head, 32
// per wave) and walks the keys that some row may see, 64 at a time.  S^T = K Q^T and O^T += V^T
// P^T with v_mfma_f32_32x32x16 (bf16; fp16 over fp8 pools), so that a lane owns a query row: its
// slope, position and limits are one register each.
//
// Keys are walked from the last to the first, so that a bias by distance, which is largest next to
// the token, meets the running max early (from the first key on, half of the blocks of steep
// heads raised it: 4096 tokens on 32768 keys 3.6 ms instead of 2.3).  An iteration has a key tile
// of 64 keys and two phases: the scores of the next tile beside the weights of this tile's lower 32
// keys, then this tile's values beside the weights of the next tile's upper 32 keys.  So each
// phase has as many matrix products as the other and half of the weights, and nothing in a phase
// waits for its products.  Where a lower block raises the running max, its upper block's weights
// are rescaled with O: the max is kept a whole number (of log2 units), so that this is exact.
// Key tiles are one ahead of value tiles; both rotate through two LDS stages, one barrier per
// iteration.
//
// Cap, bias, mask and running max enter where the weights are formed, from unscaled scores in
// fp32 (shaped_common.h): an uncapped weight is one fma and one exponential, a cap adds an
// exponential and a reciprocal, the bias one fma.  A masked score is replaced, not added to, so
// that nothing it holds matters.  The weights are rounded to the operand type (bf16: 2^-8
// relative at most) and their sum is taken after that, so numerator and denominator agree.  The
// running max is raised only when a half-row's weight sum passes 2^16 (or is not finite).
//
// Tiles that every row of the workgroup sees, wholly in the prefix or wholly among the new
// tokens, run in loops without row checks and masks; the tiles at the window's edge, at the
// prefix's end and at the diagonal take the general loop.  Rows before the first key that a row
// of the workgroup sees are not staged, and their pages not looked up.
//
// fp8 rows are widened into LDS, values with their page's scale, key codes as they are (fp16 holds
// them exactly): a key's page scale multiplies the scores in fp32.
//
// Bound by power without a cap (matrix cores busy 61% of the cycles at 1.6 GHz), with one by vector
// work beside the products (44% at 2.0): per 16 scores of a lane 112 vector operations, 48 of them
// transcendental.  Short workgroups by their start: some 16 us each beside the tiles (one of 64 keys
// 18.3 us, 32 of them 84).  4096 tokens on 32768 keys (2.34e12 operations: 32 query heads at D = 128, 64
// at D = 64): D = 128 2040 us (1145 TFLOP/s), cap 2540, slopes 2120, fp8 2270 to 2500; D = 64 2560, cap 3700,
// slopes 2550, fp8 2960.  fp8 instances of D = 128 with a cap or a bias spill 8 to 21 registers.
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

#include "../cw_internal.h"
#include "partial.h"
#include "shaped_common.h"

namespace cw {
namespace shaped {

// Read through the constant address space so that loads with a uniform address are
// scalar loads: waiting for them never waits for tile staging issued before them.
typedef __attribute__((address_space(4))) const int32_t const_i32;
typedef __attribute__((address_space(4))) const float const_f32;

constexpr int kWaves = 8, kThreads = kWaves * 64;

// What is known of the keys of an iteration: that they lie in the cached prefix or among the new
// tokens (one of them) and every row sees them, or nothing.
enum class Keys { kSeen, kAny };

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc_at(const void* base) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, -1, 0x00020000);
}

// 16 bytes per lane from base + voff + soff straight into LDS (lane l's bytes land at dst + 16 l).
// Not a template: see the extend kernel.
__device__ __forceinline__ void dma16(__amdgpu_buffer_rsrc_t r, lds_void* dst, uint32_t voff, uint32_t soff) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, dst, 16, voff, soff, 0, 0);
}

// Page scale s = p2 x fm: p2 a power of two (applied by the conversion), fm s's significand, rounded to fp16,
// times a power of two of its own: of a scale in [2^-14, 2) all of it (p2 = 1), of a larger one 1, of a
// smaller one 2^-14.  So what the conversion rounds, if anything (of scales below 2^-29), is multiplied with at
// most 2^-13, and a value is rounded once, by the product, also where fp16 has fewer bits left for it.
struct PageScale {
  float p2;
  f16x2 fm;
};
__device__ __forceinline__ PageScale page_scale(float s) {
  const uint32_t b = __float_as_uint(s);
  const uint32_t e = b & 0x7F800000u, em = min(max(e, 113u << 23), 127u << 23);
  const float p2 = __uint_as_float(e - em + (127u << 23));
  const _Float16 m = static_cast<_Float16>(__uint_as_float((b & 0x807FFFFFu) | em));
  return PageScale{p2, f16x2{m, m}};
}
template <bool HI>
__device__ __forceinline__ f16x2 fp8x2_f16x2(uint32_t w, float p2) {
  return __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(static_cast<int>(w), p2, HI);
}
__device__ __forceinline__ uint32_t as_u32(f16x2 v) { return __builtin_bit_cast(uint32_t, v); }
// Eight codes times their page's scale (values), or as they are (keys: exact).
__device__ __forceinline__ u32x4 fp8x8_f16x8(uint32_t lo, uint32_t hi, PageScale sc) {
  return u32x4{as_u32(fp8x2_f16x2<false>(lo, sc.p2) * sc.fm), as_u32(fp8x2_f16x2<true>(lo, sc.p2) * sc.fm),
               as_u32(fp8x2_f16x2<false>(hi, sc.p2) * sc.fm), as_u32(fp8x2_f16x2<true>(hi, sc.p2) * sc.fm)};
}
__device__ __forceinline__ u32x4 fp8x8_f16x8(uint32_t lo, uint32_t hi) {
  return u32x4{as_u32(fp8x2_f16x2<false>(lo, 1.f)), as_u32(fp8x2_f16x2<true>(lo, 1.f)),
               as_u32(fp8x2_f16x2<false>(hi, 1.f)), as_u32(fp8x2_f16x2<true>(hi, 1.f))};
}
__device__ __forceinline__ u32x4 bf16x8_f16x8(u32x4 x) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float lo = __uint_as_float(x[i] << 16), hi = __uint_as_float(x[i] & 0xFFFF0000u);
    r[i] = as_u32(f16x2{static_cast<_Float16>(lo), static_cast<_Float16>(hi)});
  }
  return r;
}
template <bool F16>
__device__ __forceinline__ f32x16 mfma16(u32x4 a, u32x4 b, f32x16 c) {
  if constexpr (F16)
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Chunk swizzles of the extend kernel: K rows read by ds_read_b128, V rows by
// ds_read_b64_tr_b16, both without bank conflicts.
template <int D>
__device__ __forceinline__ int k_swz(int row) {
  return D == 128 ? (swap_bits_2_3(row) & 15) : ((swap_bits_2_3(row) >> 1) & 7);
}
template <int D>
__device__ __forceinline__ int v_swz(int row) {
  return D == 128 ? 4 * (row & 3) : 4 * ((row >> 1) & 1);
}

template <int D, bool FP8>
struct Geo {
  static constexpr int RB = 2 * D;                   // bytes per 16-bit row in LDS
  static constexpr int CPR = D / 8;                  // 16-byte chunks per row
  static constexpr int RPI = 64 / CPR;               // rows per wave DMA instruction
  static constexpr int NI = BLOCK_N / RPI / kWaves;  // DMA instructions per wave and matrix
  static constexpr int TILE = BLOCK_N * RB;          // bytes of one matrix's tile
  static constexpr int KT = D / 16;                  // k-steps of K Q^T
  static constexpr int DB = D / 32;                  // 32-row blocks of O^T
  static constexpr int PRB = FP8 ? D : RB;           // bytes per pool row
  static constexpr int B8 = D / 8;                   // fp8 bytes each lane stages per matrix
  static constexpr int KS = BLOCK_N / 16;            // fp8: key scales kept per tile, one per 16 keys
  static_assert(NI * RPI == 8, "each wave stages 8 rows of a tile");
};

template <int D, bool FP8, bool CAP, bool BIAS, int AP>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2)))
void shaped_extend_kernel(ShapedParams sp, PlanArg<AP> ap) {
  using T = Geo<D, FP8>;
  const ExtendParams& p = sp.a;
  // stages of key and value tiles, each its own array so that the compiler can tell reads of
  // one stage from the DMA into another
  __shared__ __attribute__((aligned(1024))) uint8_t lds_k0[T::TILE];
  __shared__ __attribute__((aligned(1024))) uint8_t lds_k1[T::TILE];
  __shared__ __attribute__((aligned(1024))) uint8_t lds_v0[T::TILE];
  __shared__ __attribute__((aligned(1024))) uint8_t lds_v1[T::TILE];
  __shared__ int sh_lo[2][kWaves];

  const WorkItem it = plan_ptr<AP>(ap, p.ap_items, p.items)[blockIdx.x];
  if (it.seq < 0) return;  // idle padding item (uniform across the workgroup)
  const SeqInfo sq = plan_ptr<AP>(ap, p.ap_seqs, p.seqs)[it.seq];
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int h = lane >> 5, col = lane & 31;
  const int G = p.gqa_group, hkv = p.num_kv_heads, hq = hkv * G;
  const int kvh = it.kvh;
  const int lp = sq.lp, total_len = sq.lp + sq.ls;
  const int full = it.pad;  // tokens of the prefix mask, at most total_len
  const int pshift = sp.page_shift, P = 1 << pshift;
  const int32_t* bt = p.block_table + size_t(sq.bt_row) * p.bt_stride;
  const uint8_t* k_new = static_cast<const uint8_t*>(p.k_new);
  const uint8_t* v_new = static_cast<const uint8_t*>(p.v_new);

  // this lane's query row: position, keys [lo, lo + seen)
  const int r_local = wave * 32 + col;
  const bool row_ok = r_local < it.rows;
  const int r = it.q_row0 + r_local;
  const int t = r / G, g = r - t * G;
  const int pos = lp + t;
  const bool wave_active = wave * 32 < it.rows;
  const size_t out_row = size_t(sq.cu + t) * hq + size_t(kvh) * G + g;
  // over the workgroup's rows: the limits (causal, so monotonic) ...
  const int first_lim = lp + it.q_row0 / G + 1;  // of the workgroup's first row, without the prefix mask
  const int min_lim = max(first_lim, full);
  // ... and the first keys
  auto window_lo = [&](int at) { return sp.window > 0 ? max(0, at - sp.window + 1) : 0; };
  int lo = window_lo(pos);
  int wg_lo = window_lo(first_lim - 1), wg_lo_max = window_lo(lp + (it.q_row0 + it.rows - 1) / G);
  if (sp.begins != nullptr) {
    if (row_ok) lo = max(lo, min(sp.begins[sq.cu + t], total_len));
    int mn = row_ok ? lo : 0x7FFFFFFF, mx = row_ok ? lo : 0;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      mn = min(mn, __shfl_xor(mn, d));
      mx = max(mx, __shfl_xor(mx, d));
    }
    if (lane == 0) {
      sh_lo[0][wave] = mn;
      sh_lo[1][wave] = mx;
    }
  }
  const int lim = max(pos + 1, full);
  const uint32_t seen = row_ok ? max(0, lim - lo) : 0;

  // stale LDS must be finite: rows that are not staged are multiplied with weight 0
  for (int i = tid; i < T::TILE / 16; i += kThreads) {
    reinterpret_cast<u32x4*>(lds_k0)[i] = u32x4{0u, 0u, 0u, 0u};
    reinterpret_cast<u32x4*>(lds_k1)[i] = u32x4{0u, 0u, 0u, 0u};
    reinterpret_cast<u32x4*>(lds_v0)[i] = u32x4{0u, 0u, 0u, 0u};
    reinterpret_cast<u32x4*>(lds_v1)[i] = u32x4{0u, 0u, 0u, 0u};
  }

  // Q^T as the B operand: k-step kk holds dims 16 kk + 8 h + [0, 8) of this row
  u32x4 qf[T::KT];
  {
    const uint16_t* qrow = static_cast<const uint16_t*>(p.q) + out_row * D;
#pragma unroll
    for (int kk = 0; kk < T::KT; ++kk) {
      u32x4 v = {0u, 0u, 0u, 0u};
      if (row_ok) v = *reinterpret_cast<const u32x4*>(qrow + 16 * kk + 8 * h);
      qf[kk] = FP8 ? bf16x8_f16x8(v) : v;
    }
  }
  float slope2 = 0.f;
  if (BIAS && row_ok) slope2 = sp.slopes[kvh * G + g] * kLog2e;

  __syncthreads();  // zero fill done before any tile lands; sh_lo complete
  if (sp.begins != nullptr) {
    wg_lo = 0x7FFFFFFF;
    wg_lo_max = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      wg_lo = min(wg_lo, sh_lo[0][w]);
      wg_lo_max = max(wg_lo_max, sh_lo[1][w]);
    }
    wg_lo = __builtin_amdgcn_readfirstlane(wg_lo);
    wg_lo_max = __builtin_amdgcn_readfirstlane(wg_lo_max);
  }
  // the item's keys from the first tile that holds one which some row may see
  const int kv_end = it.kv_end;
  const int kv_begin = max(it.kv_begin, min(wg_lo, kv_end) / BLOCK_N * BLOCK_N);
  const int n_tiles = (kv_end - kv_begin + BLOCK_N - 1) / BLOCK_N;  // (0 where nothing is visible)
  const int new_stop = min(total_len, kv_end);  // new tokens at or past it are not staged

  // ---- staging.  Wave w stages rows [8 w, 8 w + 8) of a tile, which lie in one page.  16-bit
  // rows: DMA instruction i covers rows 8 w + RPI i on, lane l fetches the chunk that belongs at
  // position l % CPR of row l / CPR of them.
  const int dma_row = lane / T::CPR, dma_pos = lane % T::CPR;
  const int wrow0 = 8 * wave;
  // Its source lies at a lane's offset (k_off or v_off, in a page block; behind it new_off more
  // among the new tokens' rows) and the wave's and the instruction's, which are scalars; four rows
  // on, a key's swizzle differs in the bit of 8 (128 bytes), a value's not at all.
  const int lane_row = wrow0 + dma_row;
  const uint32_t k_off = uint32_t(dma_row * T::RB + 16 * (dma_pos ^ k_swz<D>(lane_row)));
  const uint32_t v_off = uint32_t(dma_row * T::RB + 16 * (dma_pos ^ v_swz<D>(lane_row)));
  const uint32_t new_off = uint32_t(dma_row) * uint32_t((hkv - 1) * T::RB);
  static_assert(T::NI == 1 || (T::NI == 2 && T::RPI == 4), "the second instruction's swizzle");
  const uint32_t page_row = uint32_t(wrow0 & (P - 1)) * T::RB, new_row = uint32_t(wrow0) * uint32_t(hkv * T::RB);
  // instruction i of a matrix, rows `row` bytes apart
  auto fetch = [&](__amdgpu_buffer_rsrc_t rs, uint8_t* dst, uint32_t off, uint32_t more, int i, uint32_t first, uint32_t row,
                   bool keys) __attribute__((always_inline)) {
    dma16(rs, (lds_void*)(dst + (wrow0 + T::RPI * i) * T::RB), (keys && i == 1 ? off ^ 128u : off) + more,
          first + i * T::RPI * row);
  };
  const uint32_t page_bytes = uint32_t(P) * T::PRB;  // one (page, head) block
  const size_t page_stride = size_t(hkv) * page_bytes;
  const uint8_t* k_pool = static_cast<const uint8_t*>(p.k_pool) + size_t(kvh) * page_bytes;
  const uint8_t* v_pool = static_cast<const uint8_t*>(p.v_pool) + size_t(kvh) * page_bytes;
  // fp8 rows.  D = 64: lane l stages 8 bytes of row 8 w + l / 8.  D = 128: load u of lane
  // l fetches what belongs at position l % 16 of row 8 w + 4 u + l / 16 (four rows on, a key's
  // swizzle differs in the bit of 8, a value's not at all).
  const int r8 = D == 128 ? wrow0 + (lane >> 4) : wrow0 + (lane >> 3);
  const int pos8 = D == 128 ? lane & 15 : lane & 7;
  const uint32_t k8_off = uint32_t((r8 & (P - 1)) * D + 8 * (pos8 ^ k_swz<D>(r8)));
  const uint32_t v8_off = uint32_t((r8 & (P - 1)) * D + 8 * (pos8 ^ v_swz<D>(r8)));

  const_i32* bt_s = (const_i32*)bt;
  const_f32* ks_s = (const_f32*)p.k_scale;
  const_f32* vs_s = (const_f32*)p.v_scale;
  // whether some of `n` keys from `key` on are cached keys that a row may see
  auto wanted = [&](int key, int n) { return key < lp && key + n > wg_lo; };
  // physical page of this wave's rows of a tile whose first key is j0 (0: no such key)
  auto load_page = [&](int j0) -> int { return wanted(j0 + wrow0, 8) ? bt_s[(j0 + wrow0) >> pshift] : 0; };

  // DMA of the tile whose first key is j0 into dst: prefix rows from pool page pg (16-bit pools
  // only), new rows from `fresh`; rows before wg_lo or at or past new_stop are left as they are.
  auto issue = [&](int j0, uint8_t* dst, int pg, bool keys) __attribute__((always_inline)) {
    const uint32_t off = keys ? k_off : v_off;
    const int k_first = j0 + wrow0, k_last = k_first + 7;
    if (!FP8 && wanted(k_first, 8)) {
      const auto rs = rsrc_at((keys ? k_pool : v_pool) + size_t(pg) * page_stride);
#pragma unroll
      for (int i = 0; i < T::NI; ++i) {
        const int key = k_first + T::RPI * i + dma_row;
        if (key < lp && key >= wg_lo) fetch(rs, dst, off, 0, i, page_row, T::RB, keys);
      }
    }
    if (k_last >= lp && k_first < new_stop) {
      // base of the tile's first key as if it were a new token (it may lie before the
      // buffer; only rows at or past the prefix end are fetched from it)
      const ptrdiff_t row0 = ptrdiff_t(sq.cu) + j0 - lp;
      const auto rs = rsrc_at((keys ? k_new : v_new) + (row0 * hkv + kvh) * T::RB);
#pragma unroll
      for (int i = 0; i < T::NI; ++i) {
        const int key = k_first + T::RPI * i + dma_row;
        if (key >= lp && key >= wg_lo && key < new_stop) fetch(rs, dst, off, new_off, i, new_row, hkv * T::RB, keys);
      }
    }
  };
  // fp8 pool rows into registers, values with their page's scale (`in_prefix`: the tile lies
  // wholly among cached keys from wg_lo on, so every row check passes)
  auto load8 = [&](int j0, int pg, const uint8_t* pool, uint32_t off, u32x4& rw, bool in_prefix,
                   bool keys) __attribute__((always_inline)) {
    if (!in_prefix && !wanted(j0 + wrow0, 8)) return;
    const auto rs = rsrc_at(pool + size_t(pg) * page_stride);
    const u32x2 a = __builtin_amdgcn_raw_buffer_load_b64(rs, off, 0, 0);
    if constexpr (T::B8 == 16) {
      const u32x2 b = __builtin_amdgcn_raw_buffer_load_b64(rs, (keys ? off ^ 64u : off) + 4 * D, 0, 0);
      rw = u32x4{a.x, a.y, b.x, b.y};
    } else {
      rw = u32x4{a.x, a.y, 0u, 0u};
    }
  };
  // `keys`: the codes are stored as they are
  auto store8 = [&](int j0, const u32x4& rw, float s, uint8_t* dst, bool in_prefix, bool keys) __attribute__((always_inline)) {
    if (!in_prefix && !wanted(j0 + wrow0, 8)) return;
    const PageScale sc = page_scale(s);
    auto widen = [&](uint32_t a, uint32_t b) { return keys ? fp8x8_f16x8(a, b) : fp8x8_f16x8(a, b, sc); };
    auto ok = [&](int key) { return in_prefix || (key < lp && key >= wg_lo); };
    if (ok(j0 + r8)) *reinterpret_cast<u32x4*>(dst + wrow0 * T::RB + 16 * lane) = widen(rw.x, rw.y);
    if constexpr (T::B8 == 16) {
      if (ok(j0 + r8 + 4)) *reinterpret_cast<u32x4*>(dst + (wrow0 + 4) * T::RB + 16 * lane) = widen(rw.z, rw.w);
    }
  };
  // fp8 pools: the new tokens' rows that this wave staged by DMA become fp16 in place
  // (before the barrier that publishes the tile)
  auto convert_new = [&](int j0, uint8_t* dst) __attribute__((always_inline)) {
    const int k_first = j0 + wrow0, k_last = k_first + 7;
    if (k_last < lp || k_first >= new_stop) return;
#pragma unroll
    for (int i = 0; i < T::NI; ++i) {
      const int key = k_first + T::RPI * i + dma_row;
      if (key >= lp && key >= wg_lo && key < new_stop) {
        u32x4* ptr = reinterpret_cast<u32x4*>(dst + (wrow0 + T::RPI * i) * T::RB + 16 * lane);
        *ptr = bf16x8_f16x8(*ptr);
      }
    }
  };

  // fp8 pools.  In the loops pages and their scales come by vector loads, which have landed with the
  // staging before them at the next iteration's barrier (by scalar loads the first LDS read of
  // each iteration waited for them: 4096 tokens on 32768 keys at D = 64 3620 us, so 3340).  Each of a
  // tile's groups of 16 keys lies in one page.  Iteration j takes, lane l, the page of group l % 4 of
  // tile j + 4 (l < 4, whose rows are loaded next) or j + 3 (scales next), and the key (l < 8) or value
  // scale of group l % 4 of tile j + 2.  Behind the prefix or before what is visible: no page, scale 1.
  const int own = wave >> 1;  // the group of this wave's rows
  auto pages_of = [&](int j0) __attribute__((always_inline)) -> int {
    const int key = j0 + (lane < 4 ? 0 : BLOCK_N) + 16 * (lane & 3);
    return wanted(key, 16) ? bt[key >> pshift] : 0;
  };
  auto scales_of = [&](int j0, int pg) __attribute__((always_inline)) -> float {
    if (lane < 4 || !wanted(j0 + 16 * (lane & 3), 16)) return 1.f;
    return (lane < 8 ? p.k_scale : p.v_scale)[size_t(pg) * hkv + kvh];
  };
  auto lane_of = [&](float v, int l) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), l)); };

  // ---- LDS fragment addresses (relative to a stage), as in the extend kernel: that of k-step kk
  // is k_addr ^ 32 kk, that of O^T block b is v_addr ^ 64 b (the swizzles are exclusive ors)
  uint32_t k_addr, v_addr;
  {
    const int R = swap_bits_2_3(col);
    k_addr = R * T::RB + 16 * (h ^ k_swz<D>(R));
    const int grp = lane >> 4, ri = lane & 15;
    const int kq = ri >> 2, a = ri & 3;
    v_addr = (8 * h + kq) * T::RB + 16 * ((2 * (grp & 1) + (a >> 1)) ^ v_swz<D>(kq)) + 8 * (a & 1);
  }
  // At D = 128 they are formed where they are used, which leaves eleven registers more.
  auto here = [&](uint32_t& addr) __attribute__((always_inline)) {
    if constexpr (D == 128) asm volatile("" : "+v"(addr));
  };

  f32x16 o[T::DB];
#pragma unroll
  for (int b = 0; b < T::DB; ++b) o[b] = f32x16{};
  // a row that sees no key of this item keeps m = kNegBig and l = 0: weight 0 in a merge
  float m_run = kNegBig, l_run = 0.f;
  const float c = sp.score_factor, cap2 = sp.cap2;
  auto tile0 = [&](int j) { return kv_begin + (n_tiles - 1 - j) * BLOCK_N; };  // the last tile first

  // The products of a phase: 2 KT steps each, the LDS reads of a step `kEarly` steps before it.
  // Scores: step i adds k-step i / 2 to s[i % 2], the lower or upper 32 keys of key tile kt.
  // Values: step i adds 16 keys of value tile vt to O^T block i % DB.
  constexpr int kSteps = 2 * T::KT, kEarly = 3;
  static_assert(kSteps == 4 * T::DB, "as many products of scores as of values");
  auto read_key = [&](const uint8_t* kt, int i, u32x4(&kf)[kSteps]) __attribute__((always_inline)) {
    kf[i] = *reinterpret_cast<const u32x4*>(kt + (k_addr ^ (32 * (i / 2))) + (i % 2) * 32 * T::RB);
  };
  auto read_value = [&](const uint8_t* vt, int i, u32x4(&vf)[kSteps]) __attribute__((always_inline)) {
    const int u = i / T::DB, b = i % T::DB;
    i16x4 part[2];
#pragma unroll
    for (int e4 = 0; e4 < 2; ++e4)
      part[e4] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(vt + (v_addr ^ (64 * b)) + (16 * u + 4 * e4) * T::RB));
    vf[i] = __builtin_bit_cast(u32x4, __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7));
  };
  // What a block's scores are multiplied with: c, over fp8 pools times the scale of their page (of
  // the keys of element group i / 8, which share one).
  struct Scales {
    float g[2];
  };
  // ... of the block of keys from k0 on, with scores s and page scales ks0, ks1.  Where the
  // prefix ends among the 16 keys of a group, they are scaled in s.
  auto block_scales = [&](float ks0, float ks1, int k0, Keys keys, f32x16& s) __attribute__((always_inline)) -> Scales {
    Scales r{{c, c}};
    if constexpr (FP8) {
      if (keys == Keys::kAny && k0 >= lp) return r;
#pragma unroll
      for (int gi = 0; gi < 2; ++gi) {
        const float f = gi == 0 ? ks0 : ks1;
        const int cached = lp - (k0 + 16 * gi);  // of these keys, where that is below 16
        r.g[gi] = keys == Keys::kSeen || cached >= 16 ? c * f : c;  // (a new key's f is 1)
        if (keys == Keys::kAny && cached > 0 && cached < 16) {
#pragma unroll
          for (int e = 0; e < 8; ++e) s[8 * gi + e] *= 8 * h + e < cached ? f : 1.f;
        }
      }
    }
    return r;
  };
  // The weights of a block of 32 keys from k0 on, with scores x: 16 elements, element i holding key
  // k0 + 16 (i / 8) + 8 h + i % 8.  Formed in units of kUnit elements, one beside each product, a
  // unit's operations spread over kDepth of them so that none waits for the one before:
  // unit(t) starts elements t and ends elements t - kDepth + 1.  Not masked: every row sees all
  // keys, none of them behind its own position if there is a bias.
  constexpr int kUnit = 16 / kSteps, kDepth = CAP ? 4 : 2, kLead = kDepth - 1;
  struct Block {
    float a[16], w[16];  // in a cap's way; weights
    float base, la, lb;
    int at, away;
  };
  auto start = [&](Block& bk, int k0, bool masked, float m) __attribute__((always_inline)) {
    bk.base = BIAS && !masked ? fmaf(slope2, static_cast<float>(k0 + 8 * h - pos), -m) : -m;
    bk.at = k0 + 8 * h - lo;
    bk.away = k0 + 8 * h - pos;
    bk.la = bk.lb = 0.f;
  };
  auto exponent_of = [&](Block& bk, const f32x16& x, const Scales& sc, bool masked, float m, int i) __attribute__((always_inline)) -> float {
    const int n = 16 * (i >> 3) + (i & 7);
    float bias = bk.base;
    if (BIAS && !masked) bias = fmaf(slope2, static_cast<float>(n), bk.base);
    if (BIAS && masked) bias = fmaf(-slope2, fabsf(static_cast<float>(bk.away + n)), -m);
    float f;
    if constexpr (CAP) f = fmaf(bk.a[i], -2.f * cap2, cap2 + bias);  // (a: 1 / (1 + 2^(s c)))
    else f = fmaf(x[i], FP8 ? sc.g[i >> 3] : c, bias);
    if (masked && static_cast<uint32_t>(bk.at + n) >= seen) f = -INFINITY;
    return f;
  };
  // Weights i - 1 and i (odd) in the operand type, and in the block's sums.
  auto round_pair = [&](Block& bk, u32x4(&pf)[2], int i) __attribute__((always_inline)) {
    float& l = i % 4 == 1 ? bk.la : bk.lb;
    uint32_t two;
    if constexpr (FP8) {
      const f16x2 v = {static_cast<_Float16>(bk.w[i - 1]), static_cast<_Float16>(bk.w[i])};
      l = __builtin_amdgcn_fdot2(v, f16x2{static_cast<_Float16>(1.f), static_cast<_Float16>(1.f)}, l, false);
      two = as_u32(v);
    } else {
      const bf16x2 v = {static_cast<__bf16>(bk.w[i - 1]), static_cast<__bf16>(bk.w[i])};
      l = __builtin_amdgcn_fdot2_f32_bf16(v, __builtin_bit_cast(bf16x2, 0x3F803F80u), l, false);
      two = __builtin_bit_cast(uint32_t, v);
    }
    pf[i >> 3][(i & 7) >> 1] = two;
  };
  auto unit = [&](Block& bk, const f32x16& x, const Scales& sc, bool masked, u32x4(&pf)[2], int t) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < kUnit; ++e) {
      if constexpr (CAP) {
        const int i = t * kUnit + e, i1 = i - kUnit;
        if (i >= 0 && i < 16) bk.a[i] = __builtin_amdgcn_exp2f(x[i] * (FP8 ? sc.g[i >> 3] : c));
        if (i1 >= 0 && i1 < 16) bk.a[i1] = __builtin_amdgcn_rcpf(1.f + bk.a[i1]);
      }
      const int i2 = (t - kDepth + 2) * kUnit + e, i3 = i2 - kUnit;
      if (i2 >= 0 && i2 < 16) bk.w[i2] = __builtin_amdgcn_exp2f(exponent_of(bk, x, sc, masked, m_run, i2));
      if (i3 >= 0 && i3 < 16 && i3 % 2 == 1) round_pair(bk, pf, i3);
    }
  };
  // Weights of a block, against the running max raised as far as they call for (RunningMax); `other`: weights
  // of another block that O does not hold yet.
  auto raise = [&](const f32x16& x, const Scales& sc, int k0, bool masked, u32x4(&pf)[2], float& lsum,
                   u32x4* other) __attribute__((always_inline)) {
    Block bk;
    float f[16];
    auto exponents = [&](float m) __attribute__((always_inline)) {
      start(bk, k0, masked, m);
#pragma unroll
      for (int i = 0; i < 16; ++i) f[i] = exponent_of(bk, x, sc, masked, m, i);
    };
    auto form = [&](bool settled, const RunningMax& rm) __attribute__((always_inline)) {
      bk.la = bk.lb = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        bk.w[i] = __builtin_amdgcn_exp2f(settled ? rm.exponent(f[i]) : f[i]);
        if (i % 2 == 1) round_pair(bk, pf, i);
      }
      lsum = bk.la + bk.lb;
    };
    auto largest = [&]() __attribute__((always_inline)) -> float {
      float mx = f[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) mx = fmaxf(mx, f[i]);
      return floorf(row_max(mx));
    };
    if constexpr (CAP) {
#pragma unroll
      for (int i = 0; i < 16; ++i) bk.a[i] = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x[i] * (FP8 ? sc.g[i >> 3] : c)));
    }
    exponents(0.f);
    RunningMax rm(m_run, largest());
    exponents(rm.near);
    form(false, rm);
    // (a row whose max rises has a weight of 2^kHeadroom, if its exponents came out as they did against 0)
    const bool off = !(lsum <= kSumLimit) || (rm.near > m_run && row_sum(lsum) < 64.f);
    if (__builtin_expect(__any(off), 0)) {
      rm.settle(m_run, largest());
      form(true, rm);
    }
    const float alpha = rm.raise(m_run);
    l_run *= alpha;
#pragma unroll
    for (int b = 0; b < T::DB; ++b) o[b] *= alpha;
    if (other != nullptr) {
#pragma unroll
      for (int gi = 0; gi < 2; ++gi) {
        if constexpr (FP8) {
          f16x8 w = __builtin_bit_cast(f16x8, other[gi]);
#pragma unroll
          for (int e = 0; e < 8; ++e) w[e] = static_cast<_Float16>(static_cast<float>(w[e]) * alpha);
          other[gi] = __builtin_bit_cast(u32x4, w);
        } else {
          bf16x8 w = __builtin_bit_cast(bf16x8, other[gi]);
#pragma unroll
          for (int e = 0; e < 8; ++e) w[e] = static_cast<__bf16>(static_cast<float>(w[e]) * alpha);
          other[gi] = __builtin_bit_cast(u32x4, w);
        }
      }
    }
  };
  // ---- state across iterations (of one parity, for the next of the other): the lower block's
  // scores of the tile in hand with their scales, its upper block's weights
  f32x16 x_low[2] = {};
  u32x4 p_up[2][2] = {};
  Scales sc_low{{c, c}};
  // The phases of iteration j: key tile kt (keys from tile0(j + 1) on), value tile vt.  `last`:
  // there is no next tile, and what is taken of it counts for nothing.
  auto phases = [&](const uint8_t* kt, const uint8_t* vt, int j, auto parity, auto where, bool last, const float (&ks)[T::KS])
      __attribute__((always_inline)) {
    constexpr Keys keys = decltype(where)::value;
    constexpr bool masked = keys == Keys::kAny;
    constexpr int in = decltype(parity)::value, out = 1 - in;
    const int k_low = tile0(j), k_next = tile0(j + 1);
    const f32x16& x = x_low[in];
    f32x16 &s_low = x_low[out], s_up;
    u32x4 kf[kSteps], vf[kSteps], p_low[2];
    Block bk;
    here(k_addr);
    here(v_addr);
#pragma unroll
    for (int i = 0; i < kEarly; ++i) read_key(kt, i, kf);
    start(bk, k_low, masked, m_run);
#pragma unroll
    for (int t = 0; t < kLead; ++t) unit(bk, x, sc_low, masked, p_low, t);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      if (i + kEarly < kSteps) read_key(kt, i + kEarly, kf);
      else read_value(vt, i + kEarly - kSteps, vf);
      f32x16& s = i % 2 == 0 ? s_low : s_up;
      s = mfma16<FP8>(kf[i], qf[i / 2], i > 1 ? s : f32x16{});
      unit(bk, x, sc_low, masked, p_low, kLead + i);
      __builtin_amdgcn_sched_barrier(0);
    }
    float lsum = bk.la + bk.lb;
    if (__builtin_expect(__any(!(lsum <= kSumLimit)), 0)) raise(x, sc_low, k_low, masked, p_low, lsum, p_up[in]);
    l_run += lsum;
    const Scales sc_up = block_scales(ks[2], ks[3], k_next + 32, keys, s_up);
    const int k_up = last ? -BLOCK_N : k_next + 32;  // (no row sees a key before the first)
    start(bk, k_up, masked, m_run);
#pragma unroll
    for (int t = 0; t < kLead; ++t) unit(bk, s_up, sc_up, masked, p_up[out], t);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      if (i + kEarly < kSteps) read_value(vt, i + kEarly, vf);
      const int u = i / T::DB;
      o[i % T::DB] = mfma16<FP8>(vf[i], u < 2 ? p_low[u] : p_up[in][u - 2], o[i % T::DB]);
      unit(bk, s_up, sc_up, masked, p_up[out], kLead + i);
      __builtin_amdgcn_sched_barrier(0);
    }
    lsum = bk.la + bk.lb;
    if (__builtin_expect(__any(!(lsum <= kSumLimit)), 0)) raise(s_up, sc_up, k_up, masked, p_up[out], lsum, nullptr);
    l_run += lsum;
    sc_low = block_scales(ks[0], ks[1], k_next, keys, s_low);
  };

  // ---- prologue: the first tile's scores, its upper block's weights against their exact max
  u32x4 k8{}, v8{};
  int pg_k = 0, pg_v = 0;  // pages of the tiles to be issued (fp8: loaded) next
  int pg_next = 0;         // page of the key tile after that (fp8: pages, of a lane each), on its way
  float sc_next = 1.f;     // fp8: scales on their way
  // At an iteration's start, what the one before has loaded: ks of the key tile, vs of the value rows to be
  // stored.
  auto arrive = [&](float (&ks)[T::KS], float& vs) __attribute__((always_inline)) {
    pg_v = pg_k;
    pg_k = FP8 ? __builtin_amdgcn_readlane(pg_next, own) : pg_next;
    if constexpr (FP8) {
#pragma unroll
      for (int gi = 0; gi < T::KS; ++gi) ks[gi] = lane_of(sc_next, 4 + gi);
      vs = lane_of(sc_next, 8 + own);
    }
  };
  // ... and what iteration j loads for the next ones.
  auto depart = [&](int j) __attribute__((always_inline)) {
    if constexpr (FP8) {
      sc_next = scales_of(tile0(j + 2), pg_next);
      pg_next = pages_of(tile0(j + 4));
    } else {
      pg_next = load_page(tile0(j + 3));
    }
  };
  if (n_tiles > 0) {
    const int b0 = tile0(0);
    const int pk0 = load_page(b0), pk1 = load_page(tile0(1));
    issue(b0, lds_k0, pk0, true);
    issue(b0, lds_v0, pk0, false);
    if (n_tiles > 1) issue(tile0(1), lds_k1, pk1, true);
    pg_k = pk1;
    pg_next = FP8 ? pages_of(tile0(2)) : load_page(tile0(2));
    if constexpr (FP8) {
      u32x4 ka{}, kb{}, va{};
      load8(b0, pk0, k_pool, k8_off, ka, false, true);
      load8(b0, pk0, v_pool, v8_off, va, false, false);
      load8(tile0(1), pk1, k_pool, k8_off, kb, false, true);
      const float vs0 = wanted(b0 + wrow0, 8) ? vs_s[size_t(pk0) * hkv + kvh] : 1.f;
      __builtin_amdgcn_s_waitcnt(0);
      store8(b0, ka, 1.f, lds_k0, false, true);
      store8(b0, va, vs0, lds_v0, false, false);
      store8(tile0(1), kb, 1.f, lds_k1, false, true);
      convert_new(b0, lds_k0);
      pg_k = __builtin_amdgcn_readlane(pg_next, own);
      load8(tile0(2), pg_k, k_pool, k8_off, k8, false, true);
      load8(tile0(1), pk1, v_pool, v8_off, v8, false, false);
      sc_next = scales_of(tile0(1), pg_next);
      pg_next = pages_of(tile0(3));
    }
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (wave_active) {
      float ks[T::KS], lsum;
#pragma unroll
      for (int gi = 0; gi < T::KS; ++gi) {
        const int key = b0 + 16 * gi;
        ks[gi] = FP8 && wanted(key, 16) ? ks_s[size_t(bt_s[key >> pshift]) * hkv + kvh] : 1.f;
      }
      f32x16 s[2];
      u32x4 kf[kSteps];
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        read_key(lds_k0, i, kf);
        s[i % 2] = mfma16<FP8>(kf[i], qf[i / 2], i > 1 ? s[i % 2] : f32x16{});
      }
      const Scales sc_up = block_scales(ks[2], ks[3], b0 + 32, Keys::kAny, s[1]);
      raise(s[1], sc_up, b0 + 32, true, p_up[0], lsum, nullptr);
      l_run = lsum;
      sc_low = block_scales(ks[0], ks[1], b0, Keys::kAny, s[0]);
      x_low[0] = s[0];
    }
    __syncthreads();  // (iteration 0 stages tile 2's keys where tile 0's were)
  }

  // iteration j: key tile j + 1 and value tile j are resident; the tiles after them go to the
  // other stages.  fp8 pool rows were loaded to registers an iteration ago.
  // Waves without rows (`rows` false) only stage: they run the same loops, without the phases.
  auto iteration = [&](auto rows, auto parity, int j, uint8_t* k_cur, uint8_t* k_nxt, uint8_t* v_cur,
                       uint8_t* v_nxt) __attribute__((always_inline)) {
    __builtin_amdgcn_s_waitcnt(0);  // this wave's staging has landed
    if constexpr (FP8) {
      if (j + 1 < n_tiles) convert_new(tile0(j + 1), k_cur);
      convert_new(tile0(j), v_cur);
    }
    __syncthreads();  // everyone's has; the other stages are no longer read
    float ks[T::KS] = {}, vs = 1.f;
    arrive(ks, vs);
    if (j + 1 < n_tiles) {
      if constexpr (FP8) {
        if (j + 2 < n_tiles) store8(tile0(j + 2), k8, 1.f, k_nxt, false, true);
        store8(tile0(j + 1), v8, vs, v_nxt, false, false);
      }
      if (j + 2 < n_tiles) issue(tile0(j + 2), k_nxt, pg_k, true);
      issue(tile0(j + 1), v_nxt, pg_v, false);
      if constexpr (FP8) {
        load8(tile0(j + 3), pg_k, k_pool, k8_off, k8, false, true);
        load8(tile0(j + 2), pg_v, v_pool, v8_off, v8, false, false);
      }
      depart(j);
    }
    // (also of tiles that no row of this wave sees: a branch around the phases made the compiler
    // copy O in every iteration)
    if constexpr (decltype(rows)::value) phases(k_cur, v_cur, j, parity, std::integral_constant<Keys, Keys::kAny>{}, j + 1 >= n_tiles, ks);
  };
  // Iterations whose staged tiles lie wholly in the cached prefix (fp8: whose loaded tiles do
  // too), or wholly among the new tokens (`fresh`), and whose keys every row sees: a wave's rows come
  // from one page or follow each other, so they carry no row checks and no mask.  (One loop for both:
  // of two loops the compiler gave one too few registers.)
  auto fast = [&](auto rows, auto parity, int j, bool fresh, uint8_t* k_cur, uint8_t* k_nxt, uint8_t* v_cur,
                  uint8_t* v_nxt) __attribute__((always_inline)) {
    __builtin_amdgcn_s_waitcnt(0);
    if (FP8 && fresh) {
      convert_new(tile0(j + 1), k_cur);
      convert_new(tile0(j), v_cur);
    }
    __syncthreads();
    float ks[T::KS] = {}, vs = 1.f;
    arrive(ks, vs);
    if (!FP8 || fresh) {
      auto base = [&](int j0, int pg, const uint8_t* pool, const uint8_t* rows_new) {
        const ptrdiff_t row0 = ptrdiff_t(sq.cu) + j0 - lp;
        return fresh ? rows_new + (row0 * hkv + kvh) * T::RB : pool + size_t(pg) * page_stride;
      };
      const auto rk = rsrc_at(base(tile0(j + 2), pg_k, k_pool, k_new)), rv = rsrc_at(base(tile0(j + 1), pg_v, v_pool, v_new));
      const uint32_t more = fresh ? new_off : 0, first = fresh ? new_row : page_row, row = (fresh ? hkv : 1) * T::RB;
#pragma unroll
      for (int i = 0; i < T::NI; ++i) fetch(rk, k_nxt, k_off, more, i, first, row, true);
#pragma unroll
      for (int i = 0; i < T::NI; ++i) fetch(rv, v_nxt, v_off, more, i, first, row, false);
    }
    if constexpr (FP8) {
      if (!fresh) {
        store8(tile0(j + 2), k8, 1.f, k_nxt, true, true);
        store8(tile0(j + 1), v8, vs, v_nxt, true, false);
      }
      load8(tile0(j + 3), pg_k, k_pool, k8_off, k8, !fresh, true);
      load8(tile0(j + 2), pg_v, v_pool, v8_off, v8, !fresh, false);
    }
    depart(j);
    if constexpr (decltype(rows)::value) phases(k_cur, v_cur, j, parity, std::integral_constant<Keys, Keys::kSeen>{}, false, ks);
  };
  // The ranges [begin, end) of iterations that may run so, new tokens and prefix.  Both: the keys of this
  // tile and the next visible to every row, and no tile that they stage (fp8: load) with a key before
  // wg_lo, as the item's last one may have.  Prefix: this tile in the prefix.  New:
  // the staged keys among the new tokens, and with a bias, which falls with the distance on both
  // sides of a token, no key behind a token.
  const int top = tile0(0);
  auto tiles_down_to = [&](int key) { return (top - key) >> 6; };  // the last j with tile0(j) >= key (floor)
  const int seen_end = tiles_down_to(wg_lo_max), staged = n_tiles - (kv_begin < wg_lo ? 1 : 0);
  const int steady_begin = (top + BLOCK_N - lp + BLOCK_N - 1) >> 6, steady_end = min(seen_end, staged - (FP8 ? 3 : 2));
  const int limit = min(BIAS ? first_lim : min_lim, total_len);
  const int new_begin = (top + BLOCK_N - limit + BLOCK_N - 1) >> 6;
  const int new_end = min(min(seen_end, staged - 2), tiles_down_to(lp) - 1);
  auto walk = [&](auto rows) __attribute__((always_inline)) {
    constexpr std::integral_constant<int, 0> even{};
    constexpr std::integral_constant<int, 1> odd{};
    int j = 0;
    // (every loop takes two iterations at a time, so that an iteration's stages are fixed)
#pragma unroll 1
    for (int phase = 0; phase < 3; ++phase) {
      const int from = (max(j, phase == 0 ? new_begin : steady_begin) + 1) & ~1;
      const int end = phase == 0 ? new_end : steady_end;
      const bool many = phase < 2 && from + 1 < end;
      const int to = phase == 2 ? n_tiles : many ? from : 0;
#pragma unroll 1
      for (; j < to; j += 2) {
        iteration(rows, even, j, lds_k1, lds_k0, lds_v0, lds_v1);
        if (j + 1 < n_tiles) iteration(rows, odd, j + 1, lds_k0, lds_k1, lds_v1, lds_v0);
      }
      if (!many) continue;
#pragma unroll 1
      for (; j + 1 < end; j += 2) {
        fast(rows, even, j, phase == 0, lds_k1, lds_k0, lds_v0, lds_v1);
        fast(rows, odd, j + 1, phase == 0, lds_k0, lds_k1, lds_v1, lds_v0);
      }
    }
  };
  if (!wave_active) {  // (as many barriers as the others)
    walk(std::false_type{});
    return;
  }
  walk(std::true_type{});

  const float l_tot = row_sum(l_run);
  if (!row_ok) return;
  if (it.part >= 0) {  // unnormalised partial, merged by the combine kernels
    const size_t slot = size_t(it.part) * p.part_rows + r_local;
#pragma unroll
    for (int b = 0; b < T::DB; ++b)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4)
        part::put4(p, slot * D + 32 * b + 8 * q4 + 4 * h,
                   part::f32x4{o[b][4 * q4], o[b][4 * q4 + 1], o[b][4 * q4 + 2], o[b][4 * q4 + 3]});
    if (h == 0) *reinterpret_cast<f32x2*>(p.part_ml + slot * 2) = f32x2{m_run, l_tot};
    return;
  }
  const float inv = l_tot == 0.f ? 0.f : 1.f / l_tot;  // (a row that sees nothing: 0)
  uint16_t* orow = static_cast<uint16_t*>(p.out) + out_row * D;
#pragma unroll
  for (int b = 0; b < T::DB; ++b)
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) {
      bf16x4 v4;
#pragma unroll
      for (int e = 0; e < 4; ++e) v4[e] = static_cast<__bf16>(o[b][4 * q4 + e] * inv);
      *reinterpret_cast<u32x2*>(orow + 32 * b + 8 * q4 + 4 * h) = __builtin_bit_cast(u32x2, v4);
    }
  if (p.lse != nullptr && h == 0) p.lse[out_row] = (m_run + __log2f(l_tot)) * kLn2;
}

template <int D, bool FP8, bool CAP, bool BIAS>
hipError_t launch_extend_t(const ShapedParams& p, hipStream_t stream, const ArgPlanBuf* ap) {
  const dim3 grid(p.a.n_items), block(kThreads);
  if (ap != nullptr && ap->small())
    hipLaunchKernelGGL((shaped_extend_kernel<D, FP8, CAP, BIAS, kPlanInSmallArgs>), grid, block, 0, stream, p, ap->small_plan());
  else if (ap != nullptr)
    hipLaunchKernelGGL((shaped_extend_kernel<D, FP8, CAP, BIAS, kPlanInArgs>), grid, block, 0, stream, p, ap->plan);
  else
    hipLaunchKernelGGL((shaped_extend_kernel<D, FP8, CAP, BIAS, kPlanInMemory>), grid, block, 0, stream, p, NoArgPlan{});
  return hipGetLastError();
}

template <int D>
hipError_t launch_extend_d(const ShapedParams& p, bool fp8, hipStream_t stream, const ArgPlanBuf* ap) {
  if (p.a.n_items <= 0) return hipSuccess;
  const bool cap = p.cap2 > 0.f, bias = p.slopes != nullptr;
  if (fp8) {
    if (cap) return bias ? launch_extend_t<D, true, true, true>(p, stream, ap) : launch_extend_t<D, true, true, false>(p, stream, ap);
    return bias ? launch_extend_t<D, true, false, true>(p, stream, ap) : launch_extend_t<D, true, false, false>(p, stream, ap);
  }
  if (cap) return bias ? launch_extend_t<D, false, true, true>(p, stream, ap) : launch_extend_t<D, false, true, false>(p, stream, ap);
  return bias ? launch_extend_t<D, false, false, true>(p, stream, ap) : launch_extend_t<D, false, false, false>(p, stream, ap);
}

}  // namespace shaped
}  // namespace cw
