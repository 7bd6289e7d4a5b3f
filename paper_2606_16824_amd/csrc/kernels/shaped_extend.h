// Attention with shaped scores for chunks of new tokens over a paged cache (the kernel; its
// instances are compiled by shaped_extend_d64.hip and shaped_extend_d128.hip).
//
// A workgroup of eight waves owns 256 packed query rows (token x query head of one kv head, 32
// per wave) and walks the keys that some row may see, 64 at a time.  S^T = K Q^T and O^T += V^T
// P^T with v_mfma_f32_32x32x16 (bf16; fp16 over fp8 pools), so that a lane owns a query row: its
// slope, position and limits are one register each.  Scores run 32 keys ahead of the values:
// while a block's weights are formed, the scores of the next 32 keys are on the matrix cores.
// Key tiles therefore cover the 64 keys from 32 behind the value tile's start; both rotate
// through two LDS stages with one barrier per 64 keys.
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
#pragma once

#include <hip/hip_runtime.h>

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
// What the compiler may move across the point between a fragment's read and a product: vector,
// scalar and transcendental operations (the weights' exponentials run beside the products).
constexpr int kMayCross = 0x2 | 0x4 | 0x400;
constexpr int kAhead = 32;  // keys by which key tiles lie behind value tiles

// Where a block of keys lies whose scores are taken: in the cached prefix, among the new
// tokens, or anywhere.
enum class Keys { kPrefix, kNew, kAny };

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc_at(const void* base) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, -1, 0x00020000);
}

// 16 bytes per lane from base + voff straight into LDS (lane l's bytes land at dst + 16 l).
// Not a template: see the extend kernel.
__device__ __forceinline__ void dma16(__amdgpu_buffer_rsrc_t r, lds_void* dst, uint32_t voff) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, dst, 16, voff, 0, 0, 0);
}

// Page scale s = p2 x fm, p2 a power of two (applied exactly by the conversion), fm in
// [1, 2) rounded to fp16.
struct PageScale {
  float p2;
  f16x2 fm;
};
__device__ __forceinline__ PageScale page_scale(float s) {
  const uint32_t b = __float_as_uint(s);
  const float p2 = __uint_as_float(b & 0x7F800000u);
  const _Float16 m = static_cast<_Float16>(__uint_as_float((b & 0x807FFFFFu) | 0x3F800000u));
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
  static constexpr int K_AHEAD = D == 64 ? 0 : FP8 ? 1 : 2, V_AHEAD = D == 64 ? 0 : 2;  // fragments read ahead
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
  // over the wave's rows and over the workgroup's: the limits (causal, so monotonic) ...
  const int wave_last_row = it.q_row0 + min(wave * 32 + 31, it.rows - 1);
  const int wave_max_lim = max(lp + wave_last_row / G + 1, full);
  const int first_lim = lp + it.q_row0 / G + 1;  // of the workgroup's first row, without the prefix mask
  const int min_lim = max(first_lim, full);
  // ... and the first keys
  auto window_lo = [&](int at) { return sp.window > 0 ? max(0, at - sp.window + 1) : 0; };
  int lo = window_lo(pos);
  int wave_lo = window_lo(lp + (it.q_row0 + wave * 32) / G);  // smallest of the wave
  int wg_lo = window_lo(first_lim - 1), wg_lo_max = window_lo(lp + (it.q_row0 + it.rows - 1) / G);
  if (sp.begins != nullptr) {
    if (row_ok) lo = max(lo, sp.begins[sq.cu + t]);
    int mn = row_ok ? lo : 0x7FFFFFFF, mx = row_ok ? lo : 0;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      mn = min(mn, __shfl_xor(mn, d));
      mx = max(mx, __shfl_xor(mx, d));
    }
    wave_lo = __builtin_amdgcn_readfirstlane(mn);
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

  // ---- staging.  Wave w stages rows [8 w, 8 w + 8) of a tile.  Row R of the key tile of
  // iteration j is key tile0(j) + kAhead + R, of the value tile key tile0(j) + R; eight
  // rows lie in one page.  16-bit rows: DMA instruction i covers rows 8 w + RPI i on, lane
  // l fetches the chunk that belongs at position l % CPR of row l / CPR of them.
  const int dma_row = lane / T::CPR, dma_pos = lane % T::CPR;
  const int wrow0 = 8 * wave;
  uint32_t k_off[T::NI], v_off[T::NI];    // within a page block
  uint32_t kn_off[T::NI], vn_off[T::NI];  // from the tile's first key among the new tokens
#pragma unroll
  for (int i = 0; i < T::NI; ++i) {
    const int R = wrow0 + T::RPI * i + dma_row;
    const uint32_t kc = 16 * (dma_pos ^ k_swz<D>(R)), vc = 16 * (dma_pos ^ v_swz<D>(R));
    k_off[i] = ((R + kAhead) & (P - 1)) * T::RB + kc;
    v_off[i] = (R & (P - 1)) * T::RB + vc;
    kn_off[i] = R * hkv * T::RB + kc;
    vn_off[i] = R * hkv * T::RB + vc;
  }
  const uint32_t page_bytes = uint32_t(P) * T::PRB;  // one (page, head) block
  const size_t page_stride = size_t(hkv) * page_bytes;
  const uint8_t* k_pool = static_cast<const uint8_t*>(p.k_pool) + size_t(kvh) * page_bytes;
  const uint8_t* v_pool = static_cast<const uint8_t*>(p.v_pool) + size_t(kvh) * page_bytes;
  // fp8 rows.  D = 64: lane l stages 8 bytes of row 8 w + l / 8.  D = 128: load u of lane
  // l fetches what belongs at position l % 16 of row 8 w + 4 u + l / 16 (four rows on, a key's
  // swizzle differs in the bit of 8, a value's not at all).
  const int r8 = D == 128 ? wrow0 + (lane >> 4) : wrow0 + (lane >> 3);
  const int pos8 = D == 128 ? lane & 15 : lane & 7;
  const uint32_t k8_off = uint32_t(((r8 + kAhead) & (P - 1)) * D + 8 * (pos8 ^ k_swz<D>(r8)));
  const uint32_t v8_off = uint32_t((r8 & (P - 1)) * D + 8 * (pos8 ^ v_swz<D>(r8)));

  const_i32* bt_s = (const_i32*)bt;
  const_f32* ks_s = (const_f32*)p.k_scale;
  const_f32* vs_s = (const_f32*)p.v_scale;
  // whether some of `n` keys from `key` on are cached keys that a row may see
  auto wanted = [&](int key, int n) { return key < lp && key + n > wg_lo; };
  // physical page of this wave's rows of a tile whose first key is j0 (0: no such key)
  auto load_page = [&](int j0) -> int { return wanted(j0 + wrow0, 8) ? bt_s[(j0 + wrow0) >> pshift] : 0; };

  // DMA of the tile whose first key is j0 into dst: prefix rows from pool page pg (16-bit pools
  // only), new rows from `fresh`; rows before `from`, before wg_lo or past the sequence are left
  // as they are.
  auto issue = [&](int j0, int from, uint8_t* dst, int pg, const uint8_t* pool, const uint8_t* fresh,
                   const uint32_t(&off)[T::NI], const uint32_t(&noff)[T::NI]) __attribute__((always_inline)) {
    const int k_first = j0 + wrow0, k_last = k_first + 7;
    if (k_last < from) return;
    if (!FP8 && wanted(k_first, 8)) {
      const auto rs = rsrc_at(pool + size_t(pg) * page_stride);
#pragma unroll
      for (int i = 0; i < T::NI; ++i) {
        const int key = k_first + T::RPI * i + dma_row;
        if (key < lp && key >= wg_lo) dma16(rs, (lds_void*)(dst + (wrow0 + T::RPI * i) * T::RB), off[i]);
      }
    }
    if (k_last >= lp && k_first < total_len) {
      // base of the tile's first key as if it were a new token (it may lie before the
      // buffer; only rows at or past the prefix end are fetched from it)
      const ptrdiff_t row0 = ptrdiff_t(sq.cu) + j0 - lp;
      const auto rs = rsrc_at(fresh + (row0 * hkv + kvh) * T::RB);
#pragma unroll
      for (int i = 0; i < T::NI; ++i) {
        const int key = k_first + T::RPI * i + dma_row;
        if (key >= lp && key >= wg_lo && key < total_len)
          dma16(rs, (lds_void*)(dst + (wrow0 + T::RPI * i) * T::RB), noff[i]);
      }
    }
  };
  // fp8 pool rows into registers, values with their page's scale (`in_prefix`: the tile lies
  // wholly among cached keys from wg_lo on, so every row check passes)
  struct Rows8 {
    u32x4 x;
    float s;
  };
  auto load8 = [&](int j0, int pg, const uint8_t* pool, uint32_t off, Rows8& rw, bool in_prefix,
                   bool keys) __attribute__((always_inline)) {
    if (!in_prefix && !wanted(j0 + wrow0, 8)) return;
    const auto rs = rsrc_at(pool + size_t(pg) * page_stride);
    if (!keys) rw.s = vs_s[size_t(pg) * hkv + kvh];
    const u32x2 a = __builtin_amdgcn_raw_buffer_load_b64(rs, off, 0, 0);
    if constexpr (T::B8 == 16) {
      const u32x2 b = __builtin_amdgcn_raw_buffer_load_b64(rs, (keys ? off ^ 64u : off) + 4 * D, 0, 0);
      rw.x = u32x4{a.x, a.y, b.x, b.y};
    } else {
      rw.x = u32x4{a.x, a.y, 0u, 0u};
    }
  };
  // `keys`: the codes are stored as they are
  auto store8 = [&](int j0, int from, const Rows8& rw, uint8_t* dst, bool in_prefix, bool keys) __attribute__((always_inline)) {
    if (!in_prefix && (!wanted(j0 + wrow0, 8) || j0 + wrow0 + 7 < from)) return;
    const PageScale sc = page_scale(rw.s);
    auto widen = [&](uint32_t a, uint32_t b) { return keys ? fp8x8_f16x8(a, b) : fp8x8_f16x8(a, b, sc); };
    auto ok = [&](int key) { return in_prefix || (key < lp && key >= wg_lo); };
    if (ok(j0 + r8)) *reinterpret_cast<u32x4*>(dst + wrow0 * T::RB + 16 * lane) = widen(rw.x.x, rw.x.y);
    if constexpr (T::B8 == 16) {
      if (ok(j0 + r8 + 4)) *reinterpret_cast<u32x4*>(dst + (wrow0 + 4) * T::RB + 16 * lane) = widen(rw.x.z, rw.x.w);
    }
  };
  // fp8 pools: the new tokens' rows that this wave staged by DMA become fp16 in place
  // (before the barrier that publishes the tile)
  auto convert_new = [&](int j0, int from, uint8_t* dst) __attribute__((always_inline)) {
    const int k_first = j0 + wrow0, k_last = k_first + 7;
    if (k_last < lp || k_first >= total_len || k_last < from) return;
#pragma unroll
    for (int i = 0; i < T::NI; ++i) {
      const int key = k_first + T::RPI * i + dma_row;
      if (key >= lp && key >= wg_lo && key < total_len) {
        u32x4* ptr = reinterpret_cast<u32x4*>(dst + (wrow0 + T::RPI * i) * T::RB + 16 * lane);
        *ptr = bf16x8_f16x8(*ptr);
      }
    }
  };

  // fp8 pools: page (then key scale) of the 16-key group gi of the key tile whose value tile
  // starts at j0.  Behind the prefix or before what is visible: no page, scale unused.
  auto group_key = [&](int j0, int gi) { return j0 + kAhead + 16 * gi; };
  auto scale_page = [&](int key) -> int { return wanted(key, 16) ? bt_s[key >> pshift] : 0; };
  auto key_scale = [&](int key, int pg) -> float { return wanted(key, 16) ? ks_s[size_t(pg) * hkv + kvh] : 1.f; };

  // ---- LDS fragment addresses (relative to a stage), as in the extend kernel
  uint32_t k_addr[T::KT];
  {
    const int R = swap_bits_2_3(col);
#pragma unroll
    for (int kk = 0; kk < T::KT; ++kk) k_addr[kk] = R * T::RB + 16 * ((2 * kk + h) ^ k_swz<D>(R));
  }
  uint32_t v_addr[T::DB];
  {
    const int grp = lane >> 4, ri = lane & 15;
    const int kq = ri >> 2, a = ri & 3;
#pragma unroll
    for (int b = 0; b < T::DB; ++b)
      v_addr[b] = (8 * h + kq) * T::RB + 16 * ((4 * b + 2 * (grp & 1) + (a >> 1)) ^ v_swz<D>(kq)) + 8 * (a & 1);
  }

  f32x16 o[T::DB];
#pragma unroll
  for (int b = 0; b < T::DB; ++b) o[b] = f32x16{};
  // a row that sees no key of this item keeps m = kNegBig and l = 0: weight 0 in a merge
  float m_run = kNegBig, l_run = 0.f;
  const float c = sp.score_factor, cap2 = sp.cap2;
  auto tile0 = [&](int j) { return kv_begin + j * BLOCK_N; };

  // scores of the 32 keys in rows 32 blk on of key tile kt
  auto scores = [&](const uint8_t* kt, int blk, f32x16& s) __attribute__((always_inline)) {
    u32x4 kf[T::KT];
    auto read = [&](int kk) { kf[kk] = *reinterpret_cast<const u32x4*>(kt + k_addr[kk] + blk * 32 * T::RB); };
#pragma unroll
    for (int kk = 0; kk < T::K_AHEAD && kk < T::KT; ++kk) read(kk);
#pragma unroll
    for (int kk = 0; kk < T::KT; ++kk) {
      if (kk + T::K_AHEAD < T::KT) read(kk + T::K_AHEAD);
      if constexpr (D == 128) __builtin_amdgcn_sched_barrier(kMayCross);
      s = mfma16<FP8>(kf[kk], qf[kk], kk > 0 ? s : f32x16{});
    }
  };
  // What the scores of the block in hand are multiplied with: c, over fp8 pools times the scale
  // of their page (of the keys of element group i / 8, which share one).
  float cg[2] = {c, c};
  // ... of the block of keys from k0 on, with scores s and page scales ks0, ks1.  Where the
  // prefix ends among the 16 keys of a group, they are scaled in s.
  auto set_scales = [&](float ks0, float ks1, int k0, Keys keys, f32x16& s) __attribute__((always_inline)) {
    if constexpr (FP8) {
      if (keys == Keys::kNew || (keys == Keys::kAny && k0 >= lp)) {
        cg[0] = cg[1] = c;
        return;
      }
#pragma unroll
      for (int gi = 0; gi < 2; ++gi) {
        const float f = gi == 0 ? ks0 : ks1;
        const int cached = lp - (k0 + 16 * gi);  // of these keys, where that is below 16
        cg[gi] = keys == Keys::kPrefix || cached >= 16 ? c * f : c;
        if (keys == Keys::kAny && cached > 0 && cached < 16) {
#pragma unroll
          for (int e = 0; e < 8; ++e) s[8 * gi + e] *= 8 * h + e < cached ? f : 1.f;
        }
      }
    }
  };
  // Exponents (less m) of the block of keys from k0 on: element i holds key k0 + 16 (i / 8) + 8 h +
  // i % 8.  Not masked: every row sees all keys, none of them behind its own position if there is
  // a bias.
  auto exponents = [&](const f32x16& x, int k0, bool masked, float m, float (&f)[16]) __attribute__((always_inline)) {
    const float base = BIAS && !masked ? fmaf(slope2, static_cast<float>(k0 + 8 * h - pos), -m) : -m;
    const int at = k0 + 8 * h - lo, away = k0 + 8 * h - pos;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int n = 16 * (i >> 3) + (i & 7);
      float bias = base;
      if (BIAS && !masked) bias = fmaf(slope2, static_cast<float>(n), base);
      if (BIAS && masked) bias = fmaf(-slope2, fabsf(static_cast<float>(away + n)), -m);
      f[i] = exponent<CAP>(x[i], FP8 ? cg[i >> 3] : c, cap2, bias);
      if (masked && static_cast<uint32_t>(at + n) >= seen) f[i] = -INFINITY;
    }
  };
  auto block_max = [&](const f32x16& x, int k0, bool masked) __attribute__((always_inline)) -> float {
    float f[16], mx = -INFINITY;
    exponents(x, k0, masked, 0.f, f);
#pragma unroll
    for (int i = 0; i < 16; ++i) mx = fmaxf(mx, f[i]);
    return row_max(mx);
  };
  auto weights = [&](const f32x16& x, int k0, bool masked, u32x4(&pf)[2], float& lsum) __attribute__((always_inline)) {
    float f[16], la = 0.f, lb = 0.f;
    exponents(x, k0, masked, m_run, f);
#pragma unroll
    for (int gi = 0; gi < 2; ++gi) {
      float w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = __builtin_amdgcn_exp2f(f[8 * gi + e]);
      if constexpr (FP8) {
        const f16x2 one = {static_cast<_Float16>(1.f), static_cast<_Float16>(1.f)};
        f16x8 b;
#pragma unroll
        for (int e = 0; e < 8; ++e) b[e] = static_cast<_Float16>(w[e]);
#pragma unroll
        for (int e = 0; e < 8; e += 4) {
          la = __builtin_amdgcn_fdot2(f16x2{b[e], b[e + 1]}, one, la, false);
          lb = __builtin_amdgcn_fdot2(f16x2{b[e + 2], b[e + 3]}, one, lb, false);
        }
        pf[gi] = __builtin_bit_cast(u32x4, b);
      } else {
        const bf16x2 one = __builtin_bit_cast(bf16x2, 0x3F803F80u);
        bf16x8 b;
#pragma unroll
        for (int e = 0; e < 8; ++e) b[e] = static_cast<__bf16>(w[e]);
#pragma unroll
        for (int e = 0; e < 8; e += 4) {
          la = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{b[e], b[e + 1]}, one, la, false);
          lb = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{b[e + 2], b[e + 3]}, one, lb, false);
        }
        pf[gi] = __builtin_bit_cast(u32x4, b);
      }
    }
    lsum = la + lb;
  };
  // O^T += V^T P^T over the 32 keys in rows 32 blk on of value tile vt
  auto accumulate = [&](const uint8_t* vt, int blk, const u32x4(&pf)[2]) __attribute__((always_inline)) {
    u32x4 vf[2 * T::DB];
    auto read = [&](int i) __attribute__((always_inline)) {
      const int u = i / T::DB, b = i % T::DB;
      i16x4 part[2];
#pragma unroll
      for (int e4 = 0; e4 < 2; ++e4)
        part[e4] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (lds_i16x4*)(vt + v_addr[b] + (32 * blk + 16 * u + 4 * e4) * T::RB));
      vf[i] = __builtin_bit_cast(u32x4, __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7));
    };
#pragma unroll
    for (int i = 0; i < T::V_AHEAD; ++i) read(i);
#pragma unroll
    for (int i = 0; i < 2 * T::DB; ++i) {
      if (i + T::V_AHEAD < 2 * T::DB) read(i + T::V_AHEAD);
      if constexpr (D == 128) __builtin_amdgcn_sched_barrier(kMayCross);
      o[i % T::DB] = mfma16<FP8>(vf[i], pf[i / T::DB], o[i % T::DB]);
    }
  };
  // One block of 32 keys from k0 on, with scores x: the next block's scores (rows 32 blk on of
  // key tile kt) while this block's weights are formed, then this block's values.
  auto step = [&](const uint8_t* kt, const uint8_t* vt, int blk, int k0, Keys keys, const float (&ks)[T::KS], f32x16& x,
                  f32x16& s) __attribute__((always_inline)) {
    const bool masked = keys == Keys::kAny;
    u32x4 pf[2];
    float lsum;
    scores(kt, blk, s);
    weights(x, k0, masked, pf, lsum);
    if (__any(!(lsum <= kSumLimit))) {
      const float mx = fmaxf(block_max(x, k0, masked) - kHeadroom, m_run);
      const float alpha = __builtin_amdgcn_exp2f(m_run - mx);
      m_run = mx;
      l_run *= alpha;
#pragma unroll
      for (int b = 0; b < T::DB; ++b) o[b] *= alpha;
      weights(x, k0, masked, pf, lsum);
    }
    l_run += lsum;
    set_scales(ks[2 * blk], ks[2 * blk + 1], k0 + 32, keys, s);
    accumulate(vt, blk, pf);
  };

  // ---- prologue: the first 32 keys' scores against their exact max
  f32x16 xa = f32x16{}, xb = f32x16{};
  Rows8 k8{}, v8{};
  int pg_k = 0, pg_v = 0;  // pages of the tiles to be issued (fp8: loaded) next
  float ks_next[T::KS];    // fp8: key scales of the tile of the next iteration, pages of the one after it
  int pg_s[T::KS];
#pragma unroll
  for (int gi = 0; gi < T::KS; ++gi) {
    ks_next[gi] = 1.f;
    pg_s[gi] = 0;
  }
  // takes the key scales of iteration j's tile and loads those of the next one's
  auto next_scales = [&](int j, float (&ks)[T::KS], bool in_prefix) __attribute__((always_inline)) {
    if constexpr (FP8) {
#pragma unroll
      for (int gi = 0; gi < T::KS; ++gi) ks[gi] = ks_next[gi];
      if (!in_prefix && group_key(tile0(j + 1), 0) >= lp) return;
#pragma unroll
      for (int gi = 0; gi < T::KS; ++gi) {
        if (in_prefix) ks_next[gi] = ks_s[size_t(pg_s[gi]) * hkv + kvh];
        else ks_next[gi] = key_scale(group_key(tile0(j + 1), gi), pg_s[gi]);
        pg_s[gi] = in_prefix ? bt_s[group_key(tile0(j + 2), gi) >> pshift] : scale_page(group_key(tile0(j + 2), gi));
      }
    }
  };
  if (n_tiles > 0) {
    const int b0 = kv_begin;
    const int pgp = wrow0 >= kAhead ? load_page(b0 - kAhead) : 0;
    const int pk0 = load_page(b0 + kAhead), pv0 = load_page(b0);
    if (wrow0 >= kAhead) issue(b0 - kAhead, b0, lds_k1, pgp, k_pool, k_new, k_off, kn_off);
    issue(b0 + kAhead, 0, lds_k0, pk0, k_pool, k_new, k_off, kn_off);
    issue(b0, 0, lds_v0, pv0, v_pool, v_new, v_off, vn_off);
    pg_k = load_page(tile0(1) + kAhead);
    pg_v = load_page(tile0(1));
    if constexpr (FP8) {
      Rows8 kp{}, kf{}, vf{};
      if (wrow0 >= kAhead) load8(b0 - kAhead, pgp, k_pool, k8_off, kp, false, true);
      load8(b0 + kAhead, pk0, k_pool, k8_off, kf, false, true);
      load8(b0, pv0, v_pool, v8_off, vf, false, false);
      __builtin_amdgcn_s_waitcnt(0);
      if (wrow0 >= kAhead) store8(b0 - kAhead, b0, kp, lds_k1, false, true);
      store8(b0 + kAhead, 0, kf, lds_k0, false, true);
      store8(b0, 0, vf, lds_v0, false, false);
      if (wrow0 >= kAhead) convert_new(b0 - kAhead, b0, lds_k1);
      load8(tile0(1) + kAhead, pg_k, k_pool, k8_off, k8, false, true);
      load8(tile0(1), pg_v, v_pool, v8_off, v8, false, false);
      pg_k = load_page(tile0(2) + kAhead);
      pg_v = load_page(tile0(2));
#pragma unroll
      for (int gi = 0; gi < T::KS; ++gi) {
        ks_next[gi] = key_scale(group_key(b0, gi), scale_page(group_key(b0, gi)));
        pg_s[gi] = scale_page(group_key(tile0(1), gi));
      }
    }
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (wave_active && b0 < wave_max_lim) {
      scores(lds_k1, 1, xa);
      if constexpr (FP8)
        set_scales(key_scale(b0, scale_page(b0)), key_scale(b0 + 16, scale_page(b0 + 16)), b0, Keys::kAny, xa);
      const float mx = block_max(xa, b0, true);
      if (mx != -INFINITY) m_run = mx - kHeadroom;
    }
  }

  // iteration j: key tile j (scores of the blocks after this tile's first) and value tile
  // j are resident; tiles j + 1 go to the other stages
  auto iteration = [&](int j, uint8_t* k_cur, uint8_t* k_nxt, uint8_t* v_cur,
                       uint8_t* v_nxt) __attribute__((always_inline)) {
    __builtin_amdgcn_s_waitcnt(0);  // this wave's staging of tile j has landed
    if constexpr (FP8) {
      convert_new(tile0(j) + kAhead, 0, k_cur);
      convert_new(tile0(j), 0, v_cur);
    }
    __syncthreads();  // everyone's has; the other stages are no longer read
    float ks[T::KS];
    next_scales(j, ks, false);
    if (j + 1 < n_tiles) {
      if constexpr (FP8) {
        store8(tile0(j + 1) + kAhead, 0, k8, k_nxt, false, true);
        store8(tile0(j + 1), 0, v8, v_nxt, false, false);
      }
      issue(tile0(j + 1) + kAhead, 0, k_nxt, pg_k, k_pool, k_new, k_off, kn_off);
      issue(tile0(j + 1), 0, v_nxt, pg_v, v_pool, v_new, v_off, vn_off);
      if constexpr (FP8) {
        load8(tile0(j + 2) + kAhead, pg_k, k_pool, k8_off, k8, false, true);
        load8(tile0(j + 2), pg_v, v_pool, v8_off, v8, false, false);
      }
      pg_k = load_page(tile0(j + (FP8 ? 3 : 2)) + kAhead);
      pg_v = load_page(tile0(j + (FP8 ? 3 : 2)));
    }
    if (!wave_active || tile0(j) >= wave_max_lim) return;  // nothing visible from here on
    if (tile0(j) + BLOCK_N <= wave_lo) {  // nothing visible yet: only the next block's scores
      scores(k_cur, 1, xa);
      if constexpr (FP8) set_scales(ks[2], ks[3], tile0(j) + 64, Keys::kAny, xa);
      return;
    }
    step(k_cur, v_cur, 0, tile0(j), Keys::kAny, ks, xa, xb);
    step(k_cur, v_cur, 1, tile0(j) + 32, Keys::kAny, ks, xb, xa);
  };
  // Iterations whose staged tiles lie wholly in the cached prefix (fp8: whose loaded tiles do
  // too) and whose keys every row sees: a wave's rows come from one page, so they carry no mode
  // decisions and no mask.
  auto steady = [&](int j, const uint8_t* k_cur, uint8_t* k_nxt, const uint8_t* v_cur,
                    uint8_t* v_nxt) __attribute__((always_inline)) {
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    float ks[T::KS];
    next_scales(j, ks, true);
    if constexpr (FP8) {
      store8(tile0(j + 1) + kAhead, 0, k8, k_nxt, true, true);
      store8(tile0(j + 1), 0, v8, v_nxt, true, false);
      load8(tile0(j + 2) + kAhead, pg_k, k_pool, k8_off, k8, true, true);
      load8(tile0(j + 2), pg_v, v_pool, v8_off, v8, true, false);
    } else {
      const auto rk = rsrc_at(k_pool + size_t(pg_k) * page_stride), rv = rsrc_at(v_pool + size_t(pg_v) * page_stride);
#pragma unroll
      for (int i = 0; i < T::NI; ++i) dma16(rk, (lds_void*)(k_nxt + (wrow0 + T::RPI * i) * T::RB), k_off[i]);
#pragma unroll
      for (int i = 0; i < T::NI; ++i) dma16(rv, (lds_void*)(v_nxt + (wrow0 + T::RPI * i) * T::RB), v_off[i]);
    }
    pg_k = load_page(tile0(j + (FP8 ? 3 : 2)) + kAhead);
    pg_v = load_page(tile0(j + (FP8 ? 3 : 2)));
    if (!wave_active) return;
    step(k_cur, v_cur, 0, tile0(j), Keys::kPrefix, ks, xa, xb);
    step(k_cur, v_cur, 1, tile0(j) + 32, Keys::kPrefix, ks, xb, xa);
  };
  // Iterations whose staged tiles lie wholly among the new tokens and whose keys every row of
  // the workgroup sees.
  auto issue_new = [&](int j0, uint8_t* dst, const uint8_t* fresh,
                       const uint32_t(&noff)[T::NI]) __attribute__((always_inline)) {
    const ptrdiff_t row0 = ptrdiff_t(sq.cu) + j0 - lp;
    const auto rs = rsrc_at(fresh + (row0 * hkv + kvh) * T::RB);
#pragma unroll
    for (int i = 0; i < T::NI; ++i) dma16(rs, (lds_void*)(dst + (wrow0 + T::RPI * i) * T::RB), noff[i]);
  };
  auto steady_new = [&](int j, uint8_t* k_cur, uint8_t* k_nxt, uint8_t* v_cur,
                        uint8_t* v_nxt) __attribute__((always_inline)) {
    __builtin_amdgcn_s_waitcnt(0);
    if constexpr (FP8) {
      convert_new(tile0(j) + kAhead, 0, k_cur);
      convert_new(tile0(j), 0, v_cur);
    }
    __syncthreads();
    const float ks[T::KS] = {};  // (new keys have none)
    issue_new(tile0(j + 1) + kAhead, k_nxt, k_new, kn_off);
    issue_new(tile0(j + 1), v_nxt, v_new, vn_off);
    if (!wave_active) return;
    step(k_cur, v_cur, 0, tile0(j), Keys::kNew, ks, xa, xb);
    step(k_cur, v_cur, 1, tile0(j) + 32, Keys::kNew, ks, xb, xa);
  };
  // The ranges of iterations that those two loops may take (floors: the numerators may be
  // negative).  The first tile whose keys all rows see at the window's side:
  const int seen_by_all = max(0, (wg_lo_max - kv_begin + BLOCK_N - 1) >> 6);
  const int n_steady = min((lp - kv_begin - 96) >> 6, n_tiles - 1) - (FP8 ? 1 : 0);
  // (fp8: the scores' keys too, so that they take no page scale)
  const int new_begin = max(seen_by_all, FP8 ? (lp - kv_begin + 31) >> 6 : ((lp - kv_begin + 63) >> 6) - 1);
  // (a bias falls with the distance on both sides of a token: the loops know one side)
  const int new_end = min(min((total_len - kv_begin - 96) >> 6, ((BIAS ? first_lim : min_lim) - kv_begin) >> 6), n_tiles - 1);
  int j = 0;
  // (every loop takes two iterations at a time, so that an iteration's stages are fixed)
#pragma unroll 1
  for (int phase = 0; phase < 3; ++phase) {
    const int from = max(j, ((phase == 0 ? seen_by_all : new_begin) + 1) & ~1);
    const bool fast = phase < 2 && from + 1 < (phase == 0 ? n_steady : new_end);
    const int to = phase == 2 ? n_tiles : fast ? from : 0;
#pragma unroll 1
    for (; j < to; j += 2) {
      iteration(j, lds_k0, lds_k1, lds_v0, lds_v1);
      if (j + 1 < n_tiles) iteration(j + 1, lds_k1, lds_k0, lds_v1, lds_v0);
    }
    if (!fast) continue;
    if (phase == 0) {
#pragma unroll 1
      for (; j + 1 < n_steady; j += 2) {
        steady(j, lds_k0, lds_k1, lds_v0, lds_v1);
        steady(j + 1, lds_k1, lds_k0, lds_v1, lds_v0);
      }
    } else {
#pragma unroll 1
      for (; j + 1 < new_end; j += 2) {
        steady_new(j, lds_k0, lds_k1, lds_v0, lds_v1);
        steady_new(j + 1, lds_k1, lds_k0, lds_v1, lds_v0);
      }
    }
  }

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
