// Differential attention of chunks of new tokens over a paged cache.
//
// A workgroup of eight waves owns 128 packed query rows (token x query pair of one key
// pair): waves 0-3 compute the first map of 32 rows each, waves 4-7 the second map of
// the same rows.  Both read the same value tile, twice as wide as a key, so per 32 keys a
// wave runs D / 16 MFMAs of scores and D / 8 of values against 16 exponentials per lane.
// At the end the second map's waves hand over lam O2 / l2 through LDS and the first map's
// waves subtract, norm and store.  The difference is taken once per row, after both
// softmaxes: taking it in the weights would need the row sums first.
//
// S^T = K Q^T and O^T += V^T P^T with v_mfma_f32_32x32x16 (bf16; fp16 over fp8 pools).  fp8
// rows are widened into LDS, values with their page's scale (2^-10 of a value in all), key
// codes as they are, which fp16 holds exactly: their page's scale multiplies the scores in
// fp32 with the softmax scale, so that no error but fp32's grows with the scores (the scale
// rounded to fp16 and applied to the keys moved a page's weights by 2^-11 of its scores, 3% at
// scores of 60).  A 16-key group has one page and so one scale, a scalar; where the prefix ends
// inside a group its scores are scaled one by one.
// Softmax scale and running max enter the exponent in fp32, exp2(s c - m); the weights
// are rounded to the operand type (bf16: 2^-8 relative at most) and their sum is taken
// after that, so numerator and denominator agree.  For bf16 pools that rounding is the
// largest error besides the output's own (relative 2-norm 2.3e-3 in all, 1.7e-3 of it the
// output's).  fp16 weights and values, converted in LDS, would be as exact as the output's
// rounding, but took 17% (D = 64) to 25% (D = 128) more time.  The running max is raised
// only when a half-row's weight sum passes 2^16 (or is not finite).
//
// Scores run 32 keys ahead of the values: while a block's weights are formed, the scores
// of the next 32 keys are on the matrix cores.  So key tiles cover the 64 keys from 32
// behind the value tile's start, and both rotate through two stages with one barrier per
// 64 keys.  Tiles wholly in the prefix, and tiles wholly in the new tokens that all rows
// see, run in loops without row checks and masks.  At D = 128 the two stages of both take
// 128 KB of LDS, one workgroup per CU.
//
// 4096 new tokens on 32768 cached ones, 8 key pairs of 4 query pairs at D = 128, take 6.1 ms,
// 1150 TFLOP/s, on a card where a plain bf16 product of 8192^3 reaches 1385 (cards differ: 5.9-6.5
// ms, products 1214-1390); at D = 64 (half the matrix work per exponential) 1063 TFLOP/s; over fp8
// pools, whose rows are widened on the way, 1031 and 932.  Bound by what surrounds the matrix
// products: at D = 128 the matrix cores are busy 57% of the cycles and the waves wait 30% of
// theirs, as every value fragment read from LDS (1.67 LDS instructions per MFMA) feeds one
// product and a SIMD has two waves.
#include <hip/hip_runtime.h>

#include "../cw_internal.h"
#include "diff_common.h"

namespace cw {
namespace {

using namespace diff;

// Read through the constant address space so that loads with a uniform address are
// scalar loads: waiting for them never waits for tile staging issued before them.
typedef __attribute__((address_space(4))) const int32_t const_i32;
typedef __attribute__((address_space(4))) const float const_f32;

constexpr int kWaves = 8, kThreads = kWaves * 64;
// What the compiler may move across the point between a fragment's read and a product: vector,
// scalar and transcendental operations (the weights' exponentials run beside the products).
constexpr int kMayCross = 0x2 | 0x4 | 0x400;
constexpr int kAhead = 32;  // keys by which key tiles lie behind value tiles

// What is known of a block of keys whose scores are taken: all in the cached prefix, all among the
// new tokens and visible to every row, or neither.
enum class Keys { kPrefix, kNew, kMasked };

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc_at(const void* base) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, -1, 0x00020000);
}

// 16 bytes per lane from base + voff + soff straight into LDS (lane l's bytes land at
// dst + 16 l).  Not a template: see the extend kernel.
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
__device__ __forceinline__ uint32_t fp8x2_f16x2(uint32_t w, PageScale sc) {
  const f16x2 v = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(static_cast<int>(w), sc.p2, HI);
  return __builtin_bit_cast(uint32_t, v * sc.fm);
}
// Eight codes times their page's scale (values), or as they are (keys: exact).
__device__ __forceinline__ u32x4 fp8x8_f16x8(uint32_t lo, uint32_t hi, PageScale sc) {
  return u32x4{fp8x2_f16x2<false>(lo, sc), fp8x2_f16x2<true>(lo, sc), fp8x2_f16x2<false>(hi, sc),
               fp8x2_f16x2<true>(hi, sc)};
}
__device__ __forceinline__ u32x4 fp8x8_f16x8(uint32_t lo, uint32_t hi) {
  auto two = [](f16x2 v) { return __builtin_bit_cast(uint32_t, v); };
  return u32x4{two(__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(static_cast<int>(lo), 1.f, false)),
               two(__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(static_cast<int>(lo), 1.f, true)),
               two(__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(static_cast<int>(hi), 1.f, false)),
               two(__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(static_cast<int>(hi), 1.f, true))};
}
__device__ __forceinline__ u32x4 bf16x8_f16x8(u32x4 x) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float lo = __uint_as_float(x[i] << 16), hi = __uint_as_float(x[i] & 0xFFFF0000u);
    r[i] = __builtin_bit_cast(uint32_t, f16x2{static_cast<_Float16>(lo), static_cast<_Float16>(hi)});
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

template <int D, int P, bool FP8>
struct Geo {
  static constexpr int RB = 2 * D;                   // bytes per 16-bit row in LDS
  static constexpr int CPR = D / 8;                  // 16-byte chunks per row
  static constexpr int RPI = 64 / CPR;               // rows per wave DMA instruction
  static constexpr int NI = BLOCK_N / RPI / kWaves;  // DMA instructions per wave and matrix
  static constexpr int TILE = BLOCK_N * RB;          // bytes of one matrix's tile
  static constexpr int KT = D / 16;                  // k-steps of K Q^T
  static constexpr int DB = D / 32;                  // 32-row blocks of O^T per value half
  static constexpr int VB = 2 * DB;
  // Fragments read ahead of their products.  At D = 128, left to the compiler, each product
  // waited for its own read (matrix cores busy 53% of the cycles): 4096 tokens on 32768 keys, 4
  // key pairs, 3.05-3.12 ms, with these 2.95-3.03, over fp8 pages 3.42-3.49 and 3.34-3.43.  At D =
  // 64 the compiler's own order is 1-2% faster than any with reads ahead.
  static constexpr int K_AHEAD = D == 64 ? 0 : FP8 ? 1 : 2, V_AHEAD = D == 64 ? 0 : 2;
  static constexpr int PRB = FP8 ? D : RB;           // bytes per pool row
  static constexpr int B8 = D / 8;                   // fp8 bytes each lane stages per matrix
  static constexpr int KS = BLOCK_N / (P < 32 ? P : 32);  // fp8: key scales kept per tile, one per page and block
  static_assert(NI * RPI == 8, "each wave stages 8 rows of a tile");
};

template <int D, int P, bool FP8, int AP>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2)))
void diff_extend_kernel(DiffParams dp, PlanArg<AP> ap) {
  using T = Geo<D, P, FP8>;
  const ExtendParams& p = dp.a;
  // stages of key tiles (both maps) and value tiles (both halves), each its own array so
  // that the compiler can tell reads of one stage from the DMA into another; each also
  // holds one row group's second map at the end
  __shared__ __attribute__((aligned(1024))) uint8_t lds_k0[2 * T::TILE];
  __shared__ __attribute__((aligned(1024))) uint8_t lds_k1[2 * T::TILE];
  __shared__ __attribute__((aligned(1024))) uint8_t lds_v0[2 * T::TILE];
  __shared__ __attribute__((aligned(1024))) uint8_t lds_v1[2 * T::TILE];
  static_assert(2 * T::TILE == T::VB * 16 * 64 * 4, "a stage holds one wave's O");

  const WorkItem it = plan_ptr<AP>(ap, p.ap_items, p.items)[blockIdx.x];
  if (it.seq < 0) return;  // idle padding item (uniform across the workgroup)
  const SeqInfo sq = plan_ptr<AP>(ap, p.ap_seqs, p.seqs)[it.seq];
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int map = wave >> 2, sub = wave & 3;
  const int h = lane >> 5, col = lane & 31;
  const int G = p.gqa_group, hkv = 2 * p.num_kv_heads, hp = p.num_kv_heads * G;  // pool heads, query pairs
  const int pair = it.kvh;
  const int lp = sq.lp, total_len = sq.lp + sq.ls;
  const int32_t* bt = p.block_table + size_t(sq.bt_row) * p.bt_stride;
  const uint8_t* k_pool = static_cast<const uint8_t*>(p.k_pool);
  const uint8_t* v_pool = static_cast<const uint8_t*>(p.v_pool);
  const uint8_t* k_new = static_cast<const uint8_t*>(p.k_new);
  const uint8_t* v_new = static_cast<const uint8_t*>(p.v_new);

  // this lane's query row and its causal limit (number of visible keys)
  const int r_local = sub * 32 + col;
  const bool row_ok = r_local < it.rows;
  const int r = it.q_row0 + r_local;
  const int t = r / G, g = r - t * G;
  const int lim = row_ok ? lp + t + 1 : 0x7FFFFFFF;
  const bool wave_active = sub * 32 < it.rows;
  const int wave_min_lim = lp + (it.q_row0 + sub * 32) / G + 1;
  const int wave_last_row = it.q_row0 + min(sub * 32 + 31, it.rows - 1);
  const int wave_max_lim = lp + wave_last_row / G + 1;
  const size_t out_row = size_t(sq.cu + t) * hp + size_t(pair) * G + g;  // packed row of query pairs

  // stale LDS must be finite: rows past the sequence are never staged
  for (int i = tid; i < 2 * T::TILE / 16; i += kThreads) {
    reinterpret_cast<u32x4*>(lds_k0)[i] = u32x4{0u, 0u, 0u, 0u};
    reinterpret_cast<u32x4*>(lds_k1)[i] = u32x4{0u, 0u, 0u, 0u};
    reinterpret_cast<u32x4*>(lds_v0)[i] = u32x4{0u, 0u, 0u, 0u};
    reinterpret_cast<u32x4*>(lds_v1)[i] = u32x4{0u, 0u, 0u, 0u};
  }

  // Q^T as the B operand: k-step kk holds dims 16 kk + 8 h + [0, 8) of this row
  u32x4 qf[T::KT];
  {
    const uint16_t* qrow = static_cast<const uint16_t*>(p.q) + (2 * out_row + map) * D;
#pragma unroll
    for (int kk = 0; kk < T::KT; ++kk) {
      u32x4 v = {0u, 0u, 0u, 0u};
      if (row_ok) v = *reinterpret_cast<const u32x4*>(qrow + 16 * kk + 8 * h);
      qf[kk] = FP8 ? bf16x8_f16x8(v) : v;
    }
  }

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
    k_off[i] = ((R + kAhead) % P) * T::RB + kc;
    v_off[i] = (R % P) * T::RB + vc;
    kn_off[i] = R * hkv * T::RB + kc;
    vn_off[i] = R * hkv * T::RB + vc;
  }
  const uint32_t page_bytes = uint32_t(P) * T::PRB;  // one (page, head) block
  // fp8 rows.  D = 64: lane l stages 8 bytes of row 8 w + l / 8.  D = 128: load u of lane
  // l fetches what belongs at position l % 16 of row 8 w + 4 u + l / 16 (four rows on, a key's
  // swizzle differs in the bit of 8, a value's not at all).
  const int r8 = D == 128 ? wrow0 + (lane >> 4) : wrow0 + (lane >> 3);
  const int pos8 = D == 128 ? lane & 15 : lane & 7;
  const uint32_t k8_off = uint32_t(((r8 + kAhead) % P) * D + 8 * (pos8 ^ k_swz<D>(r8)));
  const uint32_t v8_off = uint32_t((r8 % P) * D + 8 * (pos8 ^ v_swz<D>(r8)));

  const_i32* bt_s = (const_i32*)bt;
  const_f32* ks_s = (const_f32*)p.k_scale;
  const_f32* vs_s = (const_f32*)p.v_scale;
  // physical page of this wave's rows of a tile whose first key is j0 (0: no prefix key)
  auto load_page = [&](int j0) -> int { return j0 + wrow0 < lp ? bt_s[(j0 + wrow0) / P] : 0; };

  // DMA of both matrices (maps or halves) of the tile whose first key is j0 into dst:
  // prefix rows from pool page pg (16-bit pools only), new rows from `fresh`; rows before
  // `from` or past the sequence are left as they are.
  auto issue = [&](int j0, int from, uint8_t* dst, int pg, const uint8_t* pool, const uint8_t* fresh,
                   const uint32_t(&off)[T::NI], const uint32_t(&noff)[T::NI]) __attribute__((always_inline)) {
    const int k_first = j0 + wrow0, k_last = k_first + 7;
    if (k_last < from) return;
    if (!FP8 && k_first < lp) {
      const auto rs = rsrc_at(pool + (size_t(pg) * hkv + 2 * pair) * page_bytes);
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int i = 0; i < T::NI; ++i)
          if (k_first + T::RPI * i + dma_row < lp)
            dma16(rs, (lds_void*)(dst + m * T::TILE + (wrow0 + T::RPI * i) * T::RB), off[i], m * page_bytes);
    }
    if (k_last >= lp && k_first < total_len) {
      // base of the tile's first key as if it were a new token (it may lie before the
      // buffer; only rows at or past the prefix end are fetched from it)
      const ptrdiff_t row0 = ptrdiff_t(sq.cu) + j0 - lp;
      const auto rs = rsrc_at(fresh + (row0 * hkv + 2 * pair) * T::RB);
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int i = 0; i < T::NI; ++i) {
          const int key = k_first + T::RPI * i + dma_row;
          if (key >= lp && key < total_len)
            dma16(rs, (lds_void*)(dst + m * T::TILE + (wrow0 + T::RPI * i) * T::RB), noff[i], m * T::RB);
        }
    }
  };
  const uint8_t* k_pool_pair = k_pool + size_t(2 * pair) * page_bytes;
  const uint8_t* v_pool_pair = v_pool + size_t(2 * pair) * page_bytes;
  const size_t page_stride = size_t(hkv) * page_bytes;
  // fp8 pool rows of both matrices into registers, values with their page's scales (`in_prefix`: the
  // tile lies wholly in the cached prefix, so every row check passes)
  struct Rows8 {
    u32x4 x[2];
    float s[2];
  };
  auto load8 = [&](int j0, int pg, const uint8_t* pool_pair, uint32_t off,
                   Rows8& rw, bool in_prefix, bool keys) __attribute__((always_inline)) {
    if (!in_prefix && j0 + wrow0 >= lp) return;
    const auto rs = rsrc_at(pool_pair + size_t(pg) * page_stride);
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      if (!keys) rw.s[m] = vs_s[size_t(pg) * hkv + 2 * pair + m];
      const u32x2 a = __builtin_amdgcn_raw_buffer_load_b64(rs, off, m * page_bytes, 0);
      if constexpr (T::B8 == 16) {
        const u32x2 b = __builtin_amdgcn_raw_buffer_load_b64(rs, (keys ? off ^ 64u : off) + 4 * D, m * page_bytes, 0);
        rw.x[m] = u32x4{a.x, a.y, b.x, b.y};
      } else {
        rw.x[m] = u32x4{a.x, a.y, 0u, 0u};
      }
    }
  };
  // `keys`: the codes are stored as they are
  auto store8 = [&](int j0, int from, const Rows8& rw, uint8_t* dst, bool in_prefix, bool keys) __attribute__((always_inline)) {
    if (!in_prefix && (j0 + wrow0 >= lp || j0 + wrow0 + 7 < from)) return;
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const PageScale sc = page_scale(rw.s[m]);
      auto widen = [&](uint32_t lo, uint32_t hi) { return keys ? fp8x8_f16x8(lo, hi) : fp8x8_f16x8(lo, hi, sc); };
      if constexpr (T::B8 == 16) {
        if (in_prefix || j0 + r8 < lp)
          *reinterpret_cast<u32x4*>(dst + m * T::TILE + wrow0 * T::RB + 16 * lane) = widen(rw.x[m].x, rw.x[m].y);
        if (in_prefix || j0 + r8 + 4 < lp)
          *reinterpret_cast<u32x4*>(dst + m * T::TILE + (wrow0 + 4) * T::RB + 16 * lane) = widen(rw.x[m].z, rw.x[m].w);
      } else if (in_prefix || j0 + r8 < lp) {
        *reinterpret_cast<u32x4*>(dst + m * T::TILE + wrow0 * T::RB + 16 * lane) = widen(rw.x[m].x, rw.x[m].y);
      }
    }
  };
  // fp8 pools: the new tokens' rows that this wave staged by DMA become fp16 in place
  // (before the barrier that publishes the tile)
  auto convert_new = [&](int j0, int from, uint8_t* dst) __attribute__((always_inline)) {
    const int k_first = j0 + wrow0, k_last = k_first + 7;
    if (k_last < lp || k_first >= total_len || k_last < from) return;
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int i = 0; i < T::NI; ++i) {
        const int key = k_first + T::RPI * i + dma_row;
        if (key >= lp && key < total_len) {
          u32x4* ptr = reinterpret_cast<u32x4*>(dst + m * T::TILE + (wrow0 + T::RPI * i) * T::RB + 16 * lane);
          *ptr = bf16x8_f16x8(*ptr);
        }
      }
  };

  // fp8 pools: page (then key scale, of this wave's map) of the key group g of the key tile whose
  // value tile starts at j0.  Behind the prefix: no page, scale unused.
  auto group_key = [&](int j0, int g) { return j0 + kAhead + g * (BLOCK_N / T::KS); };
  auto scale_page = [&](int key) -> int { return key < lp ? bt_s[key / P] : 0; };
  auto key_scale = [&](int key, int pg) -> float { return key < lp ? ks_s[size_t(pg) * hkv + 2 * pair + map] : 1.f; };

  // ---- LDS fragment addresses (relative to a stage's matrix), as in the extend kernel
  uint32_t k_addr[T::KT];
  {
    const int R = swap_bits_2_3(col);
#pragma unroll
    for (int kk = 0; kk < T::KT; ++kk) k_addr[kk] = map * T::TILE + R * T::RB + 16 * ((2 * kk + h) ^ k_swz<D>(R));
  }
  uint32_t v_addr[T::DB];
  {
    const int grp = lane >> 4, ri = lane & 15;
    const int kq = ri >> 2, a = ri & 3;
#pragma unroll
    for (int b = 0; b < T::DB; ++b)
      v_addr[b] = (8 * h + kq) * T::RB + 16 * ((4 * b + 2 * (grp & 1) + (a >> 1)) ^ v_swz<D>(kq)) + 8 * (a & 1);
  }

  f32x16 o[T::VB];
#pragma unroll
  for (int b = 0; b < T::VB; ++b) o[b] = f32x16{};
  // a wave that sees no key of this item keeps m = kNegBig and l = 0: weight 0 in a merge
  float m_run = kNegBig, l_run = 0.f;
  const float c = p.scale_log2;
  const int n_tiles = (it.kv_end - it.kv_begin + BLOCK_N - 1) / BLOCK_N;
  auto tile0 = [&](int j) { return it.kv_begin + j * BLOCK_N; };

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
  // causal mask of the block of keys from k0 on: element i holds key k0 + 16 (i / 8) + 8 h + i % 8
  auto mask = [&](int k0, f32x16& s) __attribute__((always_inline)) {
    if (k0 + 32 > wave_min_lim) {
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (k0 + 16 * (i >> 3) + 8 * h + (i & 7) >= lim) s[i] = -INFINITY;
    }
  };
  // What the scores of the block in hand are multiplied with in the exponent: c, over fp8 pools
  // times the scale of their page (of the keys of element group i / 8, which share one).
  float cg[2] = {c, c};
  // ... of the block of keys from k0 on, with scores s and page scales ks[0], ks[1].  Where the
  // prefix ends among the 16 keys of a group, they are scaled in s.
  auto set_scales = [&](float ks0, float ks1, int k0, Keys keys, f32x16& s) __attribute__((always_inline)) {
    if constexpr (FP8) {
      if (keys == Keys::kNew || (keys == Keys::kMasked && k0 >= lp)) {
        cg[0] = cg[1] = c;
        return;
      }
#pragma unroll
      for (int gi = 0; gi < 2; ++gi) {
        const float f = gi == 0 ? ks0 : ks1;
        const int cached = lp - (k0 + 16 * gi);  // of these keys, where that is below 16
        cg[gi] = keys == Keys::kPrefix || cached >= 16 ? c * f : c;
        if (keys == Keys::kMasked && cached > 0 && cached < 16) {
#pragma unroll
          for (int e = 0; e < 8; ++e) s[8 * gi + e] *= 8 * h + e < cached ? f : 1.f;
        }
      }
    }
  };
  auto block_max = [&](const f32x16& x) -> float {
    float mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < 16; ++i) mx = fmaxf(mx, FP8 ? x[i] * cg[i >> 3] : x[i]);
    return FP8 ? row_max(mx) : row_max(mx) * c;
  };
  auto weights = [&](const f32x16& x, u32x4(&pf)[2], float& lsum) __attribute__((always_inline)) {
    float la = 0.f, lb = 0.f;
#pragma unroll
    for (int gi = 0; gi < 2; ++gi) {
      float w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = __builtin_amdgcn_exp2f(fmaf(x[8 * gi + e], FP8 ? cg[gi] : c, -m_run));
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
    u32x4 vf[2 * T::VB];
    auto read = [&](int i) __attribute__((always_inline)) {
      const int u = i / T::VB, b = i % T::VB;
      i16x4 part[2];
#pragma unroll
      for (int e4 = 0; e4 < 2; ++e4)
        part[e4] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (lds_i16x4*)(vt + (b / T::DB) * T::TILE + v_addr[b % T::DB] + (32 * blk + 16 * u + 4 * e4) * T::RB));
      vf[i] = __builtin_bit_cast(u32x4, __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7));
    };
#pragma unroll
    for (int i = 0; i < T::V_AHEAD; ++i) read(i);
#pragma unroll
    for (int i = 0; i < 2 * T::VB; ++i) {
      if (i + T::V_AHEAD < 2 * T::VB) read(i + T::V_AHEAD);
      if constexpr (D == 128) __builtin_amdgcn_sched_barrier(kMayCross);
      o[i % T::VB] = mfma16<FP8>(vf[i], pf[i / T::VB], o[i % T::VB]);
    }
  };
  // One block of 32 keys: the next block's scores (rows 32 blk on of key tile kt, keys from
  // k_next on) while this block's weights are formed, then this block's values.
  auto step = [&](const uint8_t* kt, const uint8_t* vt, int blk, int k_next, Keys keys, const float (&ks)[T::KS], f32x16& x,
                  f32x16& s) __attribute__((always_inline)) {
    u32x4 pf[2];
    float lsum;
    scores(kt, blk, s);
    // At D = 64 a wave that forms weights goes before the one on its SIMD that feeds the matrix
    // cores: 4096 tokens on 32768 keys 1680 -> 1659 us, over fp8 pages 1915 -> 1861 (D = 128:
    // between 1% less and 1% more).
    if constexpr (D == 64) __builtin_amdgcn_s_setprio(1);
    weights(x, pf, lsum);
    if (__any(!(lsum <= kSumLimit))) {
      const float mx = fmaxf(block_max(x) - kHeadroom, m_run);
      const float alpha = __builtin_amdgcn_exp2f(m_run - mx);
      m_run = mx;
      l_run *= alpha;
#pragma unroll
      for (int b = 0; b < T::VB; ++b) o[b] *= alpha;
      weights(x, pf, lsum);
    }
    l_run += lsum;
    if constexpr (D == 64) __builtin_amdgcn_s_setprio(0);
    set_scales(ks[blk * T::KS / 2], ks[blk * T::KS / 2 + T::KS / 4], k_next, keys, s);
    if (keys == Keys::kMasked) mask(k_next, s);
    accumulate(vt, blk, pf);
  };

  // ---- prologue: the first 32 keys' scores against their exact max
  f32x16 xa = f32x16{}, xb = f32x16{};
  Rows8 k8{}, v8{};
  int pg_k = 0, pg_v = 0;  // pages of the tiles to be issued (fp8: loaded) next
  float ks_next[T::KS];    // fp8: key scales of the tile of the next iteration, pages of the one after it
  int pg_s[T::KS];
#pragma unroll
  for (int g2 = 0; g2 < T::KS; ++g2) {
    ks_next[g2] = 1.f;
    pg_s[g2] = 0;
  }
  // takes the key scales of iteration j's tile and loads those of the next one's
  auto next_scales = [&](int j, float (&ks)[T::KS], bool in_prefix) __attribute__((always_inline)) {
    if constexpr (FP8) {
#pragma unroll
      for (int g2 = 0; g2 < T::KS; ++g2) ks[g2] = ks_next[g2];
      if (!in_prefix && group_key(tile0(j + 1), 0) >= lp) return;
#pragma unroll
      for (int g2 = 0; g2 < T::KS; ++g2) {
        if (in_prefix) ks_next[g2] = ks_s[size_t(pg_s[g2]) * hkv + 2 * pair + map];
        else ks_next[g2] = key_scale(group_key(tile0(j + 1), g2), pg_s[g2]);
        pg_s[g2] = in_prefix ? bt_s[group_key(tile0(j + 2), g2) / P] : scale_page(group_key(tile0(j + 2), g2));
      }
    }
  };
  __syncthreads();  // zero fill done before any tile lands
  {
    const int b0 = it.kv_begin;
    const int pgp = load_page(b0 - kAhead < 0 && wrow0 < kAhead ? b0 : b0 - kAhead);
    const int pk0 = load_page(b0 + kAhead), pv0 = load_page(b0);
    issue(b0 - kAhead, b0, lds_k1, pgp, k_pool, k_new, k_off, kn_off);
    issue(b0 + kAhead, 0, lds_k0, pk0, k_pool, k_new, k_off, kn_off);
    issue(b0, 0, lds_v0, pv0, v_pool, v_new, v_off, vn_off);
    pg_k = load_page(tile0(1) + kAhead);
    pg_v = load_page(tile0(1));
    if constexpr (FP8) {
      Rows8 kp{}, kf{}, vf{};
      if (wrow0 >= kAhead) load8(b0 - kAhead, pgp, k_pool_pair, k8_off, kp, false, true);
      load8(b0 + kAhead, pk0, k_pool_pair, k8_off, kf, false, true);
      load8(b0, pv0, v_pool_pair, v8_off, vf, false, false);
      __builtin_amdgcn_s_waitcnt(0);
      if (wrow0 >= kAhead) store8(b0 - kAhead, b0, kp, lds_k1, false, true);
      store8(b0 + kAhead, 0, kf, lds_k0, false, true);
      store8(b0, 0, vf, lds_v0, false, false);
      convert_new(b0 - kAhead, b0, lds_k1);
      load8(tile0(1) + kAhead, pg_k, k_pool_pair, k8_off, k8, false, true);
      load8(tile0(1), pg_v, v_pool_pair, v8_off, v8, false, false);
      pg_k = load_page(tile0(2) + kAhead);
      pg_v = load_page(tile0(2));
#pragma unroll
      for (int g2 = 0; g2 < T::KS; ++g2) {
        ks_next[g2] = key_scale(group_key(b0, g2), scale_page(group_key(b0, g2)));
        pg_s[g2] = scale_page(group_key(tile0(1), g2));
      }
    }
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (wave_active && b0 < wave_max_lim) {
      scores(lds_k1, 1, xa);
      if constexpr (FP8)
        set_scales(key_scale(b0, scale_page(b0)), key_scale(b0 + 16, scale_page(b0 + 16)), b0, Keys::kMasked, xa);
      mask(b0, xa);
      const float mx = block_max(xa);
      if (mx != -INFINITY) m_run = mx - kHeadroom;  // a row that sees none of these keys sees none of the item
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
        load8(tile0(j + 2) + kAhead, pg_k, k_pool_pair, k8_off, k8, false, true);
        load8(tile0(j + 2), pg_v, v_pool_pair, v8_off, v8, false, false);
      }
      pg_k = load_page(tile0(j + (FP8 ? 3 : 2)) + kAhead);
      pg_v = load_page(tile0(j + (FP8 ? 3 : 2)));
    }
    if (!wave_active || tile0(j) >= wave_max_lim) return;  // nothing visible from here on
    step(k_cur, v_cur, 0, tile0(j) + 32, Keys::kMasked, ks, xa, xb);
    step(k_cur, v_cur, 1, tile0(j) + 64, Keys::kMasked, ks, xb, xa);
  };
  // Iterations whose staged tiles lie wholly in the cached prefix (fp8: whose loaded tiles do
  // too): every row sees all their keys and a wave's rows come from one page, so they carry
  // no mode decisions and no mask.
  auto issue_prefix = [&](uint8_t* dst, int pg, const uint8_t* pool_pair,
                          const uint32_t(&off)[T::NI]) __attribute__((always_inline)) {
    const auto rs = rsrc_at(pool_pair + size_t(pg) * page_stride);
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int i = 0; i < T::NI; ++i)
        dma16(rs, (lds_void*)(dst + m * T::TILE + (wrow0 + T::RPI * i) * T::RB), off[i], m * page_bytes);
  };
  auto steady = [&](int j, const uint8_t* k_cur, uint8_t* k_nxt, const uint8_t* v_cur,
                    uint8_t* v_nxt) __attribute__((always_inline)) {
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    float ks[T::KS];
    next_scales(j, ks, true);
    if constexpr (FP8) {
      store8(tile0(j + 1) + kAhead, 0, k8, k_nxt, true, true);
      store8(tile0(j + 1), 0, v8, v_nxt, true, false);
      load8(tile0(j + 2) + kAhead, pg_k, k_pool_pair, k8_off, k8, true, true);
      load8(tile0(j + 2), pg_v, v_pool_pair, v8_off, v8, true, false);
    } else {
      issue_prefix(k_nxt, pg_k, k_pool_pair, k_off);
      issue_prefix(v_nxt, pg_v, v_pool_pair, v_off);
    }
    pg_k = load_page(tile0(j + (FP8 ? 3 : 2)) + kAhead);
    pg_v = load_page(tile0(j + (FP8 ? 3 : 2)));
    if (!wave_active) return;
    step(k_cur, v_cur, 0, 0, Keys::kPrefix, ks, xa, xb);
    step(k_cur, v_cur, 1, 0, Keys::kPrefix, ks, xb, xa);
  };
  // Iterations whose staged tiles lie wholly among the new tokens and whose scores every
  // row of the workgroup sees.
  auto issue_new = [&](int j0, uint8_t* dst, const uint8_t* fresh,
                       const uint32_t(&noff)[T::NI]) __attribute__((always_inline)) {
    const ptrdiff_t row0 = ptrdiff_t(sq.cu) + j0 - lp;
    const auto rs = rsrc_at(fresh + (row0 * hkv + 2 * pair) * T::RB);
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int i = 0; i < T::NI; ++i)
        dma16(rs, (lds_void*)(dst + m * T::TILE + (wrow0 + T::RPI * i) * T::RB), noff[i], m * T::RB);
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
    step(k_cur, v_cur, 0, 0, Keys::kNew, ks, xa, xb);
    step(k_cur, v_cur, 1, 0, Keys::kNew, ks, xb, xa);
  };
  // (floors: the numerators may be negative)
  const int n_steady = min((lp - it.kv_begin - 96) >> 6, n_tiles - 1) - (FP8 ? 1 : 0);
  // (fp8: the scores' keys too, so that they take no page scale)
  const int new_begin = max(0, FP8 ? (lp - it.kv_begin + 31) >> 6 : ((lp - it.kv_begin + 63) >> 6) - 1);
  const int first_lim = lp + it.q_row0 / G + 1;
  const int new_end = min(min((total_len - it.kv_begin - 96) >> 6, ((first_lim - it.kv_begin - 96) >> 6) + 1), n_tiles - 1);
  int j = 0;
  for (; j + 1 < n_steady; j += 2) {
    steady(j, lds_k0, lds_k1, lds_v0, lds_v1);
    steady(j + 1, lds_k1, lds_k0, lds_v1, lds_v0);
  }
  // (every loop takes two iterations at a time, so that an iteration's stages are fixed)
  const int from = max(j, (new_begin + 1) & ~1);
#pragma unroll 1
  for (int rest = from + 1 < new_end ? 0 : 1; rest < 2; ++rest) {
    const int to = rest == 0 ? from : n_tiles;
#pragma unroll 1
    for (; j < to; j += 2) {
      iteration(j, lds_k0, lds_k1, lds_v0, lds_v1);
      if (j + 1 < n_tiles) iteration(j + 1, lds_k1, lds_k0, lds_v1, lds_v0);
    }
    if (rest == 0) {
#pragma unroll 1
      for (; j + 1 < new_end; j += 2) {
        steady_new(j, lds_k0, lds_k1, lds_v0, lds_v1);
        steady_new(j + 1, lds_k1, lds_k0, lds_v1, lds_v0);
      }
    }
  }

  const float l_tot = row_sum(l_run);
  if (it.part >= 0) {  // unnormalised partials of both maps, merged by diff_combine
    if (!wave_active) return;
    const size_t slot = size_t(it.part) * p.part_rows + map * (p.part_rows / 2) + r_local;
    float* po = static_cast<float*>(p.part_o) + slot * (2 * D);
#pragma unroll
    for (int b = 0; b < T::VB; ++b)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4)
        *reinterpret_cast<f32x4*>(po + 32 * b + 8 * q4 + 4 * h) =
            f32x4{o[b][4 * q4], o[b][4 * q4 + 1], o[b][4 * q4 + 2], o[b][4 * q4 + 3]};
    if (h == 0) *reinterpret_cast<f32x2*>(p.part_ml + slot * 2) = f32x2{m_run, l_tot};
    return;
  }
  // the second map's waves hand over lam O2 / l2, each through a stage of its own
  __syncthreads();  // the stages are no longer read
  uint8_t* const stage = sub == 0 ? lds_k0 : sub == 1 ? lds_k1 : sub == 2 ? lds_v0 : lds_v1;
  float* const ex = reinterpret_cast<float*>(stage);
  if (map == 1 && wave_active) {
    const float f = row_ok ? dp.lam[pair * G + g] / l_tot : 0.f;
#pragma unroll
    for (int b = 0; b < T::VB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) ex[(16 * b + i) * 64 + lane] = o[b][i] * f;
  }
  __syncthreads();
  if (map == 1 || !wave_active) return;
  const float inv = 1.f / l_tot;
#pragma unroll
  for (int b = 0; b < T::VB; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[b][i] = fmaf(o[b][i], inv, -ex[(16 * b + i) * 64 + lane]);
  uint16_t* orow = static_cast<uint16_t*>(p.out) + out_row * (2 * D);
  // (both lanes of a row take part in its sum, stored or not)
  if (row_ok) store_row<T::VB>(dp, orow, h, o);
}

template <int D, int P, bool FP8>
hipError_t launch_t(const DiffParams& p, hipStream_t stream, const ArgPlanBuf* ap) {
  const dim3 grid(p.a.n_items), block(kThreads);
  if (ap != nullptr && ap->small())
    hipLaunchKernelGGL((diff_extend_kernel<D, P, FP8, kPlanInSmallArgs>), grid, block, 0, stream, p, ap->small_plan());
  else if (ap != nullptr)
    hipLaunchKernelGGL((diff_extend_kernel<D, P, FP8, kPlanInArgs>), grid, block, 0, stream, p, ap->plan);
  else
    hipLaunchKernelGGL((diff_extend_kernel<D, P, FP8, kPlanInMemory>), grid, block, 0, stream, p, NoArgPlan{});
  return hipGetLastError();
}

}  // namespace

hipError_t launch_diff_extend(const DiffParams& p, int head_dim, int page_size, bool fp8, hipStream_t stream,
                              const ArgPlanBuf* ap) {
  if (p.a.n_items <= 0) return hipSuccess;
#define CW_CASE(D_, P_)                  \
  if (head_dim == D_ && page_size == P_) \
    return fp8 ? launch_t<D_, P_, true>(p, stream, ap) : launch_t<D_, P_, false>(p, stream, ap);
  CW_CASE(64, 16)
  CW_CASE(64, 64)
  CW_CASE(128, 16)
  CW_CASE(128, 64)
#undef CW_CASE
  return hipErrorInvalidValue;
}

}  // namespace cw
