// Attention with shaped scores of single new tokens over a paged cache, HBM-streaming.
//
// Work item = one wave: the G <= 16 query heads of one kv head against a chunk of at most 64
// pages of one sequence's visible prefix, plus the new token's own key when the chunk ends the
// sequence.  The chunks start where the window does (shaped_decode_base); keys before the
// token's first visible position are skipped by whole tiles, and what is left of them in the
// first tile is fetched as the first visible key again (its score masked), so no key, value or
// page before it is read.  Every visible K/V byte is read once: bound by HBM.  48 tokens on 2k-32k
// keys, 8 kv heads of 128, capped: fp8 pages 1.64 GB in 301 us with the merge (5.4 TB/s); bf16 pages and a
// window of 4096 0.78 GB in 140 us (5.6 TB/s).
//
// The pipeline is the decode kernels': 32-key tiles, DMA'd into LDS by global_load_lds_dwordx4
// in three stages (six of 4 KB tiles) with the kernel's own vmcnt waits, three waves per CU for
// 16 KB tiles and six for smaller ones.  Queries are padded to 32 columns of an MFMA.  Cap, bias,
// mask and running max enter the exponent in fp32 (shaped_common.h).  fp8 codes stay codes in LDS
// and are widened exactly; a page's K scale multiplies its scores, its V scale the weights.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "../cw_internal.h"
#include "../plan_expand.h"
#include "shaped_common.h"

namespace cw {
namespace {

using namespace shaped;

constexpr int kScalarSearchSeqs = 8;  // up to here an item's sequence is searched by scalar loads
constexpr int kKeys = 32;             // keys of a tile
// Up to this ratio of a chunk's V scales, their products with the weights are held in fp16: a
// column's largest weight is at least 2^kHeadroom, its product at least 1, and what fp16 drops of
// any other (2^-25) at most 2^-25 of that.  Further apart they are pairs of bf16; a scale of 0 is far
// from any other (all of the large weights may be its keys').
constexpr float kNearScales = 256.f;

// 16 bytes per lane from global memory straight into LDS (lane l at LDS address m0 + 16 l),
// nontemporal: every byte is read once.  Inline assembly, so that the compiler does not
// drain the DMA in flight at the loop header; the kernel's own waits order it.
__device__ __forceinline__ void dma16(const void* src, uint32_t lds_addr) {
  asm volatile("global_load_lds_dwordx4 %0, off nt" ::"v"(src), "{m0}"(lds_addr) : "memory");
}
template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  static_assert(N >= 0 && N < 64, "vmcnt range");
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// Waits until at most `behind` tiles (up to N) of DMA instructions each are outstanding.
template <int N, int DMA>
__device__ __forceinline__ void wait_tiles(int behind) {
  if constexpr (N == 0) {
    wait_vmcnt<0>();
  } else {
    if (behind >= N) wait_vmcnt<N * DMA>();
    else wait_tiles<N - 1, DMA>(behind);
  }
}
__device__ __forceinline__ void wait_lgkmcnt0() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ uint32_t lds_addr(const void* p) {
  return static_cast<uint32_t>(reinterpret_cast<uintptr_t>((const lds_void*)p));
}

template <bool HI>
__device__ __forceinline__ uint32_t fp8x2_bf16x2(uint32_t v) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(static_cast<int>(v), 1.0f, HI));
}
__device__ __forceinline__ bf16x8 fp8x8_bf16x8(u32x2 c) {
  const u32x4 r = {fp8x2_bf16x2<false>(c.x), fp8x2_bf16x2<true>(c.x), fp8x2_bf16x2<false>(c.y), fp8x2_bf16x2<true>(c.y)};
  return __builtin_bit_cast(bf16x8, r);
}
template <bool HI>
__device__ __forceinline__ uint32_t fp8x2_f16x2(uint32_t v) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(static_cast<int>(v), 1.0f, HI));
}
__device__ __forceinline__ f16x8 fp8x8_f16x8(u32x2 c) {
  const u32x4 r = {fp8x2_f16x2<false>(c.x), fp8x2_f16x2<true>(c.x), fp8x2_f16x2<false>(c.y), fp8x2_f16x2<true>(c.y)};
  return __builtin_bit_cast(f16x8, r);
}

__host__ __device__ constexpr int tile_bytes(int d, bool fp8) { return 2 * kKeys * d * (fp8 ? 1 : 2); }
__host__ __device__ constexpr int stages(int d, bool fp8) { return tile_bytes(d, fp8) > 4096 ? 3 : 6; }

template <int D, bool FP8>
struct Geo {
  static constexpr int RB = D * (FP8 ? 1 : 2);      // bytes per row
  static constexpr int MAT = kKeys * RB;            // bytes of one matrix of a tile
  static constexpr int TILE = 2 * MAT;
  static constexpr int STAGES = stages(D, FP8);
  static constexpr int CPR = RB / 16;               // 16-byte chunks per row
  static constexpr int RPI = 64 / CPR;              // rows per DMA instruction
  static constexpr int NI = kKeys / RPI;            // DMA instructions per matrix
  static constexpr int DMA = 2 * NI;                // per tile
  static constexpr int KT = D / 16;                 // k-steps of K Q^T
  static constexpr int DB = D / 32;                 // 32-row blocks of O^T
  static_assert(RPI <= 16, "an instruction's rows lie in one page");
  static_assert((STAGES - 1) * DMA < 64, "vmcnt range");
};

// Chunk swizzles for conflict-free LDS reads, as in the decode kernel
template <int RB>
__device__ __forceinline__ int k_swz(int row) {
  const int s = swap_bits_2_3(row);
  return RB == 256 ? (s & 15) : RB == 128 ? ((s >> 1) & 7) : ((s >> 2) & 3);
}
template <int RB>
__device__ __forceinline__ int v_swz16(int row) {
  return RB == 256 ? 4 * (row & 3) : 4 * ((row >> 1) & 1);
}
template <int RB>
__device__ __forceinline__ int v_swz8(int row) {
  return RB == 128 ? 2 * ((row >> 1) & 3) : 2 * ((row >> 2) & 1);
}

template <int D, bool FP8, bool CAP, int AP>
__global__ __launch_bounds__(64) void shaped_decode_kernel(ShapedParams sp, PlanArg<AP> ap) {
  using T = Geo<D, FP8>;
  const ExtendParams& p = sp.a;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[T::STAGES * T::TILE];  // stages, then O
  __shared__ float sh_row[3][32];  // per column: l, and the factors of its O and of the new value

  WorkItem it;
  if constexpr (AP != kPlanInMemory) {  // the plan in the kernel arguments, in compact form
    const ExpandDesc& d = *reinterpret_cast<const ExpandDesc*>(ap.bytes + p.ap_desc);
    const DecodeRec* rec = reinterpret_cast<const DecodeRec*>(ap.bytes + d.rec_off);
    const int i = blockIdx.x;
    int b_full = 0;
    if (i < d.n_full) {
      if (d.n_seqs <= kScalarSearchSeqs) {
        for (int k = 1; k < d.n_seqs; ++k) b_full += rec[k].full_off <= i ? 1 : 0;  // scalar loads
      } else {
        b_full = wave_last_at_most(d.n_seqs, i, static_cast<int>(threadIdx.x), [&](int k) { return rec[k].full_off; });
      }
    }
    it = expand_item_at(rec, reinterpret_cast<const int32_t*>(ap.bytes + d.tail_off), d, i, b_full);
  } else {
    it = p.items[blockIdx.x];
  }
  if (it.seq < 0) return;
  const SeqInfo sq = plan_ptr<AP>(ap, p.ap_seqs, p.seqs)[it.seq];
  const int lane = threadIdx.x;
  const int h = lane >> 5, col = lane & 31;  // this lane's column: a query head of the group
  const int G = p.gqa_group, hkv = p.num_kv_heads, hq = hkv * G;
  const int kvh = it.kvh;
  const int lp = sq.lp;
  const int tok = sq.cu;  // the sequence's single new token
  const int pshift = sp.page_shift, P = 1 << pshift;
  const int32_t* bt = p.block_table + size_t(sq.bt_row) * p.bt_stride;
  const uint8_t* k_pool = static_cast<const uint8_t*>(p.k_pool);
  const uint8_t* v_pool = static_cast<const uint8_t*>(p.v_pool);
  const bool row_ok = col < G;

  // the visible keys of this item: of the prefix [lo, ke), taken in tiles from kb on; the new
  // key when kv_end passes lp
  const int base = shaped_decode_base(lp, sp.window, max(kKeys, P));
  int lo = sp.window > 0 ? max(0, lp + 1 - sp.window) : 0;
  if (sp.begins != nullptr) lo = max(lo, __builtin_amdgcn_readfirstlane(sp.begins[tok]));
  int kb = base + it.kv_begin;
  const int ke = min(base + it.kv_end, lp);
  const bool has_new = base + it.kv_end > lp && lo <= lp;
  if (lo > kb) kb += min(lo - kb, max(0, ke - kb)) / kKeys * kKeys;
  const int first = max(kb, lo);  // the first key that is read
  const int n_tiles = ke > first ? (ke - kb + kKeys - 1) / kKeys : 0;

  // page ids (and fp8 scales) of the chunk: lane j holds page kb / P + j
  const int page0 = kb >> pshift;
  const int n_pages = n_tiles > 0 ? ((ke - 1) >> pshift) - page0 + 1 : 0;
  const bool has_page = lane < n_pages && page0 + lane >= first >> pshift;
  int my_pg = 0;
  float my_ks = 1.f, my_vs = 0.f;
  if (has_page) {
    my_pg = bt[page0 + lane];
    if constexpr (FP8) {
      const size_t si = size_t(my_pg) * hkv + kvh;
      my_ks = p.k_scale[si];
      my_vs = p.v_scale[si];
    }
  }
  // Q^T (B operand): this column's query.  bf16 pools: k-step kk holds dims 16 kk + 8 h + e;
  // fp8 pools read 16 dims per fragment, so k-steps 2 t and 2 t + 1 hold dims 32 t + 16 h +
  // 8 (kk & 1) + e.  And the new token's key and value (PER dims per lane), read here so that
  // their latency does not end the item.
  auto dim0 = [&](int kk) { return FP8 ? 32 * (kk >> 1) + 16 * h + 8 * (kk & 1) : 16 * kk + 8 * h; };
  bf16x8 qf[T::KT];
  {
    const uint16_t* qrow = static_cast<const uint16_t*>(p.q) + (size_t(tok) * hq + size_t(kvh) * G + col) * D;
#pragma unroll
    for (int kk = 0; kk < T::KT; ++kk) {
      u32x4 v = {0u, 0u, 0u, 0u};
      if (row_ok) v = *reinterpret_cast<const u32x4*>(qrow + dim0(kk));
      qf[kk] = __builtin_bit_cast(bf16x8, v);
    }
  }
  bf16x8 k_own[T::KT];
  constexpr int PER = D / 64;
  typedef float fvec __attribute__((ext_vector_type(PER)));
  typedef uint16_t hvec __attribute__((ext_vector_type(PER)));
  const int d0 = lane * PER;
  hvec v_own = hvec(0);
  if (has_new) {
    const size_t row = (size_t(tok) * hkv + kvh) * D;
#pragma unroll
    for (int kk = 0; kk < T::KT; ++kk)
      k_own[kk] = *reinterpret_cast<const bf16x8*>(static_cast<const uint16_t*>(p.k_new) + row + dim0(kk));
    v_own = *reinterpret_cast<const hvec*>(static_cast<const uint16_t*>(p.v_new) + row + d0);
  }
  const float slope2 = sp.slopes != nullptr && row_ok ? sp.slopes[kvh * G + col] * kLog2e : 0.f;

  // DMA of tile t: instruction j of a matrix covers tile rows [j RPI, (j + 1) RPI); rows before
  // the first visible key or past the chunk's prefix end fetch the nearest visible one (their
  // scores are masked), so every tile issues exactly DMA instructions and the waits are exact.
  const int dma_row = lane / T::CPR, dma_pos = lane % T::CPR;
  auto issue_tile = [&](int t, uint32_t dst) __attribute__((always_inline)) {
    const int j0 = kb + t * kKeys;
#pragma unroll
    for (int j = 0; j < T::NI; ++j) {
      const int R = j * T::RPI + dma_row;
      const int key = max(min(j0 + R, ke - 1), first);
      const int r0 = max(min(j0 + j * T::RPI, ke - 1), first);  // (uniform: in the same page)
      const int pg = __builtin_amdgcn_readlane(my_pg, min((r0 >> pshift) - page0, 63));
      const size_t row = (size_t(pg) * hkv + kvh) * (size_t(P) * T::RB) + size_t(key & (P - 1)) * T::RB;
      const uint32_t kc = 16 * (dma_pos ^ k_swz<T::RB>(R));
      const uint32_t vc = 16 * (dma_pos ^ (FP8 ? v_swz8<T::RB>(R) : v_swz16<T::RB>(R)));
      dma16(k_pool + row + kc, dst + j * T::RPI * T::RB);
      dma16(v_pool + row + vc, dst + T::MAT + j * T::RPI * T::RB);
    }
  };

  f32x16 o[T::DB];
#pragma unroll
  for (int b = 0; b < T::DB; ++b) o[b] = f32x16{};
  float m_run = kNegBig, l_run = 0.f;
  const float c = sp.score_factor, cap2 = sp.cap2;

  // Q, the new token's rows, slopes and the page ids land first (the addresses need the ids),
  // so only DMA is outstanding in the loop
  __builtin_amdgcn_s_waitcnt((7 << 4) | (15 << 8));
  const uint32_t lds_base = lds_addr(lds);
#pragma unroll 1
  for (int t = 0; t < min(n_tiles, T::STAGES); ++t) issue_tile(t, lds_base + t * T::TILE);
  // fp8: the largest V scale of the chunk is taken out of the weights (and multiplied back at
  // the end), so that fp16 holds them whatever the scales' size; `wide`: they lie further apart
  // than kNearScales, and weights times scales keep fp32's range.
  float vs_max = 1.f;
  bool wide = false;
  if constexpr (FP8) {
    const float x = fabsf(my_vs);
    vs_max = x;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) vs_max = fmaxf(vs_max, __shfl_xor(vs_max, d));
    wide = __any(has_page && x * kNearScales < vs_max);
    if (wide || vs_max == 0.f) vs_max = 1.f;
    my_vs = my_vs / vs_max;
  }
  float x_own = 0.f;  // the new token's exponent, under the first tiles' latency
  if (has_new) {
#pragma unroll
    for (int kk = 0; kk < T::KT; ++kk)
#pragma unroll
      for (int e = 0; e < 8; ++e) x_own = fmaf(static_cast<float>(qf[kk][e]), static_cast<float>(k_own[kk][e]), x_own);
    x_own = exponent<CAP>(row_sum(x_own), c, cap2, 0.f);
  }

  // TWO: how the weights are given to the second product (below)
  auto compute = [&](int t, const uint8_t* st, auto two) __attribute__((always_inline)) {
    constexpr bool TWO = decltype(two)::value;
    const int j0 = kb + t * kKeys;
    f32x16 s = f32x16{};
    const int R = swap_bits_2_3(col);  // row m of the block reads key swap(m)
    const uint8_t* km = st + R * T::RB;
    if constexpr (FP8) {
#pragma unroll
      for (int t2 = 0; t2 < T::KT / 2; ++t2) {
        const u32x4 raw = *reinterpret_cast<const u32x4*>(km + 16 * ((2 * t2 + h) ^ k_swz<T::RB>(R)));
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fp8x8_bf16x8(u32x2{raw.x, raw.y}), qf[2 * t2], s, 0, 0, 0);
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fp8x8_bf16x8(u32x2{raw.z, raw.w}), qf[2 * t2 + 1], s, 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int kk = 0; kk < T::KT; ++kk) {
        const bf16x8 kf = *reinterpret_cast<const bf16x8*>(km + 16 * ((2 * kk + h) ^ k_swz<T::RB>(R)));
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[kk], s, 0, 0, 0);
      }
    }
    // element i holds key j0 + 16 (i / 8) + 8 h + i % 8; the keys of half-group i / 8 share a page
    float cg[2] = {c, c}, vs[2] = {1.f, 1.f};
    if constexpr (FP8) {
#pragma unroll
      for (int s8 = 0; s8 < 2; ++s8) {
        const int q = min(((j0 + 16 * s8) >> pshift) - page0, 63);
        cg[s8] = c * __int_as_float(__builtin_amdgcn_readlane(__float_as_int(my_ks), q));
        vs[s8] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(my_vs), q));
      }
    }
    // exponents against the running max as it stands
    const bool edge = j0 < first || j0 + kKeys > ke;  // (uniform)
    auto exponents = [&](float m, float(&f)[16]) __attribute__((always_inline)) {
      const float near = fmaf(slope2, static_cast<float>(j0 + 8 * h - lp), -m);
#pragma unroll
      for (int i = 0; i < 16; ++i)
        f[i] = exponent<CAP>(s[i], cg[i >> 3], cap2, fmaf(slope2, static_cast<float>(16 * (i >> 3) + (i & 7)), near));
      if (edge) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = j0 + 16 * (i >> 3) + 8 * h + (i & 7);
          if (key < first || key >= ke) f[i] = -INFINITY;
        }
      }
    };
    // weights; the max is raised only when a half-column's sum passes half of kSumLimit (a single
    // fp16 weight ends at 65504) or is not finite, as on an item's first tile
    float w[16], tsum;
    auto weights = [&]() __attribute__((always_inline)) {
      float f[16];
      exponents(m_run, f);
      tsum = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        w[i] = __builtin_amdgcn_exp2f(f[i]);
        tsum += w[i];
      }
    };
    weights();
    if (__any(!(tsum <= 0.5f * kSumLimit))) {
      float f[16];
      auto largest = [&](float m) __attribute__((always_inline)) -> float {
        exponents(m, f);
        float mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = fmaxf(mx, f[i]);
        return floorf(row_max(mx));
      };
      RunningMax rm(m_run, largest(0.f));
      rm.settle(m_run, largest(rm.near));
      const float alpha = rm.raise(m_run);
      l_run *= alpha;
#pragma unroll
      for (int b = 0; b < T::DB; ++b) o[b] *= alpha;
      tsum = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        w[i] = __builtin_amdgcn_exp2f(rm.exponent(f[i]));
        tsum += w[i];
      }
    }
    l_run += tsum;
    // O^T += V^T P^T over the tile's two 16-key slices.  Neither form of the weights adds to the
    // output's own rounding.  TWO: a weight is the sum of two bf16 (2^-16), for a second MFMA;
    // else (fp8 pools) fp16 (2^-11), which holds the codes exactly too.
    const int grp = lane >> 4, ri = lane & 15;
    const uint8_t* vt = st + T::MAT;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      bf16x8 pf, pl;
      f16x8 ph;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = FP8 ? w[8 * u + e] * vs[u] : w[8 * u + e];
        if constexpr (TWO) {
          pf[e] = static_cast<__bf16>(x);
          pl[e] = static_cast<__bf16>(x - static_cast<float>(pf[e]));
        } else {
          ph[e] = static_cast<_Float16>(x);
        }
      }
#pragma unroll
      for (int b = 0; b < T::DB; ++b) {
        u32x2 codes;
        bf16x8 vf;
        if constexpr (FP8) {
          // source lane (k, a) = (ri / 2, ri % 2): key 16 u + 8 h + k, dims 32 b + 16 (grp & 1) + 8 a
          const int Rv = 16 * u + 8 * h + (ri >> 1);
          const int dbyte = 32 * b + 16 * (grp & 1) + 8 * (ri & 1);
          const int off = Rv * T::RB + 16 * ((dbyte >> 4) ^ v_swz8<T::RB>(Rv)) + (dbyte & 15);
          const i32x2 raw = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2*)(vt + off));
          codes = u32x2{static_cast<uint32_t>(raw.x), static_cast<uint32_t>(raw.y)};
          if constexpr (TWO) vf = fp8x8_bf16x8(codes);
        } else {
          const int kq = ri >> 2, a = ri & 3;
          const int chunk = 4 * b + 2 * (grp & 1) + (a >> 1);
          i16x4 part[2];
#pragma unroll
          for (int e4 = 0; e4 < 2; ++e4) {
            const int Rv = 16 * u + 8 * h + 4 * e4 + kq;
            const int off = Rv * T::RB + 16 * (chunk ^ v_swz16<T::RB>(Rv)) + 8 * (a & 1);
            part[e4] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(vt + off));
          }
          vf = __builtin_bit_cast(bf16x8, __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7));
        }
        if constexpr (TWO) {
          o[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf, o[b], 0, 0, 0);
          o[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pl, o[b], 0, 0, 0);
        } else {
          o[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fp8x8_f16x8(codes), ph, o[b], 0, 0, 0);
        }
      }
    }
  };
  // Tile t lives in stage t % STAGES.  A step waits for its tile (those issued after it may
  // still fly), computes on it, then refills the stage if there is a tile for it.
  auto tiles = [&](auto two) __attribute__((always_inline)) {
    uint32_t off = 0;
#pragma unroll 1
    for (int t = 0; t < n_tiles; ++t) {
      const int behind = n_tiles - 1 - t;
      wait_tiles<T::STAGES - 1, T::DMA>(behind);
      compute(t, lds + off, two);
      if (behind >= T::STAGES) {
        wait_lgkmcnt0();  // the stage's reads are done before it is refilled
        issue_tile(t + T::STAGES, lds_base + off);
      }
      off = off == (T::STAGES - 1) * T::TILE ? 0u : off + T::TILE;
    }
  };
  if (FP8 && !wide) tiles(std::bool_constant<!FP8>{});
  else tiles(std::true_type{});
  wait_vmcnt<0>();  // no DMA may land in LDS after the wave has ended

  // the new token's own key: its weight, and what it leaves of the others'
  float left = 1.f, own = 0.f;
  if (has_new) {
    const float m_new = fmaxf(m_run, x_own);
    left = __builtin_amdgcn_exp2f(m_run - m_new);
    own = __builtin_amdgcn_exp2f(x_own - m_new);
    m_run = m_new;
  }
  const float l_tot = fmaf(row_sum(l_run), left, own);

  // O through LDS: a lane then holds PER consecutive values of a row.  Row `col` of the
  // accumulators is left * O + own * v_new (fp8: O times the largest scale).
  constexpr int ROW = D + 4;  // floats; the shift by 16 bytes spreads the columns over the banks
  static_assert(16 * ROW * 4 <= T::STAGES * T::TILE, "O fits the stages");
  float* const sh_o = reinterpret_cast<float*>(lds);
  if (row_ok) {
#pragma unroll
    for (int b = 0; b < T::DB; ++b)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4)
        *reinterpret_cast<f32x4*>(sh_o + col * ROW + 32 * b + 8 * q4 + 4 * h) =
            f32x4{o[b][4 * q4], o[b][4 * q4 + 1], o[b][4 * q4 + 2], o[b][4 * q4 + 3]};
  }
  if (h == 0) {
    sh_row[0][col] = l_tot;
    sh_row[1][col] = left;
    sh_row[2][col] = own;
  }
  __syncthreads();  // (one wave)
  fvec vn;
#pragma unroll
  for (int e = 0; e < PER; ++e) vn[e] = __uint_as_float(uint32_t(v_own[e]) << 16);
  auto row = [&](int rc) -> fvec {
    const fvec x = *reinterpret_cast<const fvec*>(sh_o + rc * ROW + d0);
    return x * (sh_row[1][rc] * vs_max) + vn * sh_row[2][rc];
  };
  if (it.part >= 0) {  // unnormalised partials, merged by the combine kernels
    if (row_ok && h == 0)
      *reinterpret_cast<f32x2*>(p.part_ml + (size_t(it.part) * p.part_rows + col) * 2) = f32x2{m_run, l_tot};
#pragma unroll 1
    for (int gi = 0; gi < G; ++gi)
      *reinterpret_cast<fvec*>(static_cast<float*>(p.part_o) + (size_t(it.part) * p.part_rows + gi) * D + d0) = row(gi);
    return;
  }
#pragma unroll 1
  for (int gi = 0; gi < G; ++gi) {
    const float l = sh_row[0][gi];
    const fvec x = row(gi) * (l == 0.f ? 0.f : 1.f / l);  // (a token that sees nothing: 0)
    hvec y;
#pragma unroll
    for (int e = 0; e < PER; ++e) y[e] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(x[e]));
    *reinterpret_cast<hvec*>(static_cast<uint16_t*>(p.out) + (size_t(tok) * hq + size_t(kvh) * G + gi) * D + d0) = y;
  }
  if (p.lse != nullptr && row_ok && h == 0)
    p.lse[size_t(tok) * hq + size_t(kvh) * G + col] = (m_run + __log2f(l_tot)) * kLn2;
}

template <int D, bool FP8, bool CAP>
hipError_t launch_t(const ShapedParams& p, hipStream_t stream, const ArgPlanBuf* ap) {
  const dim3 grid(p.a.n_items), block(64);
  if (ap != nullptr && ap->small())
    hipLaunchKernelGGL((shaped_decode_kernel<D, FP8, CAP, kPlanInSmallArgs>), grid, block, 0, stream, p, ap->small_plan());
  else if (ap != nullptr)
    hipLaunchKernelGGL((shaped_decode_kernel<D, FP8, CAP, kPlanInArgs>), grid, block, 0, stream, p, ap->plan);
  else
    hipLaunchKernelGGL((shaped_decode_kernel<D, FP8, CAP, kPlanInMemory>), grid, block, 0, stream, p, NoArgPlan{});
  return hipGetLastError();
}

}  // namespace

int shaped_decode_keys_per_tile() { return kKeys; }

int shaped_decode_waves_per_cu(int head_dim, bool fp8) {  // 160 KB of LDS per CU
  return (160 * 1024) / (stages(head_dim, fp8) * tile_bytes(head_dim, fp8));
}

hipError_t launch_shaped_decode(const ShapedParams& p, int head_dim, bool fp8, hipStream_t stream, const ArgPlanBuf* ap) {
  if (p.a.n_items <= 0) return hipSuccess;
  const bool cap = p.cap2 > 0.f;
#define CW_CASE(D_)                                                                                        \
  if (head_dim == D_) {                                                                                    \
    if (fp8) return cap ? launch_t<D_, true, true>(p, stream, ap) : launch_t<D_, true, false>(p, stream, ap); \
    return cap ? launch_t<D_, false, true>(p, stream, ap) : launch_t<D_, false, false>(p, stream, ap);     \
  }
  CW_CASE(64)
  CW_CASE(128)
#undef CW_CASE
  return hipErrorInvalidValue;
}

}  // namespace cw
