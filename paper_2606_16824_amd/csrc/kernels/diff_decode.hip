// Differential attention of single new tokens over a paged cache, HBM-streaming.
//
// Work item = one wave: the G <= 16 query pairs of one key pair against a chunk of at most
// 64 pages of one sequence's prefix, plus the new token's own key when the chunk ends the
// sequence.  Every cached K/V byte is read once, so the kernel is bound by HBM.
//
// Both maps share the accumulators: columns 0-15 of the 32 of an MFMA are the first map's
// queries, columns 16-31 the second's.  K1 [Q1 | Q2] and K2 [Q1 | Q2] are both taken and
// each lane keeps its map's (the others cost matrix cycles, which a streaming kernel has
// to spare); one softmax pass then serves both maps, and O^T += V^T P^T multiplies both
// maps' weights with a value row read once.
//
// A tile is 32 keys: rows of both key heads and both value halves, DMA'd into LDS by
// global_load_lds_dwordx4 with the kernel's own vmcnt waits (see the decode kernel, whose
// pipeline this is).  Bytes in flight per CU decide: 32 KB tiles (D = 128, bf16) in two
// stages and two waves per CU, smaller ones in three stages and three or six waves:
// 128-144 KB of LDS.  fp8 pools keep their codes in LDS and are widened exactly (keys to
// bf16, values to fp16 or bf16); a page's K scale of each map multiplies that map's scores, the V
// scales of the two halves multiply the weights (one set of weights per half).
//
// In a graph, 48 decodes of 2k-32k keys, 4 key pairs of 128: over 16-token pages bf16 604 us (5.7
// TB/s of K/V; a plain copy moves 4.9), fp8 336 us (5.1), over 64-token pages 561 and 296; 8
// pairs of 64: 598 and 323, over 64-token pages 550 and 314.  One decode of 131072 keys: 100 us
// bf16, 64 us fp8; of 1700 keys 12.8 us, its two launches, the page ids' and the tiles'
// latencies, and 1.7 us per tile.
#include <hip/hip_runtime.h>

#include <type_traits>

#include "../cw_internal.h"
#include "../plan_expand.h"
#include "diff_common.h"

namespace cw {
namespace {

using namespace diff;

constexpr int kScalarSearchSeqs = 8;  // up to here an item's sequence is searched by scalar loads
constexpr int kKeys = 32;             // keys of a tile
// Up to this ratio of a chunk's V scales, their products with the weights are held in fp16: a
// column's largest weight is at least 2^kHeadroom, its product at least 1, and what fp16 drops of
// any other (2^-25) at most 2^-25 of that.  Further apart (one page's scale may be far above the
// others', without any weight on it) they are pairs of bf16: 48 decodes of 2k-32k keys 329 -> 346
// us at D = 128, 314 -> 326 at 64.  A scale of 0 is far from any other: all of the large weights may
// be its page's, and the products that are left below 2^-25.
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
__device__ __forceinline__ f16x2 fp8x2_f16x2(uint32_t v) {
  return __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(static_cast<int>(v), 1.0f, HI);
}
__device__ __forceinline__ f16x8 fp8x8_f16x8(u32x2 c) {
  const u32x4 r = {__builtin_bit_cast(uint32_t, fp8x2_f16x2<false>(c.x)), __builtin_bit_cast(uint32_t, fp8x2_f16x2<true>(c.x)),
                   __builtin_bit_cast(uint32_t, fp8x2_f16x2<false>(c.y)), __builtin_bit_cast(uint32_t, fp8x2_f16x2<true>(c.y))};
  return __builtin_bit_cast(f16x8, r);
}

__host__ __device__ constexpr int tile_bytes(int d, bool fp8) { return 4 * kKeys * d * (fp8 ? 1 : 2); }
__host__ __device__ constexpr int stages(int d, bool fp8) { return tile_bytes(d, fp8) > 16384 ? 2 : 3; }

template <int D, int P, bool FP8>
struct Geo {
  static constexpr int RB = D * (FP8 ? 1 : 2);      // bytes per row
  static constexpr int MAT = kKeys * RB;            // bytes of one matrix of a tile: K1, K2, Va, Vb
  static constexpr int TILE = 4 * MAT;
  static constexpr int STAGES = stages(D, FP8);
  static constexpr int CPR = RB / 16;               // 16-byte chunks per row
  static constexpr int RPI = 64 / CPR;              // rows per DMA instruction
  static constexpr int NI = kKeys / RPI;            // DMA instructions per matrix
  static constexpr int DMA = 4 * NI;                // per tile
  static constexpr int KT = D / 16;                 // k-steps of K Q^T
  static constexpr int DB = D / 32;                 // 32-row blocks of O^T per value half
  static constexpr int VB = 2 * DB;
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

template <int D, int P, bool FP8, int AP>
__global__ __launch_bounds__(64) void diff_decode_kernel(DiffParams dp, PlanArg<AP> ap) {
  using T = Geo<D, P, FP8>;
  const ExtendParams& p = dp.a;
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
  const int h = lane >> 5, col = lane & 31;
  const int map = col >> 4, g = col & 15;  // this lane's column: a map and a query pair
  const int G = p.gqa_group, hkv = 2 * p.num_kv_heads, hp = p.num_kv_heads * G;
  const int pair = it.kvh;
  const int lp = sq.lp;
  const int tok = sq.cu;  // the sequence's single new token
  const int32_t* bt = p.block_table + size_t(sq.bt_row) * p.bt_stride;
  const uint8_t* k_pool = static_cast<const uint8_t*>(p.k_pool);
  const uint8_t* v_pool = static_cast<const uint8_t*>(p.v_pool);
  const bool row_ok = g < G;

  // prefix keys of this item: [kb, ke); the new key when kv_end passes lp
  const int kb = it.kv_begin;
  const int ke = min(it.kv_end, lp);
  const bool has_new = it.kv_end > lp;
  const int n_tiles = ke > kb ? (ke - kb + kKeys - 1) / kKeys : 0;

  // page ids (and fp8 scales) of the chunk: lane j holds page kb / P + j
  const int page0 = kb / P;
  const int n_pages = ke > kb ? (ke - 1) / P - page0 + 1 : 0;
  int my_pg = 0;
  float my_ks[2] = {1.f, 1.f}, my_vs[2] = {1.f, 1.f};
  if (lane < n_pages) {
    my_pg = bt[page0 + lane];
    if constexpr (FP8) {
      const size_t si = size_t(my_pg) * hkv + 2 * pair;
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        my_ks[m] = p.k_scale[si + m];
        my_vs[m] = p.v_scale[si + m];
      }
    }
  }
  // Q^T (B operand): this column's query.  bf16 pools: k-step kk holds dims 16 kk + 8 h + e;
  // fp8 pools read 16 dims per fragment, so k-steps 2 t and 2 t + 1 hold dims 32 t + 16 h +
  // 8 (kk & 1) + e.  And the new token's key, and what each lane needs at the end (values
  // lane * PER on of a row), read here so that their latency does not end the item.
  auto dim0 = [&](int kk) { return FP8 ? 32 * (kk >> 1) + 16 * h + 8 * (kk & 1) : 16 * kk + 8 * h; };
  bf16x8 qf[T::KT];
  {
    const uint16_t* qrow =
        static_cast<const uint16_t*>(p.q) + (2 * (size_t(tok) * hp + size_t(pair) * G + g) + map) * D;
#pragma unroll
    for (int kk = 0; kk < T::KT; ++kk) {
      u32x4 v = {0u, 0u, 0u, 0u};
      if (row_ok) v = *reinterpret_cast<const u32x4*>(qrow + dim0(kk));
      qf[kk] = __builtin_bit_cast(bf16x8, v);
    }
  }
  bf16x8 k_own[T::KT];
  constexpr int PER = 2 * D / 64;
  typedef float fvec __attribute__((ext_vector_type(PER)));
  typedef uint16_t hvec __attribute__((ext_vector_type(PER)));
  const int d0 = lane * PER;
  hvec v_own = hvec(0);
  fvec wt = fvec(1.f);
  if (has_new) {
    const uint16_t* kn = static_cast<const uint16_t*>(p.k_new) + (size_t(tok) * hkv + 2 * pair + map) * D;
#pragma unroll
    for (int kk = 0; kk < T::KT; ++kk) k_own[kk] = *reinterpret_cast<const bf16x8*>(kn + dim0(kk));
    v_own = *reinterpret_cast<const hvec*>(static_cast<const uint16_t*>(p.v_new) + (size_t(tok) * hkv + 2 * pair) * D + d0);
  }
  if (it.part < 0 && dp.weight != nullptr) wt = *reinterpret_cast<const fvec*>(dp.weight + d0);

  // DMA of tile t: instruction j of a matrix covers tile rows [j RPI, (j + 1) RPI); rows past
  // the chunk's prefix end fetch its last key again (their scores are masked), so every tile
  // issues exactly DMA instructions and the wait counts below are exact.
  const int dma_row = lane / T::CPR, dma_pos = lane % T::CPR;
  auto issue_tile = [&](int t, uint32_t dst) __attribute__((always_inline)) {
    const int j0 = kb + t * kKeys;
#pragma unroll
    for (int j = 0; j < T::NI; ++j) {
      const int R = j * T::RPI + dma_row;
      const int key = min(j0 + R, ke - 1);
      const int r0 = min(j0 + j * T::RPI, ke - 1);  // (uniform)
      const int pg = __builtin_amdgcn_readlane(my_pg, min(r0 / P - page0, 63));
      const size_t base = (size_t(pg) * hkv + 2 * pair) * P * T::RB + size_t(key % P) * T::RB;
      const uint32_t kc = 16 * (dma_pos ^ k_swz<T::RB>(R));
      const uint32_t vc = 16 * (dma_pos ^ (FP8 ? v_swz8<T::RB>(R) : v_swz16<T::RB>(R)));
#pragma unroll
      for (int m = 0; m < 2; ++m) {
        dma16(k_pool + base + m * (P * T::RB) + kc, dst + m * T::MAT + j * T::RPI * T::RB);
        dma16(v_pool + base + m * (P * T::RB) + vc, dst + (2 + m) * T::MAT + j * T::RPI * T::RB);
      }
    }
  };

  f32x16 o[T::VB];
#pragma unroll
  for (int b = 0; b < T::VB; ++b) o[b] = f32x16{};
  float m_run = kNegBig, l_run = 0.f;
  const float c = p.scale_log2;

  // Q, the new token's rows and the page ids land first (the addresses need the ids), so
  // only DMA is outstanding in the loop
  __builtin_amdgcn_s_waitcnt((7 << 4) | (15 << 8));
  const uint32_t lds_base = lds_addr(lds);
#pragma unroll 1
  for (int t = 0; t < min(n_tiles, T::STAGES); ++t) issue_tile(t, lds_base + t * T::TILE);
  // fp8: each half's largest V scale of the chunk is taken out of the weights (and multiplied
  // back at the end), so that fp16 holds them whatever the scales' size; `wide`: they lie further
  // apart than kNearScales, and weights times scales keep fp32's range.
  float vs_max[2] = {1.f, 1.f};
  bool wide = false;
  if constexpr (FP8) {
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      const float x = lane < n_pages ? fabsf(my_vs[m]) : 0.f;
      vs_max[m] = x;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) vs_max[m] = fmaxf(vs_max[m], __shfl_xor(vs_max[m], d));
      wide |= __any(lane < n_pages && x * kNearScales < vs_max[m]);
    }
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      if (wide || vs_max[m] == 0.f) vs_max[m] = 1.f;
      my_vs[m] = lane < n_pages ? my_vs[m] / vs_max[m] : 0.f;  // (a tile's end may lie behind the pages)
    }
  }
  float x_own = 0.f;  // the new token's score, under the first tiles' latency
  if (has_new) {
#pragma unroll
    for (int kk = 0; kk < T::KT; ++kk)
#pragma unroll
      for (int e = 0; e < 8; ++e) x_own = fmaf(static_cast<float>(qf[kk][e]), static_cast<float>(k_own[kk][e]), x_own);
    x_own = row_sum(x_own) * c;
  }

  // TWO: how the weights are given to the second product (below)
  auto compute = [&](int t, const uint8_t* st, auto two) __attribute__((always_inline)) {
    constexpr bool TWO = decltype(two)::value;
    const int j0 = kb + t * kKeys;
    f32x16 s = f32x16{}, s2 = f32x16{};
    const int R = swap_bits_2_3(col);  // row m of the block reads key swap(m)
    const uint8_t* km = st + R * T::RB;
    if constexpr (FP8) {
#pragma unroll
      for (int t2 = 0; t2 < T::KT / 2; ++t2) {
        const uint8_t* at = km + 16 * ((2 * t2 + h) ^ k_swz<T::RB>(R));
        const u32x4 r0 = *reinterpret_cast<const u32x4*>(at), r1 = *reinterpret_cast<const u32x4*>(at + T::MAT);
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fp8x8_bf16x8(u32x2{r0.x, r0.y}), qf[2 * t2], s, 0, 0, 0);
        s2 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fp8x8_bf16x8(u32x2{r1.x, r1.y}), qf[2 * t2], s2, 0, 0, 0);
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fp8x8_bf16x8(u32x2{r0.z, r0.w}), qf[2 * t2 + 1], s, 0, 0, 0);
        s2 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fp8x8_bf16x8(u32x2{r1.z, r1.w}), qf[2 * t2 + 1], s2, 0, 0, 0);
      }
    } else {
      // fragments are read four (two k-steps of both maps) ahead of their products (left to
      // the compiler each waited for its own read: 48 decodes over bf16 pages, with the
      // values' fragments ahead too, 615 -> 581 us, of 1700 keys 14.8 -> 12.7 us)
      bf16x8 kf[2][4];
      auto read4 = [&](int g2, bf16x8(&f)[4]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          f[i] = *reinterpret_cast<const bf16x8*>(km + 16 * ((2 * (2 * g2 + (i >> 1)) + h) ^ k_swz<T::RB>(R)) + (i & 1) * T::MAT);
      };
      read4(0, kf[0]);
#pragma unroll
      for (int g2 = 0; g2 < T::KT / 2; ++g2) {
        if (g2 + 1 < T::KT / 2) read4(g2 + 1, kf[(g2 + 1) & 1]);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          f32x16& acc = i & 1 ? s2 : s;
          acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[g2 & 1][i], qf[2 * g2 + (i >> 1)], acc, 0, 0, 0);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = map == 0 ? s[i] : s2[i];
    // element i holds key j0 + 16 (i / 8) + 8 h + i % 8; the keys of half-group i / 8 share a page
    float cg[2] = {c, c}, vs[2][2] = {{1.f, 1.f}, {1.f, 1.f}};
    if constexpr (FP8) {
#pragma unroll
      for (int s8 = 0; s8 < 2; ++s8) {
        const int q = min((j0 + 16 * s8) / P - page0, 63);
        const float k0 = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(my_ks[0]), q));
        const float k1 = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(my_ks[1]), q));
        cg[s8] = c * (map == 0 ? k0 : k1);
#pragma unroll
        for (int m = 0; m < 2; ++m) vs[s8][m] = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(my_vs[m]), q));
      }
    }
    if (j0 + kKeys > ke) {  // keys past the chunk's prefix end
      // (the page scales first: a page's may be 0, and then -inf times it is no mask)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        if constexpr (FP8) s[i] *= cg[i >> 3];
        if (j0 + 16 * (i >> 3) + 8 * h + (i & 7) >= ke) s[i] = -INFINITY;
      }
      if constexpr (FP8) cg[0] = cg[1] = 1.f;
    }
    // weights against the running max as it stands; raised only when a half-column's sum
    // passes kSumLimit (or is not finite, as on an item's first tile)
    float w[16], tsum;
    auto weights = [&]() __attribute__((always_inline)) {
      tsum = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        w[i] = __builtin_amdgcn_exp2f(fmaf(s[i], cg[i >> 3], -m_run));
        tsum += w[i];
      }
    };
    weights();
    // (half the limit: a single fp16 weight ends at 65504)
    if (__any(!(tsum <= 0.5f * kSumLimit))) {
      float mx = -INFINITY;
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[i] * cg[i >> 3]);
      mx = row_max(mx) - kHeadroom;
      if (mx > m_run) {
        const float alpha = __builtin_amdgcn_exp2f(m_run - mx);
        m_run = mx;
        l_run *= alpha;
#pragma unroll
        for (int b = 0; b < T::VB; ++b) o[b] *= alpha;
      }
      weights();
    }
    l_run += tsum;
    // O^T += V^T P^T over the tile's two 16-key slices
    const int grp = lane >> 4, ri = lane & 15;
    // Neither form of the weights adds to the output's own rounding.  TWO: a weight is the sum of
    // two bf16 (2^-16), for a second MFMA; else (fp8 pools) fp16 (2^-11), which holds the codes
    // exactly too.  One bf16 weight each: relative error 2.4e-3 instead of 1.7e-3, 1% less time
    // over bf16 pages and none over fp8 pages.  TWO is the item's: a branch in the tile loop made
    // the compiler copy O (48 decodes 368 us).
#pragma unroll
    for (int u = 0; u < 2; ++u) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const uint8_t* vt = st + (2 + half) * T::MAT;
        bf16x8 pf, pl;
        f16x8 ph;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float x = FP8 ? w[8 * u + e] * vs[u][half] : w[8 * u + e];
          if constexpr (TWO) {
            pf[e] = static_cast<__bf16>(x);
            pl[e] = static_cast<__bf16>(x - static_cast<float>(pf[e]));
          } else {
            ph[e] = static_cast<_Float16>(x);
          }
        }
#pragma unroll
        for (int b = 0; b < T::DB; ++b) {
          f32x16& ob = o[half * T::DB + b];
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
            ob = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pf, ob, 0, 0, 0);
            ob = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, pl, ob, 0, 0, 0);
          } else {
            ob = __builtin_amdgcn_mfma_f32_32x32x16_f16(fp8x8_f16x8(codes), ph, ob, 0, 0, 0);
          }
        }
      }
    }
    if constexpr (!FP8) {  // (mask 0x100: LDS reads, 0x008: MFMAs) values' fragments three ahead, fp8 two
      __builtin_amdgcn_sched_group_barrier(0x100, 6, 1);
#pragma unroll
      for (int i = 0; i < 2 * T::VB; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 2, 1);
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 1);
      }
    } else if constexpr (!TWO) {
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 1);
#pragma unroll
      for (int i = 0; i < 2 * T::VB; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 1);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 1);
      }
    }
  };
  // Tile t lives in stage t % STAGES.  A step waits for its tile (those issued after it may
  // still fly), computes on it, then refills the stage if there is a tile for it.  One copy
  // of the code for all stages: a short call runs through it cold, and fetching its
  // instructions is a large part of its time (unrolled by the stages, with O exchanged and
  // the new value added in registers, a decode of one token alone took 13.8 us at D = 128
  // against 6.9, 48 decodes over bf16 pages 635 us against 615).
  auto tiles = [&](auto two) __attribute__((always_inline)) {
    uint32_t off = 0;
#pragma unroll 1
    for (int t = 0; t < n_tiles; ++t) {
      const int behind = n_tiles - 1 - t;
      if (T::STAGES > 2 && behind >= 2) wait_vmcnt<(T::STAGES - 1) * T::DMA>();
      else if (behind >= 1) wait_vmcnt<T::DMA>();
      else wait_vmcnt<0>();
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
  // accumulators is left * O + own * v_new (fp8: O times its half's largest scale).
  constexpr int ROW = 2 * D + 4;  // floats; the shift by 16 bytes spreads the columns over the banks
  static_assert(32 * ROW * 4 <= T::STAGES * T::TILE, "O fits the stages");
  float* const sh_o = reinterpret_cast<float*>(lds);
#pragma unroll
  for (int b = 0; b < T::VB; ++b)
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4)
      *reinterpret_cast<f32x4*>(sh_o + col * ROW + 32 * b + 8 * q4 + 4 * h) =
          f32x4{o[b][4 * q4], o[b][4 * q4 + 1], o[b][4 * q4 + 2], o[b][4 * q4 + 3]};
  if (h == 0) {
    sh_row[0][col] = l_tot;
    sh_row[1][col] = left;
    sh_row[2][col] = own;
  }
  __syncthreads();  // (one wave)
  const float vs_half = vs_max[lane / 32];
  fvec vn;
#pragma unroll
  for (int e = 0; e < PER; ++e) vn[e] = __uint_as_float(uint32_t(v_own[e]) << 16);
  auto row = [&](int rc) -> fvec {
    const fvec x = *reinterpret_cast<const fvec*>(sh_o + rc * ROW + d0);
    return x * (sh_row[1][rc] * vs_half) + vn * sh_row[2][rc];
  };
  if (it.part >= 0) {  // unnormalised partials of both maps, merged by diff_combine
    if (row_ok && h == 0)
      *reinterpret_cast<f32x2*>(p.part_ml + (size_t(it.part) * p.part_rows + map * (p.part_rows / 2) + g) * 2) =
          f32x2{m_run, l_tot};
#pragma unroll 1
    for (int i = 0; i < 2 * G; ++i) {
      const int m = i < G ? 0 : 1, gi = i - m * G;
      const size_t slot = size_t(it.part) * p.part_rows + m * (p.part_rows / 2) + gi;
      *reinterpret_cast<fvec*>(static_cast<float*>(p.part_o) + slot * (2 * D) + d0) = row(16 * m + gi);
    }
    return;
  }
#pragma unroll 1
  for (int gi = 0; gi < G; ++gi) {
    const int head = pair * G + gi;
    const fvec x = row(gi) * (1.f / sh_row[0][gi]) - row(16 + gi) * (dp.lam[head] / sh_row[0][16 + gi]);
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < PER; ++e) ss = fmaf(x[e], x[e], ss);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) ss += __shfl_xor(ss, d);
    const float f = row_factor(dp, ss, D);
    hvec y;
#pragma unroll
    for (int e = 0; e < PER; ++e) y[e] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(x[e] * f * wt[e]));
    *reinterpret_cast<hvec*>(static_cast<uint16_t*>(p.out) + (size_t(tok) * hp + head) * (2 * D) + d0) = y;
  }
}

template <int D, int P, bool FP8>
hipError_t launch_t(const DiffParams& p, hipStream_t stream, const ArgPlanBuf* ap) {
  const dim3 grid(p.a.n_items), block(64);
  if (ap != nullptr && ap->small())
    hipLaunchKernelGGL((diff_decode_kernel<D, P, FP8, kPlanInSmallArgs>), grid, block, 0, stream, p, ap->small_plan());
  else if (ap != nullptr)
    hipLaunchKernelGGL((diff_decode_kernel<D, P, FP8, kPlanInArgs>), grid, block, 0, stream, p, ap->plan);
  else
    hipLaunchKernelGGL((diff_decode_kernel<D, P, FP8, kPlanInMemory>), grid, block, 0, stream, p, NoArgPlan{});
  return hipGetLastError();
}

}  // namespace

int diff_decode_keys_per_tile() { return kKeys; }

int diff_decode_waves_per_cu(int head_dim, bool fp8) {  // 160 KB of LDS per CU
  return (160 * 1024) / (stages(head_dim, fp8) * tile_bytes(head_dim, fp8));
}

hipError_t launch_diff_decode(const DiffParams& p, int head_dim, int page_size, bool fp8, hipStream_t stream,
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
