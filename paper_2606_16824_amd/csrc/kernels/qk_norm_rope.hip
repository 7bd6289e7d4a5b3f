// RMS norm of every query and key head with the position rotation, in one pass, and with
// pools the page write of the new K/V.
//
//   y = x / sqrt(mean(x^2) + eps) * w  (no weights: y = x), then for each rotated pair
//   (a, b) of y, with the position's cos and sin: (a cos - b sin, b cos + a sin)
//   pairs: elements i and i + R / 2, or 2 i and 2 i + 1 (interleaved), of the first R.
//
// All in fp32 with one rounding to bf16; the pools get what k_out and v_out hold (fp8:
// quantised from the bf16 values as the page write does), so a pool written here is the
// one that the page write of k_out and v_out makes.
//
// Bound by memory: q, k and v are read and written once, in 16-byte pieces; D / 8 lanes
// hold a head, so a wave works on 64 / (D / 8) heads at a time.  A wave keeps its token's
// angles times the weights in registers over all heads that it takes (64 bytes of them
// per 16 bytes of a head: read for each head they took a third of the loads), and issues
// the loads of kBatch heads of each lane before it uses them.  GPU time of one token (32 + 8 +
// 8 heads of 128, bf16 pages) 3.6 us, of 16384 tokens 95 us (5.0 TB/s; a plain copy moves 4.9),
// with fp8 pages 93, of 1531 tokens of 64 + 8 heads without pages 14.8 us.  With three axes a
// lane's pairs of one axis are still read in 16-byte pieces: one token 4.6 us, 16384 tokens 95 us (96 where
// neighbouring pairs follow different axes and are read one by one).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "../cw_internal.h"
#include "page_write.h"

namespace cw {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kThreads = 256;
constexpr int kBatch = 4;  // heads of a lane whose loads are in flight together
constexpr int64_t kSplitWaves = 4096;

__device__ __forceinline__ float bf16_at(u32x4 x, int e) {
  return __uint_as_float(e % 2 ? x[e / 2] & 0xFFFF0000u : x[e / 2] << 16);
}

// Eight consecutive floats from 16-byte-aligned memory.
__device__ __forceinline__ void load8(float (&f)[8], const float* src) {
  const f32x4 a = *reinterpret_cast<const f32x4*>(src), b = *reinterpret_cast<const f32x4*>(src + 4);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    f[e] = a[e];
    f[4 + e] = b[e];
  }
}

// POOL: 0 no page write, 1 bf16 pools, 2 fp8 pools.  AXES: a token has a position for each of
// several axes, and each rotated pair follows one of them.
template <int D, bool INTER, int POOL, bool AXES>
__global__ __launch_bounds__(kThreads) void qk_norm_rope_kernel(NormRopeParams p) {
  constexpr int CH = D / 8;        // lanes per head
  constexpr int RPW = 64 / CH;     // heads per wave and step
  const int lane = threadIdx.x % 64;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int c = lane % CH;         // piece of the head: elements 8 c .. 8 c + 7
  const int item = static_cast<int>(blockIdx.x) * (kThreads / 64) + wave;
  const int tok = item / p.splits;
  if (tok >= p.num_tokens) return;
  const int pos = p.positions[tok];
  bool outside = pos < 0 || pos >= p.num_positions;
  int axis_pos[4] = {pos, pos, pos, pos};
  if constexpr (AXES) {
#pragma unroll
    for (int a = 1; a < 4; ++a) {
      if (a < p.num_axes) axis_pos[a] = p.positions[int64_t(a) * p.num_tokens + tok];
      outside |= axis_pos[a] < 0 || axis_pos[a] >= p.num_positions;
    }
  }
  if (outside) return;  // a padding token: nothing of it is written
  const int heads = p.hq + p.hkv + (p.v != nullptr ? p.hkv : 0);
  const int steps = (heads + RPW - 1) / RPW;
  const int per = (steps + p.splits - 1) / p.splits;
  const int s0 = (item % p.splits) * per, s1 = min(s0 + per, steps);

  // this lane's angles, and for pairs i, i + R / 2 the lane that holds the other half: element
  // e becomes r (x[e] w[e] cs[e] + x[other] w[other] sn[e]); lanes behind the rotated
  // elements have cs = 1 and nothing to add
  const int half = p.rot / 2;
  const bool turns = 8 * c < p.rot;
  float cs[8], sn[8];
  int partner = c;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    cs[e] = 1.f;
    sn[e] = 0.f;
  }
  if (turns) {
    const float* row = p.cos_sin + size_t(pos) * p.rot;
    if constexpr (AXES) {
      // the axes of this lane's pairs (four or eight in a row), two bits each; pairs of one
      // axis are read together
      constexpr int PAIRS = INTER ? 4 : 8;
      const bool first = INTER || 8 * c < half;
      const int at = INTER ? 4 * c : first ? 8 * c : 8 * c - half;
      const uint32_t word = at < 16 ? p.axis_of[0] : at < 32 ? p.axis_of[1] : at < 48 ? p.axis_of[2] : p.axis_of[3];
      const uint32_t axes = word >> (2 * (at % 16)) & ((1u << (2 * PAIRS)) - 1);
      auto row_of = [&](uint32_t a) {
        const int at_pos = a == 0 ? axis_pos[0] : a == 1 ? axis_pos[1] : a == 2 ? axis_pos[2] : axis_pos[3];
        return p.cos_sin + size_t(at_pos) * p.rot;
      };
      float cv[8], sv[8];
      if (axes == (axes & 3) * (0x5555u & ((1u << (2 * PAIRS)) - 1))) {
        const float* src = row_of(axes & 3);
#pragma unroll
        for (int e = 0; e < PAIRS; e += 4) {
          const f32x4 a = *reinterpret_cast<const f32x4*>(src + at + e), b = *reinterpret_cast<const f32x4*>(src + half + at + e);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            cv[e + i] = a[i];
            sv[e + i] = b[i];
          }
        }
      } else {
#pragma unroll
        for (int e = 0; e < PAIRS; ++e) {
          const float* src = row_of(axes >> (2 * e) & 3);
          cv[e] = src[at + e];
          sv[e] = src[half + at + e];
        }
      }
      if constexpr (!INTER) partner = first ? c + half / 8 : c - half / 8;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        cs[e] = cv[INTER ? e / 2 : e];
        const float s = sv[INTER ? e / 2 : e];
        sn[e] = (INTER ? e % 2 != 0 : !first) ? s : -s;
      }
    } else if constexpr (INTER) {
      const f32x4 a = *reinterpret_cast<const f32x4*>(row + 4 * c), b = *reinterpret_cast<const f32x4*>(row + half + 4 * c);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        cs[e] = a[e / 2];
        sn[e] = e % 2 ? b[e / 2] : -b[e / 2];
      }
    } else {
      const bool first = 8 * c < half;  // of its pairs
      const int at = first ? 8 * c : 8 * c - half;
      load8(cs, row + at);
      load8(sn, row + half + at);
      partner = first ? c + half / 8 : c - half / 8;
#pragma unroll
      for (int e = 0; e < 8; ++e) sn[e] = first ? -sn[e] : sn[e];
    }
  }
  const int64_t slot = POOL != 0 ? p.slots[tok] : -1;
  const bool paged = POOL != 0 && slot >= 0 && slot < int64_t(p.num_pages) * p.page_size;
  const int64_t page = paged ? slot / p.page_size : 0;
  const int in_page = paged ? static_cast<int>(slot % p.page_size) : 0;

  // the factors of x[e] and of its partner for this lane's kind of head
  float fa[8], fb[8];
  int kind = -1;  // 0 a query head, 1 a key head, 2 a value head
  bool norm = false;
  auto kind_of = [&](int hd) { return hd < p.hq ? 0 : hd < p.hq + p.hkv ? 1 : 2; };

  for (int sb = s0; sb < s1; sb += kBatch) {
    u32x4 xs[kBatch];
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int hd = (sb + u) * RPW + lane / CH;
      xs[u] = u32x4{0u, 0u, 0u, 0u};
      if (sb + u < s1 && hd < heads) {
        const int kd = kind_of(hd);
        const int h = kd == 0 ? hd : kd == 1 ? hd - p.hq : hd - p.hq - p.hkv;
        const uint16_t* src = static_cast<const uint16_t*>(kd == 0 ? p.q : kd == 1 ? p.k : p.v) +
                              tok * (kd == 0 ? p.q_stride : kd == 1 ? p.k_stride : p.v_stride) + h * D + 8 * c;
        xs[u] = *reinterpret_cast<const u32x4*>(src);
      }
    }
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      if (sb + u >= s1) break;  // (uniform)
      const int hd = (sb + u) * RPW + lane / CH;
      const int kd = kind_of(hd);
      const int h = kd == 0 ? hd : kd == 1 ? hd - p.hq : hd - p.hq - p.hkv;
      if (__any(kd != kind)) {  // (once or twice per token: another kind's weights)
        kind = kd;
        const float* w = kd == 0 ? p.q_weight : p.k_weight;
        norm = w != nullptr && kd < 2;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          fa[e] = cs[e];
          fb[e] = sn[e];
        }
        if (norm) {
          float wt[8], wo[8];
          load8(wt, w + 8 * c);
          load8(wo, w + 8 * partner);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            fa[e] *= wt[e];
            fb[e] *= INTER ? wt[e ^ 1] : wo[e];
          }
        }
      }
      const u32x4 x = xs[u];
      float r = 1.f;
      {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(bf16_at(x, e), bf16_at(x, e), ss);
#pragma unroll
        for (int m = 1; m < CH; m <<= 1) ss += __shfl_xor(ss, m);
        if (norm) r = 1.f / sqrtf(ss * (1.f / D) + p.eps);
      }
      u32x4 other = x;  // what the partner elements are read from
      if constexpr (!INTER) {
#pragma unroll
        for (int e = 0; e < 4; ++e) other[e] = __shfl(x[e], (lane & ~(CH - 1)) | partner);
      }
      if (!turns) other = u32x4{0u, 0u, 0u, 0u};
      u32x4 y = x;
      if (kd < 2) {
        bf16x8 o;
#pragma unroll
        for (int e = 0; e < 8; ++e)
          o[e] = static_cast<__bf16>((bf16_at(x, e) * fa[e] + bf16_at(other, INTER ? e ^ 1 : e) * fb[e]) * r);
        y = __builtin_bit_cast(u32x4, o);
      }
      if (hd >= heads) continue;
      uint16_t* out = static_cast<uint16_t*>(kd == 0 ? p.q_out : kd == 1 ? p.k_out : p.v_out);
      if (out != nullptr)
        *reinterpret_cast<u32x4*>(out + (int64_t(tok) * (kd == 0 ? p.hq : p.hkv) + h) * D + 8 * c) = y;
      if (POOL != 0 && paged && kd != 0) {
        const int64_t at = ((page * p.hkv + h) * p.page_size + in_page) * D + 8 * c;
        void* pool = kd == 1 ? p.k_pool : p.v_pool;
        if constexpr (POOL == 2) {
          const float sc = (kd == 1 ? p.k_scale : p.v_scale)[page * p.hkv + h];
          *reinterpret_cast<pw::u32x2*>(static_cast<uint8_t*>(pool) + at) = pw::quantise8(y, sc);
        } else {
          *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(pool) + at) = y;
        }
      }
    }
  }
}

template <int D, bool INTER, bool AXES>
hipError_t launch_t(const NormRopeParams& p, int pool, hipStream_t stream) {
  constexpr int kWaves = kThreads / 64;
  const int64_t items = int64_t(p.num_tokens) * p.splits;
  const dim3 grid(static_cast<unsigned>((items + kWaves - 1) / kWaves));
  if (pool == 0) hipLaunchKernelGGL((qk_norm_rope_kernel<D, INTER, 0, AXES>), grid, dim3(kThreads), 0, stream, p);
  else if (pool == 1) hipLaunchKernelGGL((qk_norm_rope_kernel<D, INTER, 1, AXES>), grid, dim3(kThreads), 0, stream, p);
  else hipLaunchKernelGGL((qk_norm_rope_kernel<D, INTER, 2, AXES>), grid, dim3(kThreads), 0, stream, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_qk_norm_rope(NormRopeParams p, int head_dim, bool interleaved, int pool, hipStream_t stream) {
  if (p.num_tokens <= 0) return hipSuccess;
  // Few tokens: their heads spread over more waves (up to one step each, kSplitWaves in all).  Each
  // wave reads its token's angles anew: in a graph, 32 + 8 + 8 heads of 128 with bf16 pages, with up to
  // 2048, 4096, 8192 and 16384 waves 256 tokens take 4.9, 4.7, 4.7, 4.7 us, 512 6.2, 6.1, 6.9,
  // 6.9, 1024 9.0, 8.6, 10.0, 10.4, 2048 15.5, 14.0, 15.1, 17.1; up to 128 tokens are alike.
  const int rpw = 64 / (head_dim / 8);
  const int steps = (p.hq + p.hkv + (p.v != nullptr ? p.hkv : 0) + rpw - 1) / rpw;
  p.splits = static_cast<int32_t>(std::max<int64_t>(1, std::min<int64_t>(steps, kSplitWaves / p.num_tokens)));
#define CW_CASE(D_, AXES_) \
  if (head_dim == D_ && (p.num_axes > 0) == AXES_) \
    return interleaved ? launch_t<D_, true, AXES_>(p, pool, stream) : launch_t<D_, false, AXES_>(p, pool, stream);
  CW_CASE(64, false)
  CW_CASE(128, false)
  CW_CASE(64, true)
  CW_CASE(128, true)
#undef CW_CASE
  return hipErrorInvalidValue;
}

}  // namespace cw
