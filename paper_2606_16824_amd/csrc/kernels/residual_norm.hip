// The norm of a block's output, its gate, the scaled residual stream and the next block's norm
// in one pass.
//
//   u = x / sqrt(mean(x^2) + eps) * w_post   (no post weight: u = x)
//   r' = s r + gate u                        (no gate: s r + u)
//   y = r' / sqrt(mean(r'^2) + eps) * w_pre  (no pre weight: no y)
//
// All in fp32; r' is rounded once where it is stored and y is taken from it before that.
//
// Bound by memory: x and r are read once and r' and y written once, 16 bytes per lane at a time
// (fp32 residual: twice 16).  A row stays in registers from its first read to its last write: a
// wave holds rows of up to 2048 elements, four waves longer ones.  A workgroup keeps the
// weights and a gate of all tokens in registers over the rows that it takes (read for each row
// they would be as many bytes again as a row's).
//
// 16384 rows of 4096 bf16 elements: 0.54 GB in 105 us (5.1 TB/s); one row 3.2 us; an fp32 stream 155 us
// (5.2), a gate for each token 131 (5.1).  Rows above 8192 elements hold 321 to 352 registers, one wave per
// SIMD, so that no row's loads fly beside another's sums: 4096 rows of 16384 141 us (3.8 TB/s), fp32 173 (4.6).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "../cw_internal.h"

namespace cw {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kThreads = 256, kWavesPerWg = kThreads / 64;
constexpr int kWaveRow = 2048;  // elements of a row up to which a wave holds it

struct F8 {
  float v[8];
};
__device__ __forceinline__ F8 widen(u32x4 x) {
  F8 f;
#pragma unroll
  for (int e = 0; e < 8; ++e) f.v[e] = __uint_as_float(e % 2 ? x[e / 2] & 0xFFFF0000u : x[e / 2] << 16);
  return f;
}
__device__ __forceinline__ u32x4 load_bf16(const void* base, int64_t at) {
  return *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(base) + at);
}
__device__ __forceinline__ F8 load_f32(const float* src) {
  const f32x4 a = *reinterpret_cast<const f32x4*>(src), b = *reinterpret_cast<const f32x4*>(src + 4);
  return F8{{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]}};
}
__device__ __forceinline__ void store_bf16(void* base, int64_t at, const F8& f) {
  bf16x8 o;
#pragma unroll
  for (int e = 0; e < 8; ++e) o[e] = static_cast<__bf16>(f.v[e]);
  *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(base) + at) = __builtin_bit_cast(u32x4, o);
}
// Eight elements of a residual row as they are stored.
template <bool WIDE>
struct Stored {
  u32x4 w[WIDE ? 2 : 1];
  __device__ __forceinline__ void load(const void* base, int64_t at) {
    const u32x4* src = reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(base) + at * (WIDE ? 4 : 2));
    w[0] = src[0];
    if constexpr (WIDE) w[1] = src[1];
  }
  __device__ __forceinline__ F8 get() const {
    if constexpr (!WIDE) return widen(w[0]);
    F8 f;
#pragma unroll
    for (int e = 0; e < 8; ++e) f.v[e] = __uint_as_float(w[WIDE ? e / 4 : 0][e % 4]);
    return f;
  }
};

// A row's sum over the lanes that hold it (`rows` per workgroup: a wave each, or all waves one).
template <bool WAVE>
__device__ __forceinline__ float row_total(float x, float* sh) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) x += __shfl_xor(x, d);
  if constexpr (!WAVE) {
    if (threadIdx.x % 64 == 0) sh[threadIdx.x / 64] = x;
    __syncthreads();
    x = (sh[0] + sh[1]) + (sh[2] + sh[3]);
  }
  return x;
}

// K: pieces of 8 elements per lane.  WAVE: a wave holds a row.  WIDE: the residual is fp32.
template <int K, bool WAVE, bool WIDE>
__global__ __launch_bounds__(kThreads) void residual_norm_kernel(ResidualNormParams p) {
  constexpr int LANES = WAVE ? 64 : kThreads;
  __shared__ float sh[4][kWavesPerWg];
  const int lane = threadIdx.x % LANES;
  const int n = p.width;
  const float inv_n = 1.f / static_cast<float>(n);
  int at[K];
  bool ok[K];
  F8 post[K], pre[K], gate[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    at[k] = (k * LANES + lane) * 8;
    ok[k] = at[k] < n;
    post[k] = pre[k] = gate[k] = F8{{1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f}};
    if (!ok[k]) continue;
    if (p.post_weight != nullptr) post[k] = load_f32(p.post_weight + at[k]);
    if (p.pre_weight != nullptr) pre[k] = load_f32(p.pre_weight + at[k]);
    if (p.gate != nullptr && p.gate_stride == 0) gate[k] = widen(load_bf16(p.gate, at[k]));
  }
  const int first = WAVE ? static_cast<int>(blockIdx.x) * kWavesPerWg + static_cast<int>(threadIdx.x / 64) : static_cast<int>(blockIdx.x);
  const int step = WAVE ? static_cast<int>(gridDim.x) * kWavesPerWg : static_cast<int>(gridDim.x);
  // (the words of a sum are written again two rows later: one barrier at least lies between any
  // two rows' sums, so every wave has read them by then)
  int slot = 0;
  for (int64_t row = first; row < p.num_tokens; row += step, slot ^= 2) {
    u32x4 xs[K];
    Stored<WIDE> rs[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
      xs[k] = u32x4{0u, 0u, 0u, 0u};
      rs[k] = Stored<WIDE>{};
      if (!ok[k]) continue;
      xs[k] = load_bf16(p.x, row * p.x_stride + at[k]);
      rs[k].load(p.residual, row * n + at[k]);
      if (p.gate != nullptr && p.gate_stride != 0) gate[k] = widen(load_bf16(p.gate, row * p.gate_stride + at[k]));
    }
    F8 r[K];
    float f = 1.f;
    if (p.post_weight != nullptr) {  // (uniform)
      float ss = 0.f;
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const F8 x = widen(xs[k]);
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = fmaf(x.v[e], x.v[e], ss);
      }
      f = 1.f / sqrtf(row_total<WAVE>(ss, sh[slot]) * inv_n + p.eps);
    }
    float ss = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const F8 x = widen(xs[k]), old = rs[k].get();
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        r[k].v[e] = fmaf(p.scale, old.v[e], x.v[e] * f * post[k].v[e] * gate[k].v[e]);
        ss = fmaf(r[k].v[e], r[k].v[e], ss);
      }
      if (!ok[k]) continue;
      if constexpr (WIDE) {
        float* out = static_cast<float*>(p.residual_out) + row * n + at[k];
        *reinterpret_cast<f32x4*>(out) = f32x4{r[k].v[0], r[k].v[1], r[k].v[2], r[k].v[3]};
        *reinterpret_cast<f32x4*>(out + 4) = f32x4{r[k].v[4], r[k].v[5], r[k].v[6], r[k].v[7]};
      } else {
        store_bf16(p.residual_out, row * n + at[k], r[k]);
      }
    }
    if (p.pre_weight == nullptr) continue;  // (uniform)
    const float fy = 1.f / sqrtf(row_total<WAVE>(ss, sh[slot + 1]) * inv_n + p.eps);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      if (!ok[k]) continue;
      F8 y;
#pragma unroll
      for (int e = 0; e < 8; ++e) y.v[e] = r[k].v[e] * fy * pre[k].v[e];
      store_bf16(p.y_out, row * n + at[k], y);
    }
  }
}

template <int K, bool WAVE>
hipError_t launch_t(const ResidualNormParams& p, bool wide, hipStream_t stream) {
  const int64_t wgs = WAVE ? (int64_t(p.num_tokens) + kWavesPerWg - 1) / kWavesPerWg : p.num_tokens;
  const dim3 grid(static_cast<unsigned>(std::min<int64_t>(wgs, 2048)));
  if (wide) hipLaunchKernelGGL((residual_norm_kernel<K, WAVE, true>), grid, dim3(kThreads), 0, stream, p);
  else hipLaunchKernelGGL((residual_norm_kernel<K, WAVE, false>), grid, dim3(kThreads), 0, stream, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_residual_norm(const ResidualNormParams& p, bool wide, hipStream_t stream) {
  if (p.num_tokens <= 0) return hipSuccess;
  if (p.width <= kWaveRow) {
    const int k = (p.width + 511) / 512;
    if (k <= 1) return launch_t<1, true>(p, wide, stream);
    if (k <= 2) return launch_t<2, true>(p, wide, stream);
    return launch_t<4, true>(p, wide, stream);
  }
  const int k = (p.width + 2047) / 2048;
  if (k <= 2) return launch_t<2, false>(p, wide, stream);
  if (k <= 3) return launch_t<3, false>(p, wide, stream);
  if (k <= 4) return launch_t<4, false>(p, wide, stream);
  return launch_t<8, false>(p, wide, stream);
}

}  // namespace cw
