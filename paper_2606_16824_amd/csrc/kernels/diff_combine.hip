// Merge of differential attention's split-K partials: for each query pair and map, O_m =
// sum w_c O_c / sum w_c l_c with w_c = 2^(m_c - max m), then the difference of the maps,
// the norm and the store.  Fixed order, no atomics.
//
// A row's 2 D values lie over one wave; WPR waves share its partials (four where there are
// many: decodes of long prefixes) and meet in LDS.  Each wave issues the loads of kBatch
// partials of both maps before it uses them.  Bound by reading the partials (fp32: the
// difference cancels, so they are not rounded on the way): 67 MB of a 1024-token chunk's in
// 14.8 us, 4.5 TB/s; of one decode of 1700 keys 4.6 us, mostly latency, of 48 over fp8 pages 8.2.
#include <hip/hip_runtime.h>

#include "../cw_internal.h"
#include "../plan_expand.h"
#include "diff_common.h"

namespace cw {
namespace {

using namespace diff;

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kBatch = 4;
constexpr int kFewParts = 4;  // up to this many partials per row a wave merges a row alone

template <int AP>
__device__ __forceinline__ CombineGroup group_of(const ExtendParams& p, const PlanArg<AP>& ap, int grp) {
  if constexpr (AP != kPlanInMemory) {
    if (p.ap_desc > 0) {  // a decode plan in compact form: the group is rebuilt (each wave searches)
      const ExpandDesc& d = *reinterpret_cast<const ExpandDesc*>(ap.bytes + p.ap_desc);
      const DecodeRec* rec = reinterpret_cast<const DecodeRec*>(ap.bytes + d.rec_off);
      const int b = wave_last_at_most(d.n_seqs, grp, static_cast<int>(threadIdx.x % 64),
                                      [&](int k) { return rec[k].group_off; });
      return expand_group_at(rec, grp, b, d.rows);
    }
  }
  return plan_ptr<AP>(ap, p.ap_groups, p.groups)[grp];
}

template <int D, int WPR, int AP>
__global__ __launch_bounds__(kThreads) void diff_combine_kernel(DiffParams dp, PlanArg<AP> ap) {
  constexpr int PER = 2 * D / 64;        // values per lane
  constexpr int ROWS = kWaves / WPR;     // rows per workgroup
  typedef float vec __attribute__((ext_vector_type(PER)));
  __shared__ float sh_o[2][kWaves][2 * D];
  __shared__ float sh_m[2][kWaves], sh_l[2][kWaves];
  const ExtendParams& p = dp.a;
  const int half_rows = p.part_rows / 2;
  const int wgs_per_group = (half_rows + ROWS - 1) / ROWS;
  const CombineGroup cg = group_of<AP>(p, ap, blockIdx.x / wgs_per_group);
  const int lane = threadIdx.x % 64;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int lr = (blockIdx.x % wgs_per_group) * ROWS + wave / WPR;
  if (lr >= cg.rows) return;  // (where waves meet at a barrier, uniform over the workgroup: ROWS is 1)
  const int d0 = lane * PER;
  float m[2] = {-INFINITY, -INFINITY}, L[2] = {0.f, 0.f};
  vec acc[2] = {vec(0.f), vec(0.f)};
  for (int c0 = wave % WPR; c0 < cg.n_parts; c0 += kBatch * WPR) {
    f32x2 ml[2][kBatch];
    vec oc[2][kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k)
#pragma unroll
      for (int mp = 0; mp < 2; ++mp) {
        const int c = c0 + k * WPR;
        ml[mp][k] = f32x2{-INFINITY, 0.f};
        oc[mp][k] = vec(0.f);
        if (c < cg.n_parts) {
          const size_t slot = size_t(cg.part0 + c) * p.part_rows + mp * half_rows + lr;
          ml[mp][k] = *reinterpret_cast<const f32x2*>(p.part_ml + slot * 2);
          oc[mp][k] = *reinterpret_cast<const vec*>(static_cast<const float*>(p.part_o) + slot * (2 * D) + d0);
        }
      }
#pragma unroll
    for (int mp = 0; mp < 2; ++mp) {
      float m_new = m[mp];
#pragma unroll
      for (int k = 0; k < kBatch; ++k) m_new = fmaxf(m_new, ml[mp][k].x);
      const float a = __builtin_amdgcn_exp2f(m[mp] - m_new);
      L[mp] *= a;
      acc[mp] *= a;
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const float w = c0 + k * WPR < cg.n_parts ? __builtin_amdgcn_exp2f(ml[mp][k].x - m_new) : 0.f;
        L[mp] = fmaf(w, ml[mp][k].y, L[mp]);
        acc[mp] += w * oc[mp][k];
      }
      m[mp] = m_new;
    }
  }
  if constexpr (WPR > 1) {
#pragma unroll
    for (int mp = 0; mp < 2; ++mp) {
#pragma unroll
      for (int e = 0; e < PER; ++e) sh_o[mp][wave][d0 + e] = acc[mp][e];
      if (lane == 0) {
        sh_m[mp][wave] = m[mp];
        sh_l[mp][wave] = L[mp];
      }
    }
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int mp = 0; mp < 2; ++mp) {
      m[mp] = -INFINITY;
      L[mp] = 0.f;
      acc[mp] = vec(0.f);
#pragma unroll
      for (int w = 0; w < WPR; ++w) m[mp] = fmaxf(m[mp], sh_m[mp][w]);
#pragma unroll
      for (int w = 0; w < WPR; ++w) {
        const float f = sh_m[mp][w] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sh_m[mp][w] - m[mp]);
        L[mp] = fmaf(f, sh_l[mp][w], L[mp]);
#pragma unroll
        for (int e = 0; e < PER; ++e) acc[mp][e] = fmaf(f, sh_o[mp][w][d0 + e], acc[mp][e]);
      }
    }
  }
  const SeqInfo sq = plan_ptr<AP>(ap, p.ap_seqs, p.seqs)[cg.seq];
  const int G = p.gqa_group, hp = p.num_kv_heads * G;
  const int r = cg.q_row0 + lr;
  const int t = r / G, g = r - t * G;
  const int head = cg.kvh * G + g;
  const float f0 = 1.f / L[0], f1 = dp.lam[head] / L[1];
  float o[PER], ss = 0.f;
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    o[e] = acc[0][e] * f0 - acc[1][e] * f1;
    ss = fmaf(o[e], o[e], ss);
  }
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) ss += __shfl_xor(ss, x);
  const float f = row_factor(dp, ss, D);
  uint16_t* orow = static_cast<uint16_t*>(p.out) + (size_t(sq.cu + t) * hp + head) * (2 * D) + d0;
  typedef uint16_t half_vec __attribute__((ext_vector_type(PER)));
  half_vec out;
#pragma unroll
  for (int e = 0; e < PER; ++e) {
    const float w = dp.weight == nullptr ? 1.f : dp.weight[d0 + e];
    out[e] = __builtin_bit_cast(uint16_t, static_cast<__bf16>(o[e] * f * w));
  }
  *reinterpret_cast<half_vec*>(orow) = out;
}

template <int D, int WPR>
hipError_t launch_t(const DiffParams& p, hipStream_t stream, const ArgPlanBuf* ap) {
  constexpr int ROWS = kWaves / WPR;
  const dim3 grid(p.a.n_groups * ((p.a.part_rows / 2 + ROWS - 1) / ROWS)), block(kThreads);
  if (ap != nullptr && ap->small())
    hipLaunchKernelGGL((diff_combine_kernel<D, WPR, kPlanInSmallArgs>), grid, block, 0, stream, p, ap->small_plan());
  else if (ap != nullptr)
    hipLaunchKernelGGL((diff_combine_kernel<D, WPR, kPlanInArgs>), grid, block, 0, stream, p, ap->plan);
  else
    hipLaunchKernelGGL((diff_combine_kernel<D, WPR, kPlanInMemory>), grid, block, 0, stream, p, NoArgPlan{});
  return hipGetLastError();
}

}  // namespace

hipError_t launch_diff_combine(const DiffParams& p, int head_dim, int max_parts, hipStream_t stream,
                               const ArgPlanBuf* ap) {
  if (p.a.n_groups <= 0) return hipSuccess;
  const bool many = max_parts > kFewParts;
  if (head_dim == 64) return many ? launch_t<64, kWaves>(p, stream, ap) : launch_t<64, 1>(p, stream, ap);
  if (head_dim == 128) return many ? launch_t<128, kWaves>(p, stream, ap) : launch_t<128, 1>(p, stream, ap);
  return hipErrorInvalidValue;
}

}  // namespace cw
