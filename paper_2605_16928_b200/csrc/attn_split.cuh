// What the decode attention kernels share: the layout of the split partials and their log-sum-exp merge.
#pragma once

#include "rtp_device.cuh"

namespace rtp {

constexpr int kPartial = kHeadDim + 2;                     // acc[128], m, l
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

namespace {

// One CTA per (unit, head of the group): log-sum-exp merge of the split partials.
template <int SET>
__global__ void __launch_bounds__(kHeadDim) attn_merge_kernel(const Dims d, const HeadMaps hm, const int n_units,
                                                              const int G, const float* __restrict__ partial,
                                                              const int n_splits, __nv_bfloat16* __restrict__ out,
                                                              float* __restrict__ lse) {
  chain_wait();
  const int64_t unit = blockIdx.x / G;
  const int g = blockIdx.x % G;
  const int64_t r = unit / n_units;
  const int u = unit % n_units;
  const int qh = (SET == kSetList || SET == kSetPages) ? hm.ret_q_head[u] : hm.kv_list[u] * d.group + g;
  if ((SET == kSetLocal || SET == kSetUnion) && hm.skips(qh)) return;
  const float* p = partial + ((unit * G + g) * (int64_t)n_splits) * kPartial;
  const int dim = threadIdx.x;
  float mt = -INFINITY;
  for (int s = 0; s < n_splits; ++s) mt = fmaxf(mt, p[(int64_t)s * kPartial + kHeadDim]);
  float lt = 0.f, a = 0.f;
  if (mt != -INFINITY) {
    for (int s = 0; s < n_splits; ++s) {
      const float w = fast_ex2(p[(int64_t)s * kPartial + kHeadDim] - mt);
      lt += p[(int64_t)s * kPartial + kHeadDim + 1] * w;
      a += p[(int64_t)s * kPartial + dim] * w;
    }
  }
  const int64_t oh = r * d.n_q + qh;
  out[oh * kHeadDim + dim] = __float2bfloat16_rn(lt > 0.f ? a / lt : 0.f);
  if (lse && dim == 0) lse[oh] = lt > 0.f ? (mt + log2f(lt)) * kLn2 : -INFINITY;
}

}  // namespace

}  // namespace rtp
