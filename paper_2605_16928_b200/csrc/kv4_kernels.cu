// The write side of the 4-bit K/V cache and its expansion to bf16 pages.  Both are streams without reuse, bound by the
// bytes they move: a thread owns one group of 16 channels, so that the group's maximum needs no exchange between lanes;
// 16 neighbouring threads are the 8 groups of K and the 8 of V of one (token, head), whose codes are two runs of 64 bytes
// and whose scales are one run of 16.
#include "kv4.cuh"

namespace rtp {

namespace {

constexpr int kGroupsPerRow = 2 * kHeadDim / kKv4Group;   // K and V groups of a (token, head)
constexpr int kThreads = 256;

// k_new / v_new hold all n_src_heads KV heads of every token; the view stores those with a slot in its pool.
__global__ void __launch_bounds__(kThreads) kv4_append_kernel(const __grid_constant__ CacheView cv, const int n_src_heads,
                                                              const __nv_bfloat16* __restrict__ k_new,
                                                              const __nv_bfloat16* __restrict__ v_new,
                                                              const int32_t* __restrict__ tok_seq,
                                                              const int32_t* __restrict__ tok_pos, const int64_t T,
                                                              int32_t* status) {
  uint8_t* kp = const_cast<uint8_t*>(reinterpret_cast<const uint8_t*>(cv.k));
  uint8_t* vp = const_cast<uint8_t*>(reinterpret_cast<const uint8_t*>(cv.v));
  uint8_t* sp = const_cast<uint8_t*>(cv.kv_scales);
  const int64_t per_tok = (int64_t)n_src_heads * kGroupsPerRow;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < T * per_tok; i += (int64_t)gridDim.x * kThreads) {
    const int64_t t = i / per_tok;
    const int rem = (int)(i % per_tok);
    const int head = rem / kGroupsPerRow, grp = rem % kGroupsPerRow;
    const int slot = cv.kv_slot[head];
    if (slot == 0xff) continue;   // the head lives in the other pool
    const int seq = tok_seq[t], pos = tok_pos[t];
    if (seq < 0 || seq >= cv.batch || pos < 0 || pos >= cv.cap_tokens) {
      set_status(status, RTP_ERR_INVALID);
      continue;
    }
    const int phys = cv.block_table[(int64_t)seq * cv.max_pages + page_entry(cv, pos >> kPageShift)];
    if (phys < 0 || phys >= cv.num_pages) {
      set_status(status, RTP_ERR_INVALID);
      continue;
    }
    const bool is_v = grp >= kGroupsPerRow / 2;
    const int g = grp & (kGroupsPerRow / 2 - 1);
    const __nv_bfloat16* src = (is_v ? v_new : k_new) + (t * n_src_heads + head) * kHeadDim + g * kKv4Group;
    uint32_t scale;
    bool bad = false;
    const uint2 codes = kv4_encode(ld_stream_v4(src), ld_stream_v4(src + 8), scale, bad);
    if (bad) set_status(status, RTP_ERR_UNSUPPORTED);
    const int64_t row = ((int64_t)phys * cv.n_kv + slot) * kPage + (pos & (kPage - 1));
    *reinterpret_cast<uint2*>((is_v ? vp : kp) + row * kKv4TokBytes + g * 8) = codes;
    sp[row * kKv4ScaleBytes + grp] = (uint8_t)scale;
  }
}

__global__ void __launch_bounds__(kThreads) kv4_expand_kernel(const __grid_constant__ CacheView cv,
                                                              const int32_t* __restrict__ src_pages,
                                                              const int32_t* __restrict__ dst_pages, const int64_t n,
                                                              uint4* __restrict__ k_out, uint4* __restrict__ v_out,
                                                              const int n_out_pages, int32_t* status) {
  const int64_t rows_per_page = (int64_t)cv.n_kv * kPage;
  const int64_t per_page = rows_per_page * kGroupsPerRow;
  for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n * per_page; i += (int64_t)gridDim.x * kThreads) {
    const int64_t p = i / per_page;
    const int rem = (int)(i % per_page);
    const int src = src_pages[p];
    const int64_t dst = dst_pages ? dst_pages[p] : p;
    if (src < 0 || src >= cv.num_pages || dst < 0 || dst >= n_out_pages) {
      set_status(status, RTP_ERR_INVALID);
      continue;
    }
    const int grp = rem % kGroupsPerRow, in_page = rem / kGroupsPerRow;
    const bool is_v = grp >= kGroupsPerRow / 2;
    const int g = grp & (kGroupsPerRow / 2 - 1);
    const int64_t row = src * rows_per_page + in_page;
    const uint2 codes = *reinterpret_cast<const uint2*>(reinterpret_cast<const uint8_t*>(is_v ? cv.v : cv.k) + row * kKv4TokBytes + g * 8);
    const float s = kv4_scale_value(cv.kv_scales[row * kKv4ScaleBytes + grp]);
    uint32_t h[8];
    {
      uint32_t a[4], b[4];
      e2m1x8_to_f16x2(codes.x, a);
      e2m1x8_to_f16x2(codes.y, b);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        h[j] = a[j];
        h[4 + j] = b[j];
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {   // (six significant bits: the rounding to bf16 drops nothing)
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[j]));
      const __nv_bfloat162 o = __floats2bfloat162_rn(f.x * s, f.y * s);
      h[j] = *reinterpret_cast<const uint32_t*>(&o);
    }
    uint4* out = (is_v ? v_out : k_out) + (dst * rows_per_page + in_page) * (kHeadDim / 8) + g * 2;
    out[0] = make_uint4(h[0], h[1], h[2], h[3]);
    out[1] = make_uint4(h[4], h[5], h[6], h[7]);
  }
}

}  // namespace

cudaError_t launch_kv4_append(const CacheView& cv, int n_src_heads, const __nv_bfloat16* k_new, const __nv_bfloat16* v_new,
                              const int32_t* tok_seq, const int32_t* tok_pos, int64_t T, int32_t* status,
                              cudaStream_t st) {
  if (T == 0) return cudaSuccess;
  int64_t blocks = (T * n_src_heads * kGroupsPerRow + kThreads - 1) / kThreads;
  blocks = std::min<int64_t>(blocks, (int64_t)current_sm_count(148) * 32);
  kv4_append_kernel<<<(unsigned)blocks, kThreads, 0, st>>>(cv, n_src_heads, k_new, v_new, tok_seq, tok_pos, T, status);
  return cudaGetLastError();
}

cudaError_t launch_kv4_expand(const CacheView& cv, const int32_t* src_pages, const int32_t* dst_pages, int64_t n, void* k_out,
                              void* v_out, int32_t n_out_pages, int32_t* status, cudaStream_t st) {
  if (n == 0 || cv.n_kv == 0) return cudaSuccess;
  int64_t blocks = (n * cv.n_kv * kPage * kGroupsPerRow + kThreads - 1) / kThreads;
  blocks = std::min<int64_t>(blocks, (int64_t)current_sm_count(148) * 32);
  kv4_expand_kernel<<<(unsigned)blocks, kThreads, 0, st>>>(cv, src_pages, dst_pages, n, reinterpret_cast<uint4*>(k_out),
                                                           reinterpret_cast<uint4*>(v_out), n_out_pages, status);
  return cudaGetLastError();
}

}  // namespace rtp
