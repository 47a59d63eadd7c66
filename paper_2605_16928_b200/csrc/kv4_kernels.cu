// The write side of the 4-bit K/V cache and its expansion to bf16 pages.  Both are streams without reuse, bound by the
// bytes they move.  Append: a thread owns one group of 16 channels, so that the group's maximum needs no exchange between
// lanes; 16 neighbouring threads are the 8 groups of K and the 8 of V of one (token, head), whose codes are two runs of 64
// bytes and whose scales are one run of 16.  Expansion: a thread owns eight channels, 16 bytes of output, so that a warp
// writes 512 bytes in a row; a block does one (page, head).  Measured: 8192 tokens x 8 heads appended in 13.6 us (43 MB; latency
// of the token -> table -> row chain), 128K tokens x 8 heads expanded in 107 us (688 MB, 6.4 TB/s, the rate of a plain copy).
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
  chain_wait();
  uint8_t* kp = const_cast<uint8_t*>(reinterpret_cast<const uint8_t*>(cv.k));
  uint8_t* vp = const_cast<uint8_t*>(reinterpret_cast<const uint8_t*>(cv.v));
  uint8_t* sp = const_cast<uint8_t*>(cv.kv_scales);
  // (fewer than 2^31 (token, head) rows: checked by the caller)
  const unsigned n_rows = (unsigned)T * n_src_heads;
  const int grp = threadIdx.x % kGroupsPerRow, g = grp & (kGroupsPerRow / 2 - 1);
  const bool is_v = grp >= kGroupsPerRow / 2;
  for (unsigned i = blockIdx.x * (kThreads / kGroupsPerRow) + threadIdx.x / kGroupsPerRow; i < n_rows;
       i += gridDim.x * (kThreads / kGroupsPerRow)) {
    // the rows are requested before it is looked up where they go
    const __nv_bfloat16* src = (is_v ? v_new : k_new) + (int64_t)i * kHeadDim + g * kKv4Group;
    const uint4 lo = ld_stream_v4(src), hi = ld_stream_v4(src + 8);
    const unsigned t = i / n_src_heads;
    const int slot = cv.kv_slot[i % n_src_heads];
    const int seq = __ldg(tok_seq + t), pos = __ldg(tok_pos + t);
    if (slot == 0xff) continue;   // the head lives in the other pool
    if (seq < 0 || seq >= cv.batch || pos < 0 || pos >= cv.cap_tokens) {
      set_status(status, RTP_ERR_INVALID);
      continue;
    }
    const int phys = __ldg(cv.block_table + (int64_t)seq * cv.max_pages + page_entry(cv, pos >> kPageShift));
    if (phys < 0 || phys >= cv.num_pages || !page_writable(cv, phys)) {
      set_status(status, RTP_ERR_INVALID);
      continue;
    }
    uint32_t scale;
    bool bad = false;
    const uint2 codes = kv4_encode(lo, hi, scale, bad);
    if (bad) set_status(status, RTP_ERR_UNSUPPORTED);
    const int64_t row = ((int64_t)phys * cv.n_kv + slot) * kPage + (pos & (kPage - 1));
    *reinterpret_cast<uint2*>((is_v ? vp : kp) + row * kKv4TokBytes + g * 8) = codes;
    sp[row * kKv4ScaleBytes + grp] = (uint8_t)scale;
  }
}

__global__ void __launch_bounds__(kThreads) kv4_expand_kernel(const __grid_constant__ CacheView cv,
                                                              const int32_t* __restrict__ src_pages,
                                                              const int32_t* __restrict__ dst_pages, uint4* __restrict__ k_out,
                                                              uint4* __restrict__ v_out, const int n_out_pages, int32_t* status) {
  chain_wait();
  constexpr int kChunks = kHeadDim / 8;                     // 16-byte pieces of an expanded row
  constexpr int kSteps = kPage * kChunks / kThreads;
  const unsigned p = blockIdx.x / cv.n_kv, head = blockIdx.x % cv.n_kv;
  const int src = src_pages[p], dst = dst_pages ? dst_pages[p] : (int)p;
  if (src < 0 || src >= cv.num_pages || dst < 0 || dst >= n_out_pages) {
    if (threadIdx.x == 0) set_status(status, RTP_ERR_INVALID);
    return;
  }
  const int64_t row = ((int64_t)src * cv.n_kv + head) * kPage, row_out = ((int64_t)dst * cv.n_kv + head) * kPage;
  const uint32_t* codes[2] = {reinterpret_cast<const uint32_t*>(cv.k) + row * (kKv4TokBytes / 4),
                              reinterpret_cast<const uint32_t*>(cv.v) + row * (kKv4TokBytes / 4)};
  const uint8_t* scales = cv.kv_scales + row * kKv4ScaleBytes;
  uint32_t w[2][kSteps];
  float s[2][kSteps];
#pragma unroll
  for (int x = 0; x < 2; ++x)
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
      const int i = j * kThreads + threadIdx.x;             // token i / 16, piece i % 16
      w[x][j] = __ldg(codes[x] + i);
      s[x][j] = kv4_scale_value(__ldg(scales + (i / kChunks) * kKv4ScaleBytes + x * (kKv4ScaleBytes / 2) + (i % kChunks) / 2));
    }
#pragma unroll
  for (int x = 0; x < 2; ++x)
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
      uint32_t h[4];
      e2m1x8_to_f16x2(w[x][j], h);
#pragma unroll
      for (int k = 0; k < 4; ++k) {   // (six significant bits: the rounding to bf16 drops nothing)
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[k]));
        const __nv_bfloat162 o = __floats2bfloat162_rn(f.x * s[x][j], f.y * s[x][j]);
        h[k] = *reinterpret_cast<const uint32_t*>(&o);
      }
      (x ? v_out : k_out)[row_out * kChunks + j * kThreads + threadIdx.x] = make_uint4(h[0], h[1], h[2], h[3]);
    }
}

}  // namespace

cudaError_t launch_kv4_append(const CacheView& cv, int n_src_heads, const __nv_bfloat16* k_new, const __nv_bfloat16* v_new,
                              const int32_t* tok_seq, const int32_t* tok_pos, int64_t T, int32_t* status,
                              cudaStream_t st) {
  if (T == 0) return cudaSuccess;
  int64_t blocks = (T * n_src_heads * kGroupsPerRow + kThreads - 1) / kThreads;
  blocks = std::min<int64_t>(blocks, (int64_t)current_sm_count(148) * 32);
  (void)launch_chained(kv4_append_kernel, dim3((unsigned)blocks), dim3(kThreads), 0, st, cv, n_src_heads, k_new, v_new, tok_seq,
                       tok_pos, T, status);
  return cudaGetLastError();
}

cudaError_t launch_kv4_expand(const CacheView& cv, const int32_t* src_pages, const int32_t* dst_pages, int64_t n, void* k_out,
                              void* v_out, int32_t n_out_pages, int32_t* status, cudaStream_t st) {
  if (n == 0 || cv.n_kv == 0) return cudaSuccess;
  (void)launch_chained(kv4_expand_kernel, dim3((unsigned)(n * cv.n_kv)), dim3(kThreads), 0, st, cv, src_pages, dst_pages,
                       reinterpret_cast<uint4*>(k_out), reinterpret_cast<uint4*>(v_out), n_out_pages, status);
  return cudaGetLastError();
}

}  // namespace rtp
