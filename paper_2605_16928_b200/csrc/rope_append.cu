// Rotary position embedding on the way into the cache: queries rotated to a dense buffer, keys rotated and values copied to
// their pages (bf16 or 4-bit, main or local pool), index keys projected from the unrotated keys, in one launch.
//
// Channels (a, b) of a pair i at position p become (a c - b s, b c + a s) with c, s = scale * cos, sin(p f_i).  The angle is
// formed in turns and reduced in 64 bits (twice, so that positions up to 2^31 keep their angles), its sine and cosine
// are 32-bit; products and sums are 32-bit and rounded once to bf16.  A 4-bit cache holds the quantised bf16 row, as
// rtp_kv_append would have it from a caller that rotates by itself.
//
// Bound by the bytes of the rows (a read and a write each).  Eight threads own a (token, head) row: a thread holds two 16-byte
// chunks that are each other's partners (c and c + rotary_dim / 16 of the half split), so that a pair never leaves its thread and
// every access is 16 bytes wide.  Rows of a token lie next to each other in the grid, so a block forms the angles and looks up
// the pages of the few tokens that it holds once, while its rows are on their way.
#include "kv4.cuh"

namespace rtp {

namespace {

constexpr int kThreads = 256;
constexpr int kRowsAtOnce = kThreads / 8;
constexpr int kProjTokens = 16;
constexpr double kInvTwoPi = 0.15915494309189535, kInvTwoPiLow = -9.839338337591243e-18;   // 1 / (2 pi) as a sum

struct RopeArgs {
  const double* freqs;
  int32_t half;          // rotated pairs
  int32_t interleaved;
  float scale;
  const __nv_bfloat16 *q, *k, *v, *w_k;
  int64_t q_stride, k_stride, v_stride;   // elements from a token to the next
  __nv_bfloat16* q_out;
  const int32_t *tok_seq, *tok_pos;
  int32_t T, n_q, n_kv, rows_per_tok;     // rows of a token: query heads, keys, values
  int32_t proj_blocks;                    // blocks in front of the others that project index keys
  int32_t* status;
};

// Page of a token in a pool, or -1 if the row is not to be written.
__device__ __forceinline__ int page_for(const CacheView& cv, int seq, int pos) {
  if (seq < 0 || seq >= cv.batch || pos < 0 || pos >= cv.cap_tokens) return -1;
  const int phys = __ldg(cv.block_table + (int64_t)seq * cv.max_pages + page_entry(cv, pos >> kPageShift));
  return phys >= 0 && phys < cv.num_pages && page_writable(cv, phys) ? phys : -1;
}

// Index keys of 16 tokens of one index head: thread (t, j) owns output j of token t, 128 products in channel order, as
// rtp_index_keys forms them.
__device__ __forceinline__ void project_block(const CacheView& cv, const HeadMaps& hm, const RopeArgs& a, unsigned char* smem) {
  float* ws = reinterpret_cast<float*>(smem);
  __nv_bfloat16* xs = reinterpret_cast<__nv_bfloat16*>(smem + kHeadDim * kIndexDim * 4);
  const int tid = threadIdx.x, head = blockIdx.x % cv.n_ih, t0 = (int)(blockIdx.x / cv.n_ih) * kProjTokens;
  const int r = tid >> 4, c = tid & 15, t = t0 + r;
  {
    const uint4 w = ld_nc_v4(a.w_k + (int64_t)head * kHeadDim * kIndexDim + tid * 8);
    uint4 x = make_uint4(0, 0, 0, 0);
    if (t < a.T) x = ld_nc_v4(a.k + (int64_t)t * a.k_stride + hm.ih_kv[head] * kHeadDim + c * 8);
    const __nv_bfloat162* p = reinterpret_cast<const __nv_bfloat162*>(&w);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __bfloat1622float2(p[i]);
      ws[tid * 8 + 2 * i] = f.x;
      ws[tid * 8 + 2 * i + 1] = f.y;
    }
    *reinterpret_cast<uint4*>(xs + r * kHeadDim + c * 8) = x;
  }
  __syncthreads();
  float acc = 0.f;
#pragma unroll 16
  for (int i = 0; i < kHeadDim; ++i) acc = fmaf(__bfloat162float(xs[r * kHeadDim + i]), ws[i * kIndexDim + c], acc);
  if (t >= a.T) return;
  const int pos = a.tok_pos[t], phys = page_for(cv, a.tok_seq[t], pos);   // (index keys live in the main pool)
  if (phys < 0) return;
  const int64_t at = (((int64_t)phys * cv.n_ih + head) * kPage + (pos & (kPage - 1))) * kIndexDim + c;
  if (cv.ikey_fp8)
    reinterpret_cast<uint8_t*>(cv.ikey)[at] = (uint8_t)__nv_cvt_float_to_fp8(acc, __NV_SATFINITE, __NV_E4M3);
  else
    cv.ikey[at] = __float2bfloat16_rn(acc);
}

__device__ __forceinline__ uint32_t pack2(float x, float y) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(x, y);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// PASSES: rows of a block / 32.
template <int PASSES>
__global__ void __launch_bounds__(kThreads) rope_append_kernel(const __grid_constant__ CacheView cv, const __grid_constant__ CacheView lv,
                                                               const __grid_constant__ HeadMaps hm, const __grid_constant__ RopeArgs a) {
  chain_wait();
  constexpr int kRows = PASSES * kRowsAtOnce;
  constexpr int kToks = kRows / 2 + 1;             // (a token has a key and a value row at least)
  constexpr int kTable = kToks * kHeadDim / 2 * 8, kProj = kHeadDim * kIndexDim * 4 + kProjTokens * kHeadDim * 2;
  __shared__ __align__(16) unsigned char smem[kTable > kProj ? kTable : kProj];
  __shared__ int s_page[kToks], s_local[kToks], s_pos[kToks];
  if ((int)blockIdx.x < a.proj_blocks) {
    project_block(cv, hm, a, smem);
    return;
  }
  const int tid = threadIdx.x, j = tid & 7;
  const unsigned row0 = (blockIdx.x - a.proj_blocks) * kRows, n_rows = (unsigned)a.T * a.rows_per_tok;
  const unsigned t0 = row0 / a.rows_per_tok, t1 = (min(row0 + kRows, n_rows) - 1) / a.rows_per_tok;
  const int n_tok = (int)(t1 - t0) + 1;
  // the thread's two chunks of a row: partners where the row is rotated, neighbours elsewhere
  const int hc = a.half >> 3;                      // 16-byte chunks of half the rotated channels
  const int pair_a = a.interleaved || j >= hc ? 2 * j : j, pair_b = a.interleaved || j >= hc ? pair_a + 1 : j + hc;
  uint4 xa[PASSES], xb[PASSES];
  int tok[PASSES], head[PASSES];                   // head: query heads, then keys, then values; -1: no row
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const unsigned row = row0 + p * kRowsAtOnce + (tid >> 3);
    head[p] = -1;
    tok[p] = 0;
    if (row < n_rows) {
      const unsigned t = row / a.rows_per_tok;
      int h = (int)(row - t * a.rows_per_tok);
      if (!a.q) h += a.n_q;
      tok[p] = (int)(t - t0);
      head[p] = h;
      const __nv_bfloat16* src = h < a.n_q ? a.q + (int64_t)t * a.q_stride + h * kHeadDim
                                 : h < a.n_q + a.n_kv ? a.k + (int64_t)t * a.k_stride + (h - a.n_q) * kHeadDim
                                                      : a.v + (int64_t)t * a.v_stride + (h - a.n_q - a.n_kv) * kHeadDim;
      const bool rot = h < a.n_q + a.n_kv;
      // (a plain load: the queries may be rotated in place)
      xa[p] = *reinterpret_cast<const uint4*>(src + (rot ? pair_a : 2 * j) * 8);
      xb[p] = *reinterpret_cast<const uint4*>(src + (rot ? pair_b : 2 * j + 1) * 8);
    }
  }
  float2* table = reinterpret_cast<float2*>(smem);
  for (int i = tid; i < n_tok; i += kThreads) {
    const int seq = a.tok_seq[t0 + i], pos = a.tok_pos[t0 + i];
    const int main_page = cv.n_kv > 0 ? page_for(cv, seq, pos) : 0, local_page = lv.n_kv > 0 ? page_for(lv, seq, pos) : 0;
    if (main_page < 0 || local_page < 0) set_status(a.status, RTP_ERR_INVALID);
    s_page[i] = main_page;
    s_local[i] = local_page;
    s_pos[i] = pos;
  }
  for (int i = tid; i < n_tok * a.half; i += kThreads) {
    const int t = i / a.half, f = i - t * a.half;
    // p f / 2 pi as a sum of two: whole turns go, and what the first one's rounding lost comes back
    const double pos = (double)a.tok_pos[t0 + t], fr = a.freqs[f];
    const double g = fr * kInvTwoPi, g_low = fma(fr, kInvTwoPi, -g) + fr * kInvTwoPiLow;
    const double turns = pos * g, rest = fma(pos, g, -turns) + pos * g_low;
    float s, c;
    sincospif((float)(2.0 * ((turns - rint(turns)) + rest)), &s, &c);
    table[t * a.half + f] = make_float2(c * a.scale, s * a.scale);
  }
  __syncthreads();
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int h = head[p];
    if (h >= 0 && h < a.n_q + a.n_kv) {
      const float2* cs = table + tok[p] * a.half;
      uint32_t* wa = reinterpret_cast<uint32_t*>(&xa[p]);
      uint32_t* wb = reinterpret_cast<uint32_t*>(&xb[p]);
      if (a.interleaved) {
        if (j < (a.half >> 3)) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 u = cs[j * 8 + e], w = cs[j * 8 + 4 + e];
            const float ax = low(wa[e]), ay = high(wa[e]), bx = low(wb[e]), by = high(wb[e]);
            wa[e] = pack2(fmaf(ax, u.x, -(ay * u.y)), fmaf(ay, u.x, ax * u.y));
            wb[e] = pack2(fmaf(bx, w.x, -(by * w.y)), fmaf(by, w.x, bx * w.y));
          }
        }
      } else if (j < hc) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 u = cs[j * 8 + 2 * e], w = cs[j * 8 + 2 * e + 1];
          const float ax = low(wa[e]), ay = high(wa[e]), bx = low(wb[e]), by = high(wb[e]);
          wa[e] = pack2(fmaf(ax, u.x, -(bx * u.y)), fmaf(ay, w.x, -(by * w.y)));
          wb[e] = pack2(fmaf(bx, u.x, ax * u.y), fmaf(by, w.x, ay * w.y));
        }
      }
    }
    if (h >= 0 && h < a.n_q) {
      __nv_bfloat16* dst = a.q_out + ((int64_t)(t0 + tok[p]) * a.n_q + h) * kHeadDim;
      *reinterpret_cast<uint4*>(dst + pair_a * 8) = xa[p];
      *reinterpret_cast<uint4*>(dst + pair_b * 8) = xb[p];
    }
  }
  // keys and values
  const bool fp4 = cv.kv_fp4;
  if (fp4) __syncthreads();                        // (the angles are no longer read: their place takes rows)
#pragma unroll
  for (int p = 0; p < PASSES; ++p) {
    const int h = head[p] - a.n_q;                 // keys, then values
    const bool is_v = h >= a.n_kv;
    const int kvh = is_v ? h - a.n_kv : h;
    int64_t row = -1;
    bool local = false;
    if (head[p] >= a.n_q) {
      local = cv.kv_slot[kvh] == 0xff;             // (the head lives in the other pool)
      const CacheView& v = local ? lv : cv;
      const int phys = local ? s_local[tok[p]] : s_page[tok[p]];
      if (phys >= 0) row = ((int64_t)phys * v.n_kv + v.kv_slot[kvh]) * kPage + (s_pos[tok[p]] & (kPage - 1));
    }
    const int ca = is_v ? 2 * j : pair_a, cb = is_v ? 2 * j + 1 : pair_b;
    if (!fp4) {
      if (row >= 0) {
        const CacheView& v = local ? lv : cv;
        __nv_bfloat16* dst = const_cast<__nv_bfloat16*>(is_v ? v.v : v.k) + row * kHeadDim;
        *reinterpret_cast<uint4*>(dst + ca * 8) = xa[p];
        *reinterpret_cast<uint4*>(dst + cb * 8) = xb[p];
      }
    } else {   // the row through shared memory, so that a thread has the 16 channels of one scale
      uint4* st = reinterpret_cast<uint4*>(smem) + (tid >> 3) * 16;
      __syncwarp();
      st[ca] = xa[p];
      st[cb] = xb[p];
      __syncwarp();
      const uint4 lo = st[2 * j], hi = st[2 * j + 1];
      if (row >= 0) {
        const CacheView& v = local ? lv : cv;
        uint32_t scale;
        bool bad = false;
        const uint2 codes = kv4_encode(lo, hi, scale, bad);
        if (bad) set_status(a.status, RTP_ERR_UNSUPPORTED);
        uint8_t* pages = const_cast<uint8_t*>(reinterpret_cast<const uint8_t*>(is_v ? v.v : v.k));
        *reinterpret_cast<uint2*>(pages + row * kKv4TokBytes + j * 8) = codes;
        const_cast<uint8_t*>(v.kv_scales)[row * kKv4ScaleBytes + (is_v ? 8 : 0) + j] = (uint8_t)scale;
      }
    }
  }
}

}  // namespace

cudaError_t launch_rope_append(const CacheView& cv, const CacheView& lv, const Dims& d, const HeadMaps& hm, const double* freqs,
                               int rotary_dim, bool interleaved, float scale, const __nv_bfloat16* q, int64_t q_stride,
                               const __nv_bfloat16* k, int64_t k_stride, const __nv_bfloat16* v, int64_t v_stride,
                               __nv_bfloat16* q_out, const __nv_bfloat16* w_k, const int32_t* tok_seq, const int32_t* tok_pos,
                               int64_t T, int32_t* status, cudaStream_t st) {
  if (T == 0) return cudaSuccess;
  RopeArgs a = {freqs, rotary_dim / 2, interleaved, scale, q, k, v, w_k, q_stride, k_stride, v_stride, q_out, tok_seq, tok_pos,
                (int32_t)T, d.n_q, d.n_kv, (q ? d.n_q : 0) + 2 * d.n_kv, 0, status};
  a.proj_blocks = w_k ? (int)((T + kProjTokens - 1) / kProjTokens) * d.n_ih : 0;
  const int64_t rows = T * a.rows_per_tok;
  // four passes a block (fewer angles a row, more loads in flight) where two waves of such blocks are there, else one
  const bool many = rows >= (int64_t)2 * 4 * kRowsAtOnce * current_sm_count(148);
  const int per = (many ? 4 : 1) * kRowsAtOnce;
  const dim3 grid((unsigned)(a.proj_blocks + (rows + per - 1) / per));
  (void)launch_chained(many ? rope_append_kernel<4> : rope_append_kernel<1>, grid, dim3(kThreads), 0, st, cv, lv, hm, a);
  return cudaGetLastError();
}

}  // namespace rtp
