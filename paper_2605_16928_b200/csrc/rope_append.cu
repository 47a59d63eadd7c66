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
// every access is 16 bytes wide.  Two divisions of the rows among blocks, below.
#include "kv4.cuh"

namespace rtp {

namespace {

constexpr int kThreads = 256;
constexpr int kRowsAtOnce = kThreads / 8;
constexpr int kProjTokens = 16;
constexpr int kProjBytes = kHeadDim * kIndexDim * 4 + kProjTokens * kHeadDim * 2;   // weights and rows of a projection
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

__device__ __forceinline__ uint32_t pack2(float x, float y) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(x, y);
  return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ float low(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// Two products at a time, and two of them with a sum.
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 r;
  asm("{\n.reg .b64 a, b, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmul.rn.f32x2 d, a, b;\nmov.b64 {%0, %1}, d;\n}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 r;
  asm("{\n.reg .b64 a, b, c, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmov.b64 c, {%6, %7};\nfma.rn.f32x2 d, a, b, c;\nmov.b64 {%0, %1}, d;\n}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return r;
}
// Blocks that project lie evenly between those that rotate, next to those with the same tokens: the former compute while the latter
// wait for memory, and find the keys in L2.  Returns the number of projecting blocks in front of block b.
__device__ __forceinline__ int projecting_before(const RopeArgs& a, int64_t b) {
  return a.proj_blocks ? (int)(b * a.proj_blocks / gridDim.x) : 0;
}

// Index keys of 16 tokens of one index head: thread (t, j) owns output j of token t, 128 products in channel order, as
// rtp_index_keys forms them.
__device__ __forceinline__ void project_block(const CacheView& cv, const HeadMaps& hm, const RopeArgs& a, const int block, unsigned char* smem) {
  float* ws = reinterpret_cast<float*>(smem);
  __nv_bfloat16* xs = reinterpret_cast<__nv_bfloat16*>(smem + kHeadDim * kIndexDim * 4);
  const int tid = threadIdx.x, head = block % cv.n_ih, t0 = block / cv.n_ih * kProjTokens;
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
#pragma unroll 4
  for (int i = 0; i < kHeadDim; i += 8) {
    const uint4 x = *reinterpret_cast<const uint4*>(xs + r * kHeadDim + i);
    const uint32_t u[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      acc = fmaf(low(u[e]), ws[(i + 2 * e) * kIndexDim + c], acc);
      acc = fmaf(high(u[e]), ws[(i + 2 * e + 1) * kIndexDim + c], acc);
    }
  }
  if (t >= a.T) return;
  const int pos = a.tok_pos[t], phys = page_for(cv, a.tok_seq[t], pos);   // (index keys live in the main pool)
  if (phys < 0) return;
  const int64_t at = (((int64_t)phys * cv.n_ih + head) * kPage + (pos & (kPage - 1))) * kIndexDim + c;
  if (cv.ikey_fp8)
    reinterpret_cast<uint8_t*>(cv.ikey)[at] = (uint8_t)__nv_cvt_float_to_fp8(acc, __NV_SATFINITE, __NV_E4M3);
  else
    cv.ikey[at] = __float2bfloat16_rn(acc);
}

// Cosine and sine of a position's angle: p f / 2 pi as a sum of two, whole turns go, and what the first one's rounding lost comes back.
__device__ __forceinline__ float2 turn(int pos, double fr, float scale) {
  const double g = fr * kInvTwoPi, g_low = fma(fr, kInvTwoPi, -g) + fr * kInvTwoPiLow;
  const double turns = pos * g, rest = fma((double)pos, g, -turns) + pos * g_low;
  float s, c;
  sincospif((float)(2.0 * ((turns - rint(turns)) + rest)), &s, &c);
  return make_float2(c * scale, s * scale);
}
// A thread's two chunks, partners of each other (half split) or neighbours of four pairs each (interleaved), by eight angles.
__device__ __forceinline__ void rotate(uint4& a, uint4& b, const float2 (&cs)[8], bool interleaved) {
  uint32_t* wa = reinterpret_cast<uint32_t*>(&a);
  uint32_t* wb = reinterpret_cast<uint32_t*>(&b);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float ax = low(wa[e]), ay = high(wa[e]), bx = low(wb[e]), by = high(wb[e]);
    // two pairs (p, q) side by side and their angles
    const float2 u = interleaved ? cs[e] : cs[2 * e], w = interleaved ? cs[4 + e] : cs[2 * e + 1];
    const float2 p = interleaved ? make_float2(ax, bx) : make_float2(ax, ay), q = interleaved ? make_float2(ay, by) : make_float2(bx, by);
    const float2 c = make_float2(u.x, w.x), s = make_float2(u.y, w.y);
    const float2 pr = fma2(p, c, mul2(q, make_float2(-s.x, -s.y))), qr = fma2(q, c, mul2(p, s));
    wa[e] = interleaved ? pack2(pr.x, qr.x) : pack2(pr.x, pr.y);
    wb[e] = interleaved ? pack2(pr.y, qr.y) : pack2(qr.x, qr.y);
  }
}
// The chunks of a row that thread j of its eight owns: partners where the row is rotated, neighbours elsewhere.
__device__ __forceinline__ int2 chunks_of(const RopeArgs& a, int j) {
  const int hc = a.half >> 3;                      // 16-byte chunks of half the rotated channels
  return a.interleaved || j >= hc ? make_int2(2 * j, 2 * j + 1) : make_int2(j, j + hc);
}

// Few tokens, or a 4-bit cache: 32 rows to a block, token after token.
__global__ void __launch_bounds__(kThreads) rope_rows_kernel(const __grid_constant__ CacheView cv, const __grid_constant__ CacheView lv,
                                                               const __grid_constant__ HeadMaps hm, const __grid_constant__ RopeArgs a) {
  chain_wait();
  constexpr int kToks = kRowsAtOnce / 2 + 1;       // (a token has a key and a value row at least)
  constexpr int kTable = kToks * kHeadDim / 2 * 8;
  __shared__ __align__(16) unsigned char smem[kTable > kProjBytes ? kTable : kProjBytes];
  __shared__ int s_page[kToks], s_local[kToks], s_pos[kToks];
  const int before = a.proj_blocks;                // (the projecting blocks first: theirs is the longest way)
  if ((int)blockIdx.x < before) {
    project_block(cv, hm, a, blockIdx.x, smem);
    return;
  }
  const int tid = threadIdx.x, j = tid & 7;
  const unsigned row0 = (blockIdx.x - before) * kRowsAtOnce, n_rows = (unsigned)a.T * a.rows_per_tok;
  const unsigned t0 = row0 / a.rows_per_tok, t1 = (min(row0 + kRowsAtOnce, n_rows) - 1) / a.rows_per_tok;
  const int n_tok = (int)(t1 - t0) + 1;
  const int2 mine = chunks_of(a, j);
  const unsigned row = row0 + (tid >> 3);
  int head = -1, tok = 0;                          // head: query heads, then keys, then values; -1: no row
  uint4 xa = make_uint4(0, 0, 0, 0), xb = xa;
  if (row < n_rows) {
    const unsigned t = row / a.rows_per_tok;
    head = (int)(row - t * a.rows_per_tok) + (a.q ? 0 : a.n_q);
    tok = (int)(t - t0);
    const __nv_bfloat16* src = head < a.n_q ? a.q + (int64_t)t * a.q_stride + head * kHeadDim
                               : head < a.n_q + a.n_kv ? a.k + (int64_t)t * a.k_stride + (head - a.n_q) * kHeadDim
                                                       : a.v + (int64_t)t * a.v_stride + (head - a.n_q - a.n_kv) * kHeadDim;
    const bool rot = head < a.n_q + a.n_kv;
    // (a plain load: the queries may be rotated in place)
    xa = *reinterpret_cast<const uint4*>(src + (rot ? mine.x : 2 * j) * 8);
    xb = *reinterpret_cast<const uint4*>(src + (rot ? mine.y : 2 * j + 1) * 8);
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
    table[i] = turn(a.tok_pos[t0 + t], a.freqs[f], a.scale);
  }
  __syncthreads();
  if (head >= 0 && head < a.n_q + a.n_kv && j < (a.half >> 3)) {
    float2 cs[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) cs[e] = table[tok * a.half + j * 8 + e];
    rotate(xa, xb, cs, a.interleaved);
  }
  if (head >= 0 && head < a.n_q) {
    __nv_bfloat16* dst = a.q_out + ((int64_t)(t0 + tok) * a.n_q + head) * kHeadDim;
    *reinterpret_cast<uint4*>(dst + mine.x * 8) = xa;
    *reinterpret_cast<uint4*>(dst + mine.y * 8) = xb;
  }
  // keys and values
  const bool is_v = head >= a.n_q + a.n_kv;
  const int kvh = head - a.n_q - (is_v ? a.n_kv : 0);
  int64_t to = -1;
  bool local = false;
  if (head >= a.n_q) {
    local = cv.kv_slot[kvh] == 0xff;               // (the head lives in the other pool)
    const CacheView& v = local ? lv : cv;
    const int phys = local ? s_local[tok] : s_page[tok];
    if (phys >= 0) to = ((int64_t)phys * v.n_kv + v.kv_slot[kvh]) * kPage + (s_pos[tok] & (kPage - 1));
  }
  const CacheView& v = local ? lv : cv;
  const int ca = is_v ? 2 * j : mine.x, cb = is_v ? 2 * j + 1 : mine.y;
  if (!cv.kv_fp4) {
    if (to >= 0) {
      __nv_bfloat16* dst = const_cast<__nv_bfloat16*>(is_v ? v.v : v.k) + to * kHeadDim;
      *reinterpret_cast<uint4*>(dst + ca * 8) = xa;
      *reinterpret_cast<uint4*>(dst + cb * 8) = xb;
    }
    return;
  }
  // the row through shared memory (the angles are no longer read), so that a thread has the 16 channels of one scale
  __syncthreads();
  uint4* st = reinterpret_cast<uint4*>(smem) + (tid >> 3) * 16;
  st[ca] = xa;
  st[cb] = xb;
  __syncwarp();
  if (to >= 0) {
    uint32_t scale;
    bool bad = false;
    const uint2 codes = kv4_encode(st[2 * j], st[2 * j + 1], scale, bad);
    if (bad) set_status(a.status, RTP_ERR_UNSUPPORTED);
    uint8_t* pages = const_cast<uint8_t*>(reinterpret_cast<const uint8_t*>(is_v ? v.v : v.k));
    *reinterpret_cast<uint2*>(pages + to * kKv4TokBytes + j * 8) = codes;
    const_cast<uint8_t*>(v.kv_scales)[to * kKv4ScaleBytes + (is_v ? 8 : 0) + j] = (uint8_t)scale;
  }
}

// Many tokens on a bf16 cache: a block has eight tokens and all their rows.  A thread keeps to one token and one pair of chunks and goes
// through the heads, every fourth, so that its eight angles stay in registers and what is left of a row is two loads, the products and two
// stores.  8192 tokens of 48 rows: 40.8 us (202 MB at 4.9 TB/s; without the products 36), 51 with 128 rows to a block and the angles in
// shared memory.
constexpr int kBlockToks = 8;
constexpr int kAhead = 2;                          // rows in flight per thread (five blocks per SM; four rows and four blocks: 41.4 us)
__global__ void __launch_bounds__(kThreads, 5) rope_tokens_kernel(const __grid_constant__ CacheView cv, const __grid_constant__ CacheView lv,
                                                               const __grid_constant__ HeadMaps hm, const __grid_constant__ RopeArgs a) {
  chain_wait();
  __shared__ __align__(16) unsigned char smem[kProjBytes];   // (eight tokens' angles are 4 KB)
  __shared__ int s_page[kBlockToks], s_local[kBlockToks];
  const int before = projecting_before(a, blockIdx.x);
  if (projecting_before(a, (int64_t)blockIdx.x + 1) > before) {
    project_block(cv, hm, a, before, smem);
    return;
  }
  const int tid = threadIdx.x, j = tid & 7, tk = (tid >> 3) & (kBlockToks - 1), h0 = tid >> 6;
  const int t0 = (blockIdx.x - before) * kBlockToks, t = t0 + tk;
  constexpr int kStep = kThreads / 8 / kBlockToks;           // heads at a time
  float2* table = reinterpret_cast<float2*>(smem);
  if (tid < kBlockToks && t0 + tid < a.T) {
    const int seq = a.tok_seq[t0 + tid], pos = a.tok_pos[t0 + tid];
    const int main_page = cv.n_kv > 0 ? page_for(cv, seq, pos) : 0, local_page = lv.n_kv > 0 ? page_for(lv, seq, pos) : 0;
    if (main_page < 0 || local_page < 0) set_status(a.status, RTP_ERR_INVALID);
    s_page[tid] = main_page;
    s_local[tid] = local_page;
  }
  for (int i = tid; i < kBlockToks * a.half; i += kThreads) {
    const int r = i / a.half, f = i - r * a.half;
    if (t0 + r < a.T) table[i] = turn(a.tok_pos[t0 + r], a.freqs[f], a.scale);
  }
  __syncthreads();
  if (t >= a.T) return;
  const int2 mine = chunks_of(a, j);
  const bool rot = j < (a.half >> 3);
  float2 cs[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) cs[e] = rot ? table[tk * a.half + j * 8 + e] : make_float2(1.f, 0.f);
  const int pos = a.tok_pos[t] & (kPage - 1);
  auto heads = [&](int n, const __nv_bfloat16* src, int ca, int cb, bool turned, auto&& store) {
    for (int h = h0; h < n; h += kAhead * kStep) {
      uint4 xa[kAhead], xb[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (h + u * kStep < n) {                   // (a plain load: the queries may be rotated in place)
          xa[u] = *reinterpret_cast<const uint4*>(src + (h + u * kStep) * kHeadDim + ca * 8);
          xb[u] = *reinterpret_cast<const uint4*>(src + (h + u * kStep) * kHeadDim + cb * 8);
        }
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (h + u * kStep < n) {
          if (turned) rotate(xa[u], xb[u], cs, a.interleaved);
          if (__nv_bfloat16* dst = store(h + u * kStep)) {
            *reinterpret_cast<uint4*>(dst + ca * 8) = xa[u];
            *reinterpret_cast<uint4*>(dst + cb * 8) = xb[u];
          }
        }
    }
  };
  auto place = [&](int h, bool values) -> __nv_bfloat16* {
    const bool local = cv.kv_slot[h] == 0xff;      // (the head lives in the other pool)
    const CacheView& v = local ? lv : cv;
    const int phys = local ? s_local[tk] : s_page[tk];
    return phys < 0 ? nullptr : const_cast<__nv_bfloat16*>(values ? v.v : v.k) + (((int64_t)phys * v.n_kv + v.kv_slot[h]) * kPage + pos) * kHeadDim;
  };
  if (a.q) {
    __nv_bfloat16* out = a.q_out + (int64_t)t * a.n_q * kHeadDim;
    heads(a.n_q, a.q + (int64_t)t * a.q_stride, mine.x, mine.y, rot, [&](int h) { return out + h * kHeadDim; });
  }
  heads(a.n_kv, a.k + (int64_t)t * a.k_stride, mine.x, mine.y, rot, [&](int h) { return place(h, false); });
  heads(a.n_kv, a.v + (int64_t)t * a.v_stride, 2 * j, 2 * j + 1, false, [&](int h) { return place(h, true); });
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
  // blocks of eight tokens where there are two for every SM, else of 32 rows (48 heads; 16 tokens: 7.1 us with the former, 2.7 with the
  // latter, 1184: 9.5 and 8.6, 2368: 14.7 and 14.8, 4096: 20.9 and 26.0)
  const bool many = !cv.kv_fp4 && T >= (int64_t)2 * kBlockToks * current_sm_count(148);
  const int64_t blocks = many ? (T + kBlockToks - 1) / kBlockToks : (T * a.rows_per_tok + kRowsAtOnce - 1) / kRowsAtOnce;
  (void)launch_chained(many ? rope_tokens_kernel : rope_rows_kernel, dim3((unsigned)(a.proj_blocks + blocks)), dim3(kThreads), 0, st, cv, lv, hm, a);
  return cudaGetLastError();
}

}  // namespace rtp
