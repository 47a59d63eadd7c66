// Selection of a beam search step: the k best continuations of every group of beams, score = scores[beam] + log_softmax(logits)[token],
// equal scores going to the lower (beam, token).
//
// Bound by the one read of the logits.  A row is cut into slices, one CTA each, that hold their logits in registers: maximum and
// sum of exponentials, and the slice's k best tokens.  Those need no sort: the k-th largest of the 256 threads' maxima is a
// lower bound of the k-th largest logit that only a few more than k logits reach; they go to a list, which is ordered by
// counting.  A second kernel, one CTA per group, joins the rows' sums and takes the k best of the sorted lists one by one.
// Tokens of one row are ordered by their logits alone; where rows meet, scores are 64-bit (sums of exponentials are 32-bit
// within a slice, 64-bit across slices), so that neighbours are not swapped by the rounding of a normaliser.
#include "rtp_device.cuh"

namespace rtp {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxEl = 32;               // logits per thread
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kSlack = 8;                // the search for the bound stops when that many threads too many reach it
// Threads whose maximum is above the bound: fewer than k + slack.  Each may have all of its logits above it.
constexpr int kList = (RTP_MAX_BEAM_K + kSlack) * kMaxEl + RTP_MAX_BEAM_K;

struct Cand {
  float x;
  int32_t token;
};

struct BeamArgs {
  const void* logits;
  int64_t row_stride;
  int32_t n_beams, vocab, k, n_slices, pad_token;
  const float* scores;
  const int32_t* finished;
  Cand* cand;        // [rows, slices, k], best first
  int32_t* count;    // [rows, slices]
  float2* stat;      // [rows, slices]: maximum, sum of exp(x - maximum)
  int32_t *parent, *token;
  float* scores_out;
  int32_t* status;
};

template <class T> struct Vec;           // 16 bytes of logits
template <> struct Vec<float> { static constexpr int n = 4; };
template <> struct Vec<__nv_bfloat16> { static constexpr int n = 8; };
template <> struct Vec<__half> { static constexpr int n = 8; };
__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f(__half x) { return __half2float(x); }

// Slices are counted from the 16-byte boundary at or below the row's first logit, so that whole pieces are single loads whatever
// the row's alignment; pieces that reach over an end of the row are loaded one by one.
template <class T, int EL>
__global__ void __launch_bounds__(kThreads) beam_slice_kernel(const __grid_constant__ BeamArgs a) {
  chain_wait();
  constexpr int VN = Vec<T>::n, NV = EL / VN;
  static_assert(EL % VN == 0 && EL <= kMaxEl, "");
  __shared__ __align__(8) uint2 s_list[kList];     // ordered key, token
  __shared__ float s_max[kWarps], s_sum[kWarps];
  __shared__ uint32_t s_min[kWarps];
  __shared__ int s_n, s_scan[kWarps];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t row = blockIdx.x / a.n_slices;
  const int slice = (int)(blockIdx.x - row * a.n_slices);
  const int64_t out = row * a.n_slices + slice;
  if (a.finished && a.finished[row] != 0) {
    if (tid == 0) a.count[out] = 0;
    return;
  }
  const T* base = reinterpret_cast<const T*>(a.logits) + row * a.row_stride;
  const int skew = (int)((reinterpret_cast<uintptr_t>(base) & 15u) / sizeof(T));
  const int first = slice * (kThreads * EL) - skew + tid * VN;   // token of the thread's first logit (may be negative)
  float x[EL];
  bool odd = false;                                // the thread has logits that are not there, or that are no numbers
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int t0 = first + v * kThreads * VN;
    if (t0 >= 0 && t0 + VN <= a.vocab) {
      const uint4 w = ld_stream_v4(base + t0);
      const T* e = reinterpret_cast<const T*>(&w);
#pragma unroll
      for (int i = 0; i < VN; ++i) x[v * VN + i] = to_f(e[i]);
    } else {
      odd = true;
#pragma unroll
      for (int i = 0; i < VN; ++i) x[v * VN + i] = t0 + i >= 0 && t0 + i < a.vocab ? to_f(base[t0 + i]) : -INFINITY;
    }
  }
  if (tid == 0) s_n = 0;
  // A logit that is NaN or +infinity is none that can be chosen: as -infinity.
  float mine = x[0];
#pragma unroll
  for (int i = 1; i < EL; ++i) mine = fmaxf(mine, x[i]);   // (NaN is passed over)
  {
    float nan = 0.f;
#pragma unroll
    for (int i = 0; i < EL; ++i) nan += x[i];              // not a number, or +infinity, if one of them is (or -infinity)
    if (!(nan < INFINITY) || mine == INFINITY) {
      bool bad = false;
#pragma unroll
      for (int i = 0; i < EL; ++i)
        if (!(x[i] < INFINITY)) {
          x[i] = -INFINITY;
          bad = true;
        }
      if (bad) set_status(a.status, RTP_ERR_INVALID);
      mine = x[0];
#pragma unroll
      for (int i = 1; i < EL; ++i) mine = fmaxf(mine, x[i]);
    }
  }
  // whether the thread has any token at all (-infinity is one that is ruled out; a place behind the row's end is none)
  bool some = true;
  if (odd) {
    some = false;
#pragma unroll
    for (int v = 0; v < NV; ++v) some = some || (first + v * kThreads * VN + VN > 0 && first + v * kThreads * VN < a.vocab);
  }
  const uint32_t key = some ? okey(mine) : 0u;
  const float w_max = warp_max(mine);
  const uint32_t w_min = __reduce_min_sync(0xffffffffu, key);
  if (lane == 0) {
    s_max[warp] = w_max;
    s_min[warp] = w_min;
  }
  __syncthreads();
  float m = s_max[0];
  uint32_t lo = s_min[0];
#pragma unroll
  for (int w = 1; w < kWarps; ++w) {
    m = fmaxf(m, s_max[w]);
    lo = min(lo, s_min[w]);
  }
  // sum of exponentials relative to the slice's maximum: four chains
  const float mb = m == -INFINITY ? 0.f : m;   // (taken off first: the type's largest values times log2(e) are no numbers)
  float sum4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < EL; ++i) sum4[i & 3] += fast_ex2((x[i] - mb) * kLog2e);
  const float sum = warp_sum((sum4[0] + sum4[1]) + (sum4[2] + sum4[3]));
  if (lane == 0) s_sum[warp] = sum;
  // the largest bound that k threads' maxima reach (or that a few more do), between the smallest and the largest of them
  uint32_t hi = okey(m);
  while (lo < hi) {
    const uint32_t mid = lo + (hi - lo) / 2 + 1;
    const int n = __syncthreads_count(key >= mid);
    if (n >= a.k) lo = mid; else hi = mid - 1;
    if (n >= a.k && n <= a.k + kSlack) break;
  }
  const uint32_t bound = max(lo, 1u);
  auto token_of = [&](int i) { return first + (i / VN) * kThreads * VN + i % VN; };
  auto there = [&](int i) { return !odd || (token_of(i) >= 0 && token_of(i) < a.vocab); };
  int reach = 0;
  if (key >= bound) {
    const float at = bound <= okey(-INFINITY) ? -INFINITY : okey_to_float(bound);
#pragma unroll
    for (int i = 0; i < EL; ++i) reach += x[i] >= at && there(i);
  }
  const int w_reach = __reduce_add_sync(0xffffffffu, reach);
  if (lane == 0 && w_reach) atomicAdd(&s_n, w_reach);
  __syncthreads();
  const bool all = s_n <= kList;                    // else too many equal the bound: the first of them are taken in order
  __syncthreads();
  if (tid == 0) s_n = 0;
  __syncthreads();
  if (reach) {
#pragma unroll
    for (int i = 0; i < EL; ++i) {
      const uint32_t ki = there(i) ? okey(x[i]) : 0u;
      if (ki > bound || (all && ki == bound)) s_list[atomicAdd(&s_n, 1)] = make_uint2(ki, (uint32_t)token_of(i));
    }
  }
  __syncthreads();
  int n = s_n;
  if (!all && n < a.k) {
    const int need = a.k - n;
    int before = 0;                                 // equal ones in front of this piece
#pragma unroll 1
    for (int v = 0; v < NV; ++v) {
      uint32_t eq = 0;
#pragma unroll
      for (int i = 0; i < EL; ++i)
        if (i / VN == v && there(i) && okey(x[i]) == bound) eq |= 1u << (i % VN);
      const int c = __popc(eq);
      int s = c;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += y;
      }
      __syncthreads();
      if (lane == 31) s_scan[warp] = s;
      __syncthreads();
      int at = before + s - c, total = 0;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        at += w < warp ? s_scan[w] : 0;
        total += s_scan[w];
      }
      for (int i = 0; i < VN; ++i)
        if ((eq >> i) & 1u) {
          if (at < need) s_list[n + at] = make_uint2(bound, (uint32_t)(first + v * kThreads * VN + i));
          ++at;
        }
      before += total;
      if (before >= need) break;                    // (the same in all threads)
    }
    n += min(before, need);
    __syncthreads();
  }
  // ordered by counting
  for (int i = tid; i < n; i += kThreads) {
    const uint2 me = s_list[i];
    int rank = 0;
    for (int o = 0; o < n; ++o) {
      const uint2 y = s_list[o];
      rank += y.x > me.x || (y.x == me.x && y.y < me.y);
    }
    if (rank < a.k) a.cand[out * a.k + rank] = Cand{okey_to_float(me.x), (int32_t)me.y};
  }
  if (tid == 0) {
    a.count[out] = min(n, a.k);
    float z = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) z += s_sum[w];
    a.stat[out] = make_float2(m, z);
  }
}

// One CTA per group.  Every thread watches the heads of the lists list = thread, thread + 256, ... and knows the best of them.
__global__ void __launch_bounds__(kThreads) beam_pick_kernel(const __grid_constant__ BeamArgs a) {
  chain_wait();
  extern __shared__ __align__(16) unsigned char s_at[];   // uint8 [lists]: entries taken of each list
  __shared__ double s_off[RTP_MAX_BEAMS];                  // score of a token with the row's largest logit
  __shared__ float s_max[RTP_MAX_BEAMS];                   // that logit
  __shared__ int s_state[RTP_MAX_BEAMS];                   // 1: ended, 2: no token has a probability
  __shared__ uint4 s_best[2][kWarps];                      // score (ordered, 64 bits), list, place of the winner in its list
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t row0 = (int64_t)blockIdx.x * a.n_beams;
  const int lists = a.n_beams * a.n_slices;
  for (int b = warp; b < a.n_beams; b += kWarps) {
    const int64_t row = row0 + b;
    float m = -INFINITY;
    const float2* st = a.stat + row * a.n_slices;
    const bool ended = a.finished && a.finished[row] != 0;
    if (!ended)
      for (int s = lane; s < a.n_slices; s += 32) m = fmaxf(m, st[s].x);
    m = warp_max(m);
    double z = 0.0;
    if (m != -INFINITY)
      for (int s = lane; s < a.n_slices; s += 32) z += (double)st[s].y * exp((double)st[s].x - (double)m);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
    if (lane == 0) {
      double off = a.scores ? (double)a.scores[row] : 0.0;
      if (!(off < (double)INFINITY)) {
        set_status(a.status, RTP_ERR_INVALID);
        off = -(double)INFINITY;
      }
      s_state[b] = ended ? 1 : m == -INFINITY ? 2 : 0;
      if (!ended && m != -INFINITY) off -= log(z);
      s_off[b] = off;
      s_max[b] = m;
    }
  }
  for (int l = tid; l < lists; l += kThreads) s_at[l] = 0;
  __syncthreads();
  auto head_of = [&](int l, uint64_t& key, int& token) -> bool {   // the next candidate of a list; keys order like scores
    const int b = l / a.n_slices, at = s_at[l];
    const int64_t li = (row0 + b) * a.n_slices + (l - b * a.n_slices);
    double score;
    if (s_state[b] == 1) {
      if (l != b * a.n_slices || at > 0) return false;
      score = s_off[b];
      token = a.pad_token;
    } else {
      if (at >= a.count[li]) return false;
      const Cand c = a.cand[li * a.k + at];
      token = c.token;
      score = s_state[b] == 2 ? -(double)INFINITY : s_off[b] + ((double)c.x - (double)s_max[b]);
    }
    const uint64_t u = (uint64_t)__double_as_longlong(score + 0.0);
    key = (u >> 63) ? ~u : u | 0x8000000000000000ull;
    return true;
  };
  // Lists are in the order of (beam, token), so that among equal scores the lower list goes first; within a list it is sorted so.
  // (Two slices of a row hold disjoint, ascending ranges of tokens.)
  uint64_t best = 0;
  int best_l = 0x7fffffff, best_tok = 0;
  auto look = [&]() {
    best = 0;
    best_l = 0x7fffffff;
    for (int l = tid; l < lists; l += kThreads) {
      uint64_t key;
      int token;
      if (head_of(l, key, token) && key > best) {
        best = key;
        best_l = l;
        best_tok = token;
      }
    }
  };
  look();
  for (int i = 0; i < a.k; ++i) {
    const uint32_t h = __reduce_max_sync(0xffffffffu, (uint32_t)(best >> 32));
    const uint32_t lo = __reduce_max_sync(0xffffffffu, (uint32_t)(best >> 32) == h ? (uint32_t)best : 0u);
    const bool tie = best == (((uint64_t)h << 32) | lo);
    const int l = __reduce_min_sync(0xffffffffu, tie ? best_l : 0x7fffffff);
    const int tok = __shfl_sync(0xffffffffu, best_tok, l & 31);
    if (lane == 0) s_best[i & 1][warp] = make_uint4(h, lo, (uint32_t)l, (uint32_t)tok);
    __syncthreads();
    uint4 win = s_best[i & 1][0];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) {
      const uint4 o = s_best[i & 1][w];
      const uint64_t ko = ((uint64_t)o.x << 32) | o.y, kw = ((uint64_t)win.x << 32) | win.y;
      if (ko > kw || (ko == kw && o.z < win.z)) win = o;
    }
    const bool some = (win.x | win.y) != 0u;
    if (tid == 0) {
      const int64_t at = (int64_t)blockIdx.x * a.k + i;
      const uint64_t u = ((uint64_t)win.x << 32) | win.y;
      const double score = __longlong_as_double((long long)((u >> 63) ? u & 0x7fffffffffffffffull : ~u));
      a.parent[at] = some ? (int32_t)(row0 + win.z / a.n_slices) : -1;
      a.token[at] = some ? (int32_t)win.w : -1;
      a.scores_out[at] = some ? (float)score : -INFINITY;
    }
    if (some && (int)(win.z % kThreads) == tid) {
      s_at[win.z] += 1;
      look();
    }
  }
}

// Logits per thread: as many CTAs as fill the device twice, within what a slice can hold.
int beam_el(int64_t rows, int64_t vocab, int sm_count) {
  const int64_t want = rows * vocab / ((int64_t)2 * sm_count * kThreads);
  return want >= 32 ? 32 : want >= 16 ? 16 : 8;
}
int beam_slices(int64_t vocab, int el) { return (int)((vocab + 7 + (int64_t)kThreads * el - 1) / ((int64_t)kThreads * el)); }   // (7: a row's skew)

template <class T>
cudaError_t launch_slices(const BeamArgs& a, int el, int64_t rows, cudaStream_t st) {
  const dim3 grid((unsigned)(rows * a.n_slices)), block(kThreads);
  if (el == 32) (void)launch_chained(beam_slice_kernel<T, 32>, grid, block, 0, st, a);
  else if (el == 16) (void)launch_chained(beam_slice_kernel<T, 16>, grid, block, 0, st, a);
  else (void)launch_chained(beam_slice_kernel<T, 8>, grid, block, 0, st, a);
  return cudaGetLastError();
}

}  // namespace

size_t beam_workspace_bytes(int64_t rows, int64_t vocab, int k, int sm_count) {
  const int64_t lists = rows * beam_slices(vocab, beam_el(rows, vocab, sm_count));
  return (size_t)lists * (k * sizeof(Cand) + sizeof(float2) + sizeof(int32_t)) + 2 * 256;
}

cudaError_t launch_beam_select(const void* logits, int format, int64_t row_stride, int64_t n_groups, int n_beams, int64_t vocab,
                               const float* scores, const int32_t* finished, int pad_token, int k, int32_t* parent, int32_t* token,
                               float* scores_out, void* ws, int32_t* status, int sm_count, cudaStream_t st) {
  const int64_t rows = n_groups * n_beams;
  const int el = beam_el(rows, vocab, sm_count);
  BeamArgs a = {logits, row_stride, n_beams, (int32_t)vocab, k, beam_slices(vocab, el), pad_token, scores, finished,
                nullptr, nullptr, nullptr, parent, token, scores_out, status};
  const int64_t lists = rows * a.n_slices;
  if (lists >= (int64_t)1 << 31 || (int64_t)n_beams * a.n_slices > 40000) return cudaErrorNotSupported;
  char* p = reinterpret_cast<char*>(ws);
  a.cand = reinterpret_cast<Cand*>(p);
  p += ((size_t)lists * k * sizeof(Cand) + 255) & ~(size_t)255;
  a.stat = reinterpret_cast<float2*>(p);
  p += (size_t)lists * sizeof(float2);
  a.count = reinterpret_cast<int32_t*>(p);
  cudaError_t e = format == RTP_LOGITS_F32 ? launch_slices<float>(a, el, rows, st)
                  : format == RTP_LOGITS_BF16 ? launch_slices<__nv_bfloat16>(a, el, rows, st) : launch_slices<__half>(a, el, rows, st);
  if (e != cudaSuccess) return e;
  (void)launch_chained(beam_pick_kernel, dim3((unsigned)n_groups), dim3(kThreads), (size_t)n_beams * a.n_slices, st, a);
  return cudaGetLastError();
}

}  // namespace rtp
