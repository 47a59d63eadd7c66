// Selection of a beam search step: the k best continuations of every group of beams, score = scores[beam] + log_softmax(logits)[token],
// equal scores going to the lower (beam, token).
//
// A row is cut into slices of whole chunks, one CTA each, whose threads hold the logits of two chunks in registers while the next ones are on
// their way and keep a running maximum and sum of exponentials each.  The slice's k best tokens need no second pass: the k-th largest of
// the 256 threads' maxima is a lower bound of the k-th largest logit, and only the threads that reach it, k and a few, have logits that
// do.  Those are read again (from L2), go to a list, and the list's k best are put in order.  A second kernel, one CTA per group, joins the
// rows' sums and picks the k best of the sorted lists in the same way.
// Tokens of one row are ordered by their logits, or rather by scores[beam] + logit in 64 bits: where a large score swallows the differences
// (all of them, at -infinity), tokens are equal and the lower one goes first.  Where rows meet, scores are 64-bit (sums of exponentials
// are 32-bit within a slice, 64-bit across slices), so that neighbours are not swapped by the rounding of a normaliser.
// Bound by the one read of the logits in principle (10 us for 32 x 8 beams over 128K in bf16); measured 22.7 us: the slices 18, of which the
// pass over the logits is about 11 (the special function unit's rate for one exponential per logit is 8), launch, first loads, bound and
// lists the rest; the second kernel 4 to 5.  4 beams over 32K: 9.0 us, two launches and chains of dependent loads and reductions.
// Tried and left: a list that grows during the pass under a bound from its first chunk (the slices 26 us: additions were 40 % of the
// instructions); k rounds over the lists' heads in the second kernel (8 us; still there for lists that do not fit); logits of short
// slices kept in registers for the list and the second kernel launched ahead (no difference).
#include <type_traits>

#include "rtp_device.cuh"

namespace rtp {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kSlack = 32;               // the search for the bound stops when that many threads too many reach it
constexpr int kKeep = 512;               // a list that is longer is cut to its k best before more is added
constexpr int kList = kKeep + kWarps * 32 * 8;   // (a warp adds at most a piece per lane at a time)
constexpr int kShort = 64;               // lists that are ordered without a bound
constexpr int kSelect = 256;
constexpr int kTops = kThreads / 4;
static_assert(kTops >= RTP_MAX_BEAM_K, "a bound is the k-th of them");

struct Cand {
  float x;
  int32_t token;
};

struct BeamArgs {
  const void* logits;
  int64_t row_stride;
  int32_t n_beams, vocab, k, n_slices, chunks, pad_token;   // chunks: of a slice
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

// Pieces to 32 bits.
__device__ __forceinline__ void unpack(const uint4& w, float* x, float) {
  x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y); x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w);
}
__device__ __forceinline__ void unpack(const uint4& w, float* x, __nv_bfloat16) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(u[i] << 16);
    x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void unpack(const uint4& w, float* x, __half) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u[i]));
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
  }
}
// The thread's largest logit, or NaN if one of them is.
__device__ __forceinline__ float max_nan(float a, float b) {
  float m;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b));
  return m;
}
template <int N>
__device__ __forceinline__ float max_of(const uint4 (&w)[N], float) {
  float m = __uint_as_float(w[0].x);
#pragma unroll
  for (int v = 0; v < N; ++v)
    m = max_nan(m, max_nan(max_nan(__uint_as_float(w[v].x), __uint_as_float(w[v].y)), max_nan(__uint_as_float(w[v].z), __uint_as_float(w[v].w))));
  return m;
}
template <class P, int N>
__device__ __forceinline__ P max_pair(const uint4 (&w)[N]) {
  P m = *reinterpret_cast<const P*>(&w[0].x);
#pragma unroll
  for (int v = 0; v < N; ++v) {
    const P* p = reinterpret_cast<const P*>(&w[v]);
    m = __hmax2_nan(m, __hmax2_nan(__hmax2_nan(p[0], p[1]), __hmax2_nan(p[2], p[3])));
  }
  return m;
}
template <int N>
__device__ __forceinline__ float max_of(const uint4 (&w)[N], __nv_bfloat16) {
  const float2 f = __bfloat1622float2(max_pair<__nv_bfloat162>(w));
  return max_nan(f.x, f.y);
}
template <int N>
__device__ __forceinline__ float max_of(const uint4 (&w)[N], __half) {
  const float2 f = __half22float2(max_pair<__half2>(w));
  return max_nan(f.x, f.y);
}
// NaN and +infinity become -infinity.
template <int N>
__device__ __forceinline__ void rule_out(uint4 (&w)[N], float) {
  auto f = [](uint32_t u) { return __uint_as_float(u) < INFINITY ? u : 0xff800000u; };
#pragma unroll
  for (int v = 0; v < N; ++v) w[v] = make_uint4(f(w[v].x), f(w[v].y), f(w[v].z), f(w[v].w));
}
template <int N, class H>
__device__ __forceinline__ void rule_out(uint4 (&w)[N], H) {
  const uint32_t none = std::is_same<H, __half>::value ? 0xfc00u : 0xff80u, top = none & 0x7fffu;
  auto f = [=](uint32_t u) {                       // (a half-word is NaN or infinity from its type's infinity on)
    const uint32_t lo = (u & 0x7fffu) >= top ? none : u & 0xffffu, hi = ((u >> 16) & 0x7fffu) >= top ? none : u >> 16;
    return lo | hi << 16;
  };
#pragma unroll
  for (int v = 0; v < N; ++v) w[v] = make_uint4(f(w[v].x), f(w[v].y), f(w[v].z), f(w[v].w));
}
// Two numbers at a time.
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 r;
  asm("{\n.reg .b64 a, b, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nadd.rn.f32x2 d, a, b;\nmov.b64 {%0, %1}, d;\n}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 r;
  asm("{\n.reg .b64 a, b, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmul.rn.f32x2 d, a, b;\nmov.b64 {%0, %1}, d;\n}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
// The sum of exp(x + off).
template <class T, int N>
__device__ __forceinline__ float weigh(const uint4 (&w)[N], float off) {
  const float2 o2 = make_float2(off, off), l2 = make_float2(kLog2e, kLog2e);
  float2 s0 = make_float2(0.f, 0.f), s1 = s0;
#pragma unroll
  for (int v = 0; v < N; ++v) {
    float x[Vec<T>::n];
    unpack(w[v], x, T());
#pragma unroll
    for (int i = 0; i < Vec<T>::n; i += 4) {
      const float2 u = mul2(add2(make_float2(x[i], x[i + 1]), o2), l2), y = mul2(add2(make_float2(x[i + 2], x[i + 3]), o2), l2);
      s0 = add2(s0, make_float2(fast_ex2(u.x), fast_ex2(u.y)));
      s1 = add2(s1, make_float2(fast_ex2(y.x), fast_ex2(y.y)));
    }
  }
  s0 = add2(s0, s1);
  return s0.x + s0.y;
}

// Which token is whose is the same whatever the row's alignment, so that rows of equal logits have equal normalisers.  A row that does not
// begin at a 16-byte boundary is read in aligned pieces all the same: a thread's eight or four logits lie in two of them, which a shift joins
// (twice the loads, most of them from L1).  Pieces that reach over an end of the row are loaded one by one.
template <class T>
__device__ __forceinline__ uint4 join(const uint4& lo, const uint4& hi, int s) {   // the 16 bytes from element s of lo on
  uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
  const int bytes = s * (int)sizeof(T);
  if (bytes & 8) {
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
  }
  if (bytes & 4) {
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
  }
  const int bits = 8 * (bytes & 3);
  return make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits), __funnelshift_r(w[2], w[3], bits),
                    __funnelshift_r(w[3], w[4], bits));
}
// A piece of which only the logits lo .. hi - 1 exist: the others are -infinity.
template <class T>
struct __align__(16) Piece {
  T e[Vec<T>::n];
};
template <class T>
__device__ __noinline__ uint4 edge_piece(const T* base, int t0, int lo, int hi) {
  static_assert(sizeof(Piece<T>) == sizeof(uint4) && alignof(Piece<T>) == alignof(uint4), "read as one");
  Piece<T> p;
#pragma unroll
  for (int i = 0; i < Vec<T>::n; ++i) p.e[i] = t0 + i >= lo && t0 + i < hi ? base[t0 + i] : T(-INFINITY);
  return *reinterpret_cast<const uint4*>(&p);
}
// What a logit counts as beside the others of its row: what is left of score + x, in 64 bits, when the score is taken off again.  That is x
// itself where the score is below 2^26 |x| (64 bits then keep more than half of what is between two 32-bit numbers), and a function of the
// sum alone, of which 32 bits hold all: the difference is x, or a multiple of the sum's last place that is as small as x.
__device__ __forceinline__ float counts_as(float x, float score) {
  if (fabsf(score) < 0x1p26f * fabsf(x)) return x;
  const double sum = (double)score + (double)x;
  return sum == -(double)INFINITY ? -INFINITY : (float)(sum - (double)score);
}
__device__ __forceinline__ uint32_t counts_as_key(uint32_t key, float score) { return okey(counts_as(okey_to_float(key), score) + 0.f); }
constexpr uint32_t kLowest = 0x007fffffu, kLargest = 0xff7fffffu;   // keys of -infinity and of the largest number
// The keys low .. high that count like `key`.
__device__ __noinline__ uint2 alike(uint32_t key, float score) {
  const int lane = threadIdx.x & 31;
  const uint32_t as = counts_as_key(key, score);
  const uint32_t low = (uint32_t)warp_search_first(kLowest, key, lane, [&](uint32_t u) { return counts_as_key(u, score) >= as; });
  return make_uint2(low, (uint32_t)(warp_search_first(key, kLargest, lane, [&](uint32_t u) { return counts_as_key(u, score) > as; }) - 1));
}
// The keys of a list, as they count.
__device__ __noinline__ void settle(uint2* list, int n, float score) {
  for (int i = threadIdx.x; i < n; i += kThreads) list[i].x = counts_as_key(list[i].x, score);
}
__device__ __forceinline__ uint4 ld_piece(const void* p) { return __ldg(reinterpret_cast<const uint4*>(p)); }

template <class T>
__global__ void __launch_bounds__(kThreads, 4) beam_slice_kernel(const __grid_constant__ BeamArgs a) {
  chain_wait();
  constexpr int VN = Vec<T>::n, NV = 2, kChunk = kThreads * NV * VN;   // (a chunk: 8 KB)
  __shared__ __align__(16) uint2 s_list[kList];    // ordered key, token
  __shared__ __align__(16) uint2 s_sel[kSelect];
  __shared__ uint2 s_best[RTP_MAX_BEAM_K];
  __shared__ __align__(16) uint32_t s_top[kTops];
  __shared__ uint32_t s_range[2];
  __shared__ uint8_t s_column[kThreads];
  __shared__ float s_max[kWarps], s_sum[kWarps], s_score;
  __shared__ int s_n, s_sel_n, s_columns, s_scan[kWarps];
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
  const int c_lo = slice * a.chunks, c_hi = min(c_lo + a.chunks, (a.vocab + kChunk - 1) / kChunk);
  const int stop = (int)min((int64_t)c_hi * kChunk, (int64_t)a.vocab);     // the slice's tokens end here
  const uint32_t none = sizeof(T) == 4 ? 0xff800000u : std::is_same<T, __half>::value ? 0xfc00fc00u : 0xff80ff80u;   // -infinity
  // ---- the thread's maximum and sum, two chunks at a time; tokens behind the slice are -infinity
  auto piece = [&](int t0) -> uint4 {              // of a row without skew
    return t0 + VN <= stop ? ld_stream_v4(base + t0) : t0 < stop ? edge_piece(base, t0, t0, stop) : make_uint4(none, none, none, none);
  };
  auto two_pieces = [&](int t0, uint4& lo, uint4& hi) {   // that hold the logits from t0 on of a row with skew
    const int first = t0 - skew;
    if (first >= 0 && first + 2 * VN <= stop) {
      lo = ld_piece(base + first);
      hi = ld_piece(base + first + VN);
    } else if (t0 < stop) {
      lo = edge_piece(base, first, t0, min(t0 + VN, stop));
      hi = edge_piece(base, first + VN, t0, min(t0 + VN, stop));
    } else {
      lo = hi = make_uint4(none, none, none, none);
    }
  };
  uint4 wa[2 * NV], wb[2 * NV];                    // chunks c and c + 1, c + 2 and c + 3; of a row with skew the pieces of two chunks
  auto load_pair = [&](int c, uint4 (&w)[2 * NV]) {
    const int t0 = c * kChunk + tid * VN;
    if ((c + 2) * kChunk <= stop) {
#pragma unroll
      for (int v = 0; v < 2 * NV; ++v) w[v] = ld_stream_v4(base + t0 + v * kThreads * VN);
    } else {
#pragma unroll
      for (int v = 0; v < 2 * NV; ++v) w[v] = piece(t0 + v * kThreads * VN);
    }
  };
  auto load_pieces = [&](int c) {
#pragma unroll
    for (int v = 0; v < 2 * NV; ++v) two_pieces(c * kChunk + tid * VN + v * kThreads * VN, wa[v], wb[v]);
  };
  // the beam's score, which is needed after the pass
  if (tid == 0) {
    if (a.scores)
      asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"((uint32_t)__cvta_generic_to_shared(&s_score)), "l"(a.scores + row) : "memory");
    else
      s_score = 0.f;
  }
  float m = -INFINITY, sum = 0.f;
  // (The maximum is taken off first: the largest logit's term is 1 and nothing else, so that rows with one certain token each are equal, and
  // the type's largest values times log2(e) would be no numbers.)
  auto account = [&](uint4 (&w)[2 * NV]) {
    float top = max_of(w, T());
    if (!(top < INFINITY)) {                       // NaN and +infinity are none that can be chosen: as -infinity
      set_status(a.status, RTP_ERR_INVALID);
      rule_out(w, T());
      top = max_of(w, T());
    }
    const float m_was = m;
    m = fmaxf(m, top);
    const float off = m == -INFINITY ? 0.f : -m;
    sum = sum * fast_ex2((m_was + off) * kLog2e) + weigh<T>(w, off);   // (nothing yet: 0 * 0)
  };
  if (skew) {
    load_pieces(c_lo);
#pragma unroll 1
    for (int c = c_lo; c < c_hi; c += 2) {
      uint4 u[2 * NV];
#pragma unroll
      for (int v = 0; v < 2 * NV; ++v) u[v] = join<T>(wa[v], wb[v], skew);
      if (c + 2 < c_hi) load_pieces(c + 2);
      account(u);
    }
  } else {
    load_pair(c_lo, wa);
    load_pair(c_lo + 2, wb);
#pragma unroll 1
    for (int c = c_lo; c < c_hi; c += 4) {
      account(wa);
      if (c + 4 < c_hi) load_pair(c + 4, wa);
      if (c + 2 >= c_hi) break;
      account(wb);
      if (c + 6 < c_hi) load_pair(c + 6, wb);
    }
  }
  // ---- the slice's k best
  float score = 0.f;
  bool plain = true;                               // the score swallows nothing of what may be on the list
  auto range = [&](uint32_t key) -> uint2 {        // of keys that count like this one; most often it is the only one
    return key < kLowest || score == 0.f || fabsf(score) < 0x1p26f * fabsf(okey_to_float(key)) ? make_uint2(key, key) : alike(key, score);
  };
  int n = 0;                                       // entries of the list (the same in all threads, like what follows)
  uint32_t least = 0;                              // the list takes keys from here on
  // The largest bound that k threads' keys reach (or that a few more do), or 0.  The k-th largest of 64 keys, each the largest of four
  // threads', is one that k threads reach, and few more do unless k is near 64: from there the search goes on by halves.
  auto search = [&](uint32_t key) -> uint32_t {
    uint32_t four = max(key, __shfl_xor_sync(0xffffffffu, key, 1));
    four = max(four, __shfl_xor_sync(0xffffffffu, four, 2));
    __syncthreads();
    if ((lane & 3) == 0) s_top[tid >> 2] = four;
    if (tid == 0) {
      s_range[0] = 0xffffffffu;
      s_range[1] = 0u;
    }
    __syncthreads();
    int more = 0;                                  // keys above this one, a quarter of them in each of its threads
#pragma unroll
    for (int i = 0; i < kTops / 4; i += 4) {
      const uint4 o = *reinterpret_cast<const uint4*>(s_top + (lane & 3) * (kTops / 4) + i);
      more += (o.x > four) + (o.y > four) + (o.z > four) + (o.w > four);
    }
    more += __shfl_xor_sync(0xffffffffu, more, 1);
    more += __shfl_xor_sync(0xffffffffu, more, 2);
    const uint32_t w_lo = __reduce_min_sync(0xffffffffu, more < a.k ? four : 0xffffffffu), w_hi = __reduce_max_sync(0xffffffffu, four);
    if (lane == 0) {
      atomicMin(&s_range[0], w_lo);                // (the k-th largest is the least that fewer than k are above)
      atomicMax(&s_range[1], w_hi);
    }
    __syncthreads();
    uint32_t lo = s_range[0], hi = s_range[1];
    for (uint32_t mid = lo; ; mid = lo + (hi - lo) / 2 + 1) {
      const int r = __syncthreads_count(key >= mid);
      if (r >= a.k) lo = mid; else hi = mid - 1;
      if (lo >= hi || (r >= a.k && r <= a.k + kSlack)) return lo;
    }
  };
  // The list's k best in their order, counted out; of a long list only those that reach a bound of its threads' best.
  auto rank_of = [&](const uint2* v, int count, uint2 me) {
    const uint64_t mk = ((uint64_t)me.x << 32) | ~me.y;     // (larger key first, then lower token)
    int rank = 0, o = 0;
    for (; o + 1 < count; o += 2) {
      const uint4 y = *reinterpret_cast<const uint4*>(v + o);
      rank += (((uint64_t)y.x << 32) | ~y.y) > mk;
      rank += (((uint64_t)y.z << 32) | ~y.w) > mk;
    }
    if (o < count) rank += (((uint64_t)v[o].x << 32) | ~v[o].y) > mk;
    return rank;
  };
  auto order = [&]() {
    __syncthreads();
    if (!plain) {
      settle(s_list, n, score);
      __syncthreads();
    }
    const uint2* v = s_list;
    int count = n;
    if (n > kShort) {
      uint32_t best = 0;
      for (int i = tid; i < n; i += kThreads) best = max(best, s_list[i].x);
      const uint32_t bound = search(best);
      if (tid == 0) s_sel_n = 0;
      __syncthreads();
      for (int i = tid; i < n; i += kThreads)
        if (s_list[i].x >= bound) {
          const int to = atomicAdd(&s_sel_n, 1);
          if (to < kSelect) s_sel[to] = s_list[i];
        }
      __syncthreads();
      if (s_sel_n <= kSelect) {                             // (else many are equal: all of them are looked at)
        v = s_sel;
        count = s_sel_n;
      }
    }
    for (int i = tid; i < count; i += kThreads) {
      const uint2 me = v[i];
      const int rank = rank_of(v, count, me);
      if (rank < a.k) s_best[rank] = me;
    }
    __syncthreads();
  };
  auto cut = [&]() {
    order();
    n = min(n, a.k);
    for (int i = tid; i < n; i += kThreads) s_list[i] = s_best[i];
    if (tid == 0) s_n = n;
    least = max(least, range(s_best[a.k - 1].x).x);   // (n is k: there were more)
    __syncthreads();
  };
  // Threads whose maximum reaches the bound, or what counts like it, have what is to be looked at again: few of them, unless more equal the
  // bound than that.  Then it is what lies above it, and of the equal ones the first in the order of their tokens.
  const uint32_t key = c_lo * kChunk + tid * VN < stop ? okey(m + 0.f) : 0u;   // orders like the maximum (-0 is 0); 0: no token
  if (tid == 0) asm volatile("cp.async.wait_all;" ::: "memory");
  const uint32_t bound = search(key);
  score = s_score < INFINITY ? s_score : -INFINITY;        // (as the second kernel takes it)
  const uint2 equal = range(max(bound, 1u));       // (1: less than any logit's key)
  plain = score == 0.f || fabsf(score) < 0x1p26f * okey_to_float(equal.x);   // (no key of the list will be less)
  const bool few = __syncthreads_count(key >= equal.x) <= a.k + kSlack;
  least = few ? equal.x : equal.y + 1;
  if (tid == 0) s_n = s_columns = 0;
  __syncthreads();
  if (key >= least) s_column[atomicAdd(&s_columns, 1)] = (uint8_t)tid;
  __syncthreads();
  // A warp goes through a thread's logits, a piece per lane.
  const int columns = s_columns, pieces = (c_hi - c_lo) * NV;
  auto look = [&](int column, int p) {
    const int t0 = c_lo * kChunk + p * kThreads * VN + s_column[column] * VN;
    if (t0 >= stop) return;
    uint4 w, hi;
    if (skew) {
      two_pieces(t0, w, hi);
      w = join<T>(w, hi, skew);
    } else {
      w = piece(t0);
    }
    float x[VN];
    unpack(w, x, T());
#pragma unroll
    for (int i = 0; i < VN; ++i) {
      const uint32_t u = x[i] < INFINITY ? okey(x[i] + 0.f) : okey(-INFINITY);
      if (u >= least && t0 + i < stop) {
        const int to = atomicAdd(&s_n, 1);
        if (to < kList) s_list[to] = make_uint2(u, (uint32_t)(t0 + i));
      }
    }
  };
  for (int j = warp; j < columns; j += kWarps)
    for (int p = lane; p < pieces; p += 32) look(j, p);
  __syncthreads();
  n = s_n;
  if (n > kList) {                                 // so many in a few threads: again, with cuts in between that raise the bound
    __syncthreads();
    if (tid == 0) s_n = 0;
    n = 0;
    __syncthreads();
    for (int j = 0; j < columns; j += kWarps)
      for (int p = 0; p < pieces; p += 32) {
        if (j + warp < columns && p + lane < pieces) look(j + warp, p + lane);
        __syncthreads();
        n = s_n;
        __syncthreads();
        if (n > kKeep) cut();
      }
  }
  if (!few && n < a.k) {
    int need = a.k - n;
#pragma unroll 1
    for (int p = 0; p < pieces && need > 0; ++p) {
      const int t0 = c_lo * kChunk + p * kThreads * VN + tid * VN;
      uint32_t eq = 0;                             // a bit for each of the thread's logits that is one
      if (t0 < stop) {
        uint4 w, hi;
        if (skew) {
          two_pieces(t0, w, hi);
          w = join<T>(w, hi, skew);
        } else {
          w = piece(t0);
        }
        float x[VN];
        unpack(w, x, T());
#pragma unroll
        for (int i = 0; i < VN; ++i)
          if (t0 + i < stop) {
            const uint32_t u = x[i] < INFINITY ? okey(x[i] + 0.f) : okey(-INFINITY);
            eq |= (uint32_t)(u >= equal.x && u <= equal.y) << i;
          }
      }
      const int cnt = __popc(eq);
      int s = cnt;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += y;
      }
      __syncthreads();
      if (lane == 31) s_scan[warp] = s;
      __syncthreads();
      int at = s - cnt, total = 0;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        at += w < warp ? s_scan[w] : 0;
        total += s_scan[w];
      }
      for (; eq; eq &= eq - 1, ++at)
        if (at < need) s_list[n + at] = make_uint2(bound, (uint32_t)(t0 + __ffs(eq) - 1));
      n += min(total, need);
      need -= min(total, need);
    }
  }
  __syncthreads();
  order();
  const int kept = min(n, a.k);
  for (int i = tid; i < kept; i += kThreads) a.cand[out * a.k + i] = Cand{okey_to_float(s_best[i].x), (int32_t)s_best[i].y};
  // the slice's maximum and sum
  const float w_max = warp_max(m);
  if (lane == 0) s_max[warp] = w_max;
  __syncthreads();
  float top = s_max[0];
#pragma unroll
  for (int w = 1; w < kWarps; ++w) top = fmaxf(top, s_max[w]);
  const float part = warp_sum(m == -INFINITY ? 0.f : sum * fast_ex2((m - top) * kLog2e));
  if (lane == 0) s_sum[warp] = part;
  __syncthreads();
  if (tid == 0) {
    float z = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) z += s_sum[w];
    a.count[out] = kept;
    a.stat[out] = make_float2(top, z);
  }
}

// One CTA per group.  The rows' normalisers, then the lists' entries as 64-bit scores in shared memory; those that reach a bound (a few more
// than k) are ranked against each other.  Where the lists do not fit, or many are equal, k rounds take one entry each: every lane knows the
// best of the lists list = thread, thread + threads, ..; a single warp does the rounds where 32 lanes have few lists each.
// Lists are in the order of (beam, token): the slices of a row hold disjoint, ascending ranges of tokens, and a list is sorted.  So of
// equal scores the lower entry goes first.
// Entries in shared memory: what the 48 KB hold that a kernel has without asking, beside the rest.  8 rows of 128K in 32 bits, 32 slices each: 3072
// entries (k = 12) 15.8 us, ranked; 3328 (k = 13) 18.2 and 4096 (k = 16) 20.0 in rounds, which cost about 0.6 us each.
constexpr int kPickCached = 3200;
constexpr int kPickFew = 256;                      // entries that are ranked against each other
__device__ __forceinline__ double score_of(uint64_t key) {
  return __longlong_as_double((long long)((key >> 63) ? key & 0x7fffffffffffffffull : ~key));
}
__global__ void __launch_bounds__(kThreads) beam_pick_kernel(const __grid_constant__ BeamArgs a, const int cached) {
  chain_wait();
  extern __shared__ __align__(16) unsigned char smem_pick[];
  uint64_t* s_key = reinterpret_cast<uint64_t*>(smem_pick);              // [lists * k] if cached
  int32_t* s_tok = reinterpret_cast<int32_t*>(s_key + cached);           // [lists * k] if cached
  uint8_t* s_at = reinterpret_cast<uint8_t*>(s_tok + cached);            // [lists]: entries taken of each
  uint8_t* s_cnt = s_at + a.n_beams * a.n_slices;                        // [lists]: entries of each
  __shared__ double s_off[RTP_MAX_BEAMS];                  // score of a token with the row's largest logit
  __shared__ float s_max[RTP_MAX_BEAMS];                   // that logit
  __shared__ int s_state[RTP_MAX_BEAMS];                   // 1: ended, 2: all scores are -infinity
  __shared__ __align__(16) uint64_t s_top[kTops];
  __shared__ unsigned long long s_low;
  __shared__ int s_n;
  __shared__ uint4 s_few[kPickFew];                        // key, entry
  __shared__ uint4 s_best[2][kWarps];                      // score (ordered, 64 bits), list, token of each warp's best
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t row0 = (int64_t)blockIdx.x * a.n_beams;
  const int lists = a.n_beams * a.n_slices;
  // The lists are on their way while the normalisers are made.
  constexpr int kEarly = 4;
  const Cand* cand = a.cand + row0 * a.n_slices * a.k;
  Cand early[kEarly];
#pragma unroll
  for (int j = 0; j < kEarly; ++j) {
    const int e = tid + j * kThreads;
    early[j] = e < cached ? cand[e] : Cand{0.f, 0};
  }
  for (int l = tid; l < lists; l += kThreads) {
    const int b = l / a.n_slices, count = a.count[row0 * a.n_slices + l];
    s_at[l] = 0;
    s_cnt[l] = a.finished && a.finished[row0 + b] != 0 ? (l == b * a.n_slices) : (uint8_t)count;
  }
  for (int b = warp; b < a.n_beams; b += kWarps) {
    const int64_t row = row0 + b;
    const float2* st = a.stat + row * a.n_slices;
    const float2 first = lane < a.n_slices ? st[lane] : make_float2(-INFINITY, 0.f);   // (nothing of a row that has ended is used)
    double off = a.scores ? (double)a.scores[row] : 0.0;
    const bool ended = a.finished && a.finished[row] != 0;
    float m = first.x;
    for (int s = lane + 32; s < a.n_slices; s += 32) m = fmaxf(m, st[s].x);
    m = ended ? -INFINITY : warp_max(m);
    double z = 0.0;
    if (m != -INFINITY) {
      // (a term's error is 2^-22 of it, the difference's rounding included where the term counts)
      z = (double)first.y * (double)expf(first.x - m);
      for (int s = lane + 32; s < a.n_slices; s += 32) z += (double)st[s].y * (double)expf(st[s].x - m);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) z += __shfl_xor_sync(0xffffffffu, z, o);
    if (lane == 0) {
      if (!(off < (double)INFINITY)) {
        set_status(a.status, RTP_ERR_INVALID);
        off = -(double)INFINITY;
      }
      // (the maximum as it counts beside the score: what is left of the others is on the same grid, and no two sums become one)
      s_max[b] = counts_as(m, (float)off);
      s_state[b] = ended ? 1 : m == -INFINITY || off == -(double)INFINITY ? 2 : 0;
      if (!ended && m != -INFINITY) off -= log(z);
      s_off[b] = off;
    }
  }
  __syncthreads();
  auto entry = [&](int l, const Cand& c, int& token) -> uint64_t {   // of a list; keys order like scores
    const int b = l / a.n_slices;
    double score = s_off[b];
    if (s_state[b] == 1) {
      token = a.pad_token;
    } else {
      token = c.token;
      score = s_state[b] == 2 ? -(double)INFINITY : score + ((double)c.x - (double)s_max[b]);
    }
    const uint64_t u = (uint64_t)__double_as_longlong(score + 0.0);
    return (u >> 63) ? ~u : u | 0x8000000000000000ull;
  };
  if (cached) {
    uint64_t best = 0;                                     // the thread's best entry (no score has key 0)
    auto keep = [&](int e, const Cand& c) {
      const int l = e / a.k;
      const uint64_t key = e - l * a.k < s_cnt[l] ? entry(l, c, s_tok[e]) : 0ull;
      s_key[e] = key;
      best = max(best, key);
    };
#pragma unroll
    for (int j = 0; j < kEarly; ++j)
      if (tid + j * kThreads < cached) keep(tid + j * kThreads, early[j]);
    for (int e = tid + kEarly * kThreads; e < cached; e += kThreads) keep(e, cand[e]);
    // The k-th largest of 64 keys, each the best of four threads': what is among the k best reaches it, and little else does.
    uint64_t four = max(best, __shfl_xor_sync(0xffffffffu, best, 1));
    four = max(four, __shfl_xor_sync(0xffffffffu, four, 2));
    if ((lane & 3) == 0) s_top[tid >> 2] = four;
    if (tid == 0) {
      s_low = ~0ull;
      s_n = 0;
    }
    __syncthreads();
    int more = 0;                                          // keys above this one, a quarter of them in each of its threads
#pragma unroll
    for (int i = 0; i < kTops / 4; i += 2) {
      const ulonglong2 o = *reinterpret_cast<const ulonglong2*>(s_top + (lane & 3) * (kTops / 4) + i);
      more += (o.x > four) + (o.y > four);
    }
    more += __shfl_xor_sync(0xffffffffu, more, 1);
    more += __shfl_xor_sync(0xffffffffu, more, 2);
    const uint64_t mine = more < a.k ? four : ~0ull;
    const uint32_t h = __reduce_min_sync(0xffffffffu, (uint32_t)(mine >> 32));
    const uint32_t lo = __reduce_min_sync(0xffffffffu, (uint32_t)(mine >> 32) == h ? (uint32_t)mine : 0xffffffffu);
    if (lane == 0) atomicMin(&s_low, (unsigned long long)h << 32 | lo);
    __syncthreads();
    const uint64_t bound = max((uint64_t)s_low, (uint64_t)1);
    if (best >= bound)
      for (int e = tid; e < cached; e += kThreads)
        if (s_key[e] >= bound) {
          const int to = atomicAdd(&s_n, 1);
          if (to < kPickFew) s_few[to] = make_uint4((uint32_t)(s_key[e] >> 32), (uint32_t)s_key[e], (uint32_t)e, 0u);
        }
    __syncthreads();
    const int n = s_n;
    if (n <= kPickFew) {                                   // (else many are equal, and are taken one by one)
      for (int c = tid; c < n; c += kThreads) {
        const uint4 me = s_few[c];
        const uint64_t key = (uint64_t)me.x << 32 | me.y;
        int rank = 0;
#pragma unroll 4
        for (int o = 0; o < n; ++o) {
          const uint4 u = s_few[o];
          const uint64_t other = (uint64_t)u.x << 32 | u.y;
          rank += other > key || (other == key && u.z < me.z);
        }
        if (rank < a.k) {
          const int64_t at = (int64_t)blockIdx.x * a.k + rank;
          a.parent[at] = (int32_t)(row0 + me.z / (unsigned)a.k / (unsigned)a.n_slices);
          a.token[at] = s_tok[me.z];
          a.scores_out[at] = (float)score_of(key);
        }
      }
      for (int i = n + tid; i < a.k; i += kThreads) {
        const int64_t at = (int64_t)blockIdx.x * a.k + i;
        a.parent[at] = a.token[at] = -1;
        a.scores_out[at] = -INFINITY;
      }
      return;
    }
  }
  const int threads = lists <= 128 ? 32 : kThreads;        // that do the rounds
  if (tid >= threads) return;
  uint64_t best = 0;                                       // (no score has key 0)
  int best_l = 0x7fffffff, best_tok = 0;
  auto look = [&]() {
    best = 0;
    best_l = 0x7fffffff;
    for (int l = tid; l < lists; l += threads) {
      const int i = s_at[l];
      if (i >= s_cnt[l]) continue;
      int token = 0;
      const uint64_t key = cached ? s_key[l * a.k + i] : entry(l, s_state[l / a.n_slices] == 1 ? Cand{0.f, 0} : cand[l * a.k + i], token);
      if (key > best) {
        best = key;
        best_l = l;
        best_tok = cached ? s_tok[l * a.k + i] : token;
      }
    }
  };
  look();
  uint4 won = make_uint4(0, 0, 0, 0);                      // lane i: what round i, i + 32, .. chose
  for (int i = 0; i < a.k; ++i) {
    const uint32_t h = __reduce_max_sync(0xffffffffu, (uint32_t)(best >> 32));
    const uint32_t lo = __reduce_max_sync(0xffffffffu, (uint32_t)(best >> 32) == h ? (uint32_t)best : 0u);
    const int l = __reduce_min_sync(0xffffffffu, best == (((uint64_t)h << 32) | lo) ? best_l : 0x7fffffff);
    const int tok = __shfl_sync(0xffffffffu, best_tok, l & 31);
    uint4 win = make_uint4(h, lo, (uint32_t)l, (uint32_t)tok);
    if (threads > 32) {
      if (lane == 0) s_best[i & 1][warp] = win;
      __syncthreads();
      win = s_best[i & 1][0];
#pragma unroll
      for (int w = 1; w < kWarps; ++w) {
        const uint4 o = s_best[i & 1][w];
        const uint64_t ko = ((uint64_t)o.x << 32) | o.y, kw = ((uint64_t)win.x << 32) | win.y;
        if (ko > kw || (ko == kw && o.z < win.z)) win = o;
      }
    }
    const bool some = (win.x | win.y) != 0u;
    if (lane == (i & 31)) won = win;
    if (warp == 0 && ((i & 31) == 31 || i + 1 == a.k) && (i & ~31) + lane <= i) {
      const int64_t at = (int64_t)blockIdx.x * a.k + (i & ~31) + lane;
      const bool any = (won.x | won.y) != 0u;
      const double score = score_of(((uint64_t)won.x << 32) | won.y);
      a.parent[at] = any ? (int32_t)(row0 + won.z / a.n_slices) : -1;
      a.token[at] = any ? (int32_t)won.w : -1;
      a.scores_out[at] = any ? (float)score : -INFINITY;
    }
    if (some && (int)(win.z % threads) == tid) {
      s_at[win.z] += 1;
      look();
    }
  }
}

// How a row is cut: as many slices as make one wave of four CTAs per SM, each of two whole chunks at least (of one: 11.2 us instead of 9.1 for
// 15 rows of 50001 in 32 bits, whose second kernel then has twice the lists) and of 32 at most.  The latter keeps a row's normaliser right to
// 2^-16 however long it is: a thread then adds up 16 times, at 2^-24 for the sum and 2^-22 + 2^-24 for the factor where its maximum rose
// (2^-17.5 in all); a term's exponential is 2^-22 off, and its distance d from the maximum 2.3 x 2^-24 d (of 2^30 terms, those that count
// are at 18 on the average at most: 2^-18.6); sums within a step, over lanes and warps take 24 roundings of 2^-24, exponentials
// across warps and slices 2^-22 each.
constexpr int kMostChunks = 32;
struct BeamCut {
  int chunks, slices;                              // chunks per slice, slices per row
};
BeamCut beam_cut(int64_t rows, int64_t vocab, int bytes, int sm_count) {
  BeamCut c;
  const int64_t chunk = kThreads * 32 / bytes, chunks = (vocab + chunk - 1) / chunk;
  const int64_t want = std::max<int64_t>({1, std::min(chunks / 2, (int64_t)4 * sm_count / rows), (chunks + kMostChunks - 1) / kMostChunks});
  c.chunks = (int)((chunks + want - 1) / want);
  c.slices = (int)((chunks + c.chunks - 1) / c.chunks);
  return c;
}

template <class T>
cudaError_t launch_slices(const BeamArgs& a, int64_t rows, cudaStream_t st) {
  (void)launch_chained(beam_slice_kernel<T>, dim3((unsigned)(rows * a.n_slices)), dim3(kThreads), 0, st, a);
  return cudaGetLastError();
}

}  // namespace

size_t beam_workspace_bytes(int64_t rows, int64_t vocab, int k, int sm_count) {
  const int64_t lists = rows * std::max(beam_cut(rows, vocab, 4, sm_count).slices, beam_cut(rows, vocab, 2, sm_count).slices);
  return (size_t)lists * (k * sizeof(Cand) + sizeof(float2) + sizeof(int32_t)) + 2 * 256;
}

cudaError_t launch_beam_select(const void* logits, int format, int64_t row_stride, int64_t n_groups, int n_beams, int64_t vocab,
                               const float* scores, const int32_t* finished, int pad_token, int k, int32_t* parent, int32_t* token,
                               float* scores_out, void* ws, int32_t* status, int sm_count, cudaStream_t st) {
  const int64_t rows = n_groups * n_beams;
  const BeamCut cut = beam_cut(rows, vocab, format == RTP_LOGITS_F32 ? 4 : 2, sm_count);
  BeamArgs a = {logits, row_stride, n_beams, (int32_t)vocab, k, cut.slices, cut.chunks, pad_token, scores, finished,
                nullptr, nullptr, nullptr, parent, token, scores_out, status};
  const int64_t lists = rows * a.n_slices, group_lists = (int64_t)n_beams * a.n_slices;
  if (lists >= (int64_t)1 << 31) return cudaErrorNotSupported;
  char* p = reinterpret_cast<char*>(ws);
  a.cand = reinterpret_cast<Cand*>(p);
  p += ((size_t)lists * k * sizeof(Cand) + 255) & ~(size_t)255;
  a.stat = reinterpret_cast<float2*>(p);
  p += (size_t)lists * sizeof(float2);
  a.count = reinterpret_cast<int32_t*>(p);
  cudaError_t e = format == RTP_LOGITS_F32 ? launch_slices<float>(a, rows, st)
                  : format == RTP_LOGITS_BF16 ? launch_slices<__nv_bfloat16>(a, rows, st) : launch_slices<__half>(a, rows, st);
  if (e != cudaSuccess) return e;
  const int cached = group_lists * k <= kPickCached ? (int)(group_lists * k) : 0;
  const size_t smem = (size_t)cached * 12 + 2 * group_lists;
  if (smem > kPickCached * 12 + 2048) {            // (two bytes for each of up to 2^31 / 2^16 lists and one per beam: vocabularies of millions)
    static PerDeviceOnce once;
    e = set_dyn_smem_once(beam_pick_kernel, 2 * ((1 << 15) + RTP_MAX_BEAMS), once);
    if (e != cudaSuccess) return e;
  }
  (void)launch_chained(beam_pick_kernel, dim3((unsigned)n_groups), dim3(kThreads), smem, st, a, cached);
  return cudaGetLastError();
}

}  // namespace rtp
