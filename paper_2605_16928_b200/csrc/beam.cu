// Selection of a beam search step: the k best continuations of every group of beams, score = scores[beam] + log_softmax(logits)[token],
// equal scores going to the lower (beam, token).
//
// A row is cut into slices of whole chunks, one CTA each, whose threads hold the logits of a chunk in registers while the next ones are on
// their way; every thread keeps a running maximum and sum of exponentials of its own.  The slice's k best tokens need no sort of the
// chunks: in the first one, the k-th largest of the 256 threads' maxima is a lower bound of the k-th largest logit that only a few more
// than k logits reach.  Those go to a list, and of the later chunks only what lies above the list's bound.  A second kernel, one CTA per
// group, joins the rows' sums and takes the k best of the sorted lists one by one.
// Tokens of one row are ordered by their logits alone; where rows meet, scores are 64-bit (sums of exponentials are 32-bit
// within a slice, 64-bit across slices), so that neighbours are not swapped by the rounding of a normaliser.
// Bound by the one read of the logits in principle (10 us for 32 x 8 beams over 128K in bf16); measured 32.5 us: the slices 25.6, of which 5
// go by before the first list stands (loads of all CTAs at once, search, additions) and the rest is instruction issue and latency (210
// warp instructions per 512 logits, of which 16 are exponentials and about 60 the additions to the lists), the second kernel 8.
// 4 beams over 32K: 10 us, two launches of 4 and 7 us, chains of dependent loads, reductions and k rounds.
// Tried and left: pairs of chunks per step (fewer instructions, more than the instruction cache holds: 31 us for the slices), one copy of
// the chunk loop (27), groups that grow with the chunks seen (30), the second kernel launched ahead (no difference).
#include "rtp_device.cuh"

namespace rtp {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxEl = 16;               // logits of a chunk per thread
constexpr float kLog2e = 1.4426950408889634f;
constexpr int kSlack = 8;                // the search for the bound stops when that many threads too many reach it
// Threads whose maximum is above the bound: fewer than k + slack, and each may have all of its logits above it.
constexpr int kAdd = (RTP_MAX_BEAM_K + kSlack) * kMaxEl + RTP_MAX_BEAM_K;
constexpr int kKeep = 512;               // a list that is longer is cut to its k best before more is added
constexpr int kList = kKeep + kAdd;
constexpr int kShort = 64;               // lists that are ordered without a bound
constexpr int kSelect = 256;
constexpr int kTops = kThreads / 4;
static_assert(kTops >= RTP_MAX_BEAM_K, "a bound is the k-th of them");
constexpr int kGroup = 8;                // chunks between two barriers (the bound is that old)

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
__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f(__half x) { return __half2float(x); }

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
// The thread's largest logit; NaN is passed over (-infinity or NaN if there is nothing else).
template <int NV>
__device__ __forceinline__ float max_of(const uint4 (&w)[NV], float) {
  float m = __uint_as_float(w[0].x);
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const float a = fmaxf(__uint_as_float(w[v].x), __uint_as_float(w[v].y)), b = fmaxf(__uint_as_float(w[v].z), __uint_as_float(w[v].w));
    m = fmaxf(m, fmaxf(a, b));
  }
  return m;
}
template <class P, int NV>
__device__ __forceinline__ P max_pair(const uint4 (&w)[NV]) {
  P m = *reinterpret_cast<const P*>(&w[0].x);
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const P* p = reinterpret_cast<const P*>(&w[v]);
    m = __hmax2(m, __hmax2(__hmax2(p[0], p[1]), __hmax2(p[2], p[3])));
  }
  return m;
}
template <int NV>
__device__ __forceinline__ float max_of(const uint4 (&w)[NV], __nv_bfloat16) {
  const float2 f = __bfloat1622float2(max_pair<__nv_bfloat162>(w));
  return fmaxf(f.x, f.y);
}
template <int NV>
__device__ __forceinline__ float max_of(const uint4 (&w)[NV], __half) {
  const float2 f = __half22float2(max_pair<__half2>(w));
  return fmaxf(f.x, f.y);
}
// A thread's i-th logit, counted from its first one.
template <int EL, int VN>
__device__ __forceinline__ int token_of(int i) { return (i / VN) * kThreads * VN + i % VN; }
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
// m becomes the maximum of m and mine; returns the sum of exp(x - m).  Not below +infinity if one of x is NaN or +infinity.
// (The maximum is taken off first: the largest logit's term is 1 and nothing else, so that rows with one certain token each are equal,
// and the type's largest values times log2(e) would be no numbers.)
template <int EL>
__device__ __forceinline__ float weigh(const float (&x)[EL], float mine, float& m) {
  m = fmaxf(m, mine);
  const float off = m == -INFINITY ? 0.f : -m;
  const float2 o2 = make_float2(off, off), l2 = make_float2(kLog2e, kLog2e);
  float2 s0 = make_float2(0.f, 0.f), s1 = s0;
#pragma unroll
  for (int i = 0; i < EL; i += 4) {
    const float2 u = mul2(add2(make_float2(x[i], x[i + 1]), o2), l2), v = mul2(add2(make_float2(x[i + 2], x[i + 3]), o2), l2);
    s0 = add2(s0, make_float2(fast_ex2(u.x), fast_ex2(u.y)));
    s1 = add2(s1, make_float2(fast_ex2(v.x), fast_ex2(v.y)));
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
__device__ __forceinline__ uint4 ld_piece(const void* p) { return __ldg(reinterpret_cast<const uint4*>(p)); }

template <class T, int EL>
__global__ void __launch_bounds__(kThreads, 4) beam_slice_kernel(const __grid_constant__ BeamArgs a) {
  chain_wait();
  constexpr int VN = Vec<T>::n, NV = EL / VN, kChunk = kThreads * EL;
  static_assert(EL % VN == 0 && EL <= kMaxEl, "");
  __shared__ __align__(16) uint2 s_list[kList];    // ordered key, token
  __shared__ __align__(16) uint2 s_sel[kSelect];
  __shared__ uint2 s_best[RTP_MAX_BEAM_K];
  __shared__ __align__(16) uint32_t s_top[kTops];
  __shared__ uint32_t s_range[2];
  __shared__ float s_max[kWarps], s_sum[kWarps];
  __shared__ int s_n, s_sel_n, s_scan[kWarps];
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
  // no piece of the chunk reaches over an end of the row
  auto whole = [&](int c) { return skew ? c > 0 && (c + 1) * kChunk + VN <= a.vocab : (c + 1) * kChunk <= a.vocab; };
  auto load = [&](int c, uint4 (&w)[NV]) {          // the thread's pieces of chunk c of a row without skew
    const T* p = base + c * kChunk + tid * VN;
    if (whole(c)) {
#pragma unroll
      for (int v = 0; v < NV; ++v) w[v] = ld_stream_v4(p + v * kThreads * VN);
      return;
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int t0 = c * kChunk + tid * VN + v * kThreads * VN;
      if (t0 + VN <= a.vocab) {
        w[v] = ld_stream_v4(base + t0);
      } else {
        T e[VN];
#pragma unroll
        for (int i = 0; i < VN; ++i) e[i] = t0 + i < a.vocab ? base[t0 + i] : T(-INFINITY);
        w[v] = *reinterpret_cast<const uint4*>(e);
      }
    }
  };
  auto load_two = [&](int c, uint4 (&lo)[NV], uint4 (&hi)[NV]) {   // and of one with
    const T* p = base + c * kChunk + tid * VN - skew;
    if (whole(c)) {
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        lo[v] = ld_piece(p + v * kThreads * VN);
        hi[v] = ld_piece(p + v * kThreads * VN + VN);
      }
      return;
    }
#pragma unroll 1
    for (int v = 0; v < NV; ++v) {
      const int t0 = c * kChunk + tid * VN + v * kThreads * VN, first = t0 - skew;
      uint4 u[2];
      if (first >= 0 && first + 2 * VN <= a.vocab) {
        u[0] = ld_piece(base + first);
        u[1] = ld_piece(base + first + VN);
      } else {
        T e[2 * VN];
#pragma unroll
        for (int i = 0; i < 2 * VN; ++i) e[i] = first + i >= t0 && first + i < min(t0 + VN, a.vocab) ? base[first + i] : T(-INFINITY);
        u[0] = reinterpret_cast<const uint4*>(e)[0];
        u[1] = reinterpret_cast<const uint4*>(e)[1];
      }
#pragma unroll
      for (int y = 0; y < NV; ++y)
        if (y == v) {
          lo[y] = u[0];
          hi[y] = u[1];
        }
    }
  };
  if (tid == 0) s_n = 0;
  int n = 0;                                       // entries of the list (the same in all threads, like what follows)
  uint32_t least = 0;                              // a key that k entries of the list reach, once there are as many
  float m = -INFINITY, sum = 0.f;                  // this thread's
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
    if (n == a.k) least = max(least, s_best[a.k - 1].x);
    __syncthreads();
  };
  // Once the list has k entries, chunks go by in groups without a barrier: what is above the bound is added, up to the list's end.  A group
  // that would add more than there is room for (logits that rise along the row) is gone through again, chunk by chunk.
  uint4 w0[NV], w1[NV];                            // chunks c and c + 1; of a row with skew the two pieces of chunk c
  int c = c_lo, again_end = c_lo;                  // (the same in all threads, like n and least)
  auto fetch = [&]() {
    if (skew) {
      if (c < c_hi) load_two(c, w0, w1);
    } else {
      if (c < c_hi) load(c, w0);
      if (c + 1 < c_hi) load(c + 1, w1);
    }
  };
  // the chunk's logits out of their registers, and loads into those; returns the largest
  auto unpack_all = [&](float (&x)[EL], const uint4 (&u)[NV]) -> float {
#pragma unroll
    for (int v = 0; v < NV; ++v) unpack(u[v], x + v * VN, T());
    return max_of(u, T());
  };
  auto take_straight = [&](float (&x)[EL], uint4 (&w)[NV], int at_c) -> float {
    const float top = unpack_all(x, w);
    if (at_c + 2 < c_hi) load(at_c + 2, w);
    return top;
  };
  auto take_skewed = [&](float (&x)[EL], int at_c) -> float {
    uint4 u[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) u[v] = join<T>(w0[v], w1[v], skew);
    const float top = unpack_all(x, u);
    if (at_c + 1 < c_hi) load_two(at_c + 1, w0, w1);
    return top;
  };
  // few are added: they are read again, so that one short loop does for all places
  auto add = [&](int first, uint32_t mask) {
    while (mask) {
      const int t = first + token_of<EL, VN>(__ffs(mask) - 1);
      mask &= mask - 1;
      const float v = to_f(base[t]);
      const int to = atomicAdd(&s_n, 1);
      if (to < kList) s_list[to] = make_uint2(v < INFINITY ? okey(v + 0.f) : okey(-INFINITY), (uint32_t)t);
    }
  };
  // the thread's logits into its maximum and sum; returns the largest of them
  auto account = [&](float (&x)[EL], float mine) -> float {
    const float m_was = m;
    float part = weigh(x, mine, m);
    if (!(part < INFINITY)) {
      // a logit that is NaN or +infinity is none that can be chosen: as -infinity
      set_status(a.status, RTP_ERR_INVALID);
      mine = -INFINITY;
#pragma unroll
      for (int i = 0; i < EL; ++i) {
        if (!(x[i] < INFINITY)) x[i] = -INFINITY;
        mine = fmaxf(mine, x[i]);
      }
      m = m_was;
      part = weigh(x, mine, m);
    }
    sum = sum * fast_ex2((m_was - (m == -INFINITY ? 0.f : m)) * kLog2e) + part;   // (nothing yet: 0 * 0)
    return mine;
  };
  // a chunk of a group (logits behind the row's end are -infinity: not above any bound)
  auto stream = [&](float (&x)[EL], float top, int at_c, float at) {
    const float mine = account(x, top);
    if (mine > at) {
      uint32_t mask = 0;
#pragma unroll
      for (int i = 0; i < EL; ++i)
        if (x[i] > at) mask |= 1u << i;
      if ((mask & (mask - 1)) == 0) {              // mostly one: the largest
        const int to = atomicAdd(&s_n, 1);
        if (to < kList) s_list[to] = make_uint2(okey(mine + 0.f), (uint32_t)(at_c * kChunk + tid * VN + token_of<EL, VN>(__ffs(mask) - 1)));
      } else {
        add(at_c * kChunk + tid * VN, mask);
      }
    }
  };
  fetch();
#pragma unroll 1
  while (c < c_hi) {
    if (n >= a.k && c >= again_end) {
      const int begin = c, end = min(c + kGroup, c_hi);
      const float m_was = m, sum_was = sum, at = okey_to_float(max(least, okey(-INFINITY)));
      if (skew) {
#pragma unroll 1
        for (; c < end; ++c) {
          float x[EL];
          const float top = take_skewed(x, c);
          stream(x, top, c, at);
        }
      } else {
#pragma unroll 1
        for (; c < end; c += 2) {
          float x[EL];
          const float top = take_straight(x, w0, c);
          stream(x, top, c, at);
          if (c + 1 < end) {                       // (an odd group is the last one)
            float y[EL];
            const float top1 = take_straight(y, w1, c + 1);
            stream(y, top1, c + 1, at);
          }
        }
        c = end;
      }
      __syncthreads();
      const int have = s_n;
      __syncthreads();
      if (have > kList) {
        again_end = end;
        c = begin;
        m = m_was;
        sum = sum_was;
        if (tid == 0) s_n = n;
        fetch();
        __syncthreads();
        continue;
      }
      n = have;
      if (n > 2 * a.k + 16) cut();
      continue;
    }
    {
      float x[EL], mine;
      if (skew) {
        mine = take_skewed(x, c);
      } else {
        mine = take_straight(x, w0, c);        // (chunk c + 2 into w0, which then change places)
#pragma unroll
        for (int v = 0; v < NV; ++v) {
          const uint4 u = w0[v];
          w0[v] = w1[v];
          w1[v] = u;
        }
      }
      const int first = c * kChunk + tid * VN;     // token of the thread's first logit
      mine = account(x, mine);
      // keys order like the logits; 0: the thread has no token here (-infinity is a token that is ruled out)
      uint32_t valid = (1u << EL) - 1u;            // a bit for each of the thread's logits; pieces may reach over the row's ends
      if (!whole(c)) {
#pragma unroll
        for (int i = 0; i < EL; ++i)
          if (first + token_of<EL, VN>(i) >= a.vocab) valid &= ~(1u << i);
      }
      const uint32_t key = valid ? okey(mine + 0.f) : 0u;   // (-0 is 0)
      // the thread's logits of key `bound` and above; those above it
      auto from = [&](uint32_t bound) {
        const float at = bound <= okey(-INFINITY) ? -INFINITY : okey_to_float(bound);
        uint32_t mask = 0;
#pragma unroll
        for (int i = 0; i < EL; ++i)
          if (x[i] >= at) mask |= 1u << i;
        return mask & valid;
      };
      auto above = [&](uint32_t bound) {
        const float at = bound < okey(-INFINITY) ? -INFINITY : okey_to_float(bound);
        uint32_t mask = 0;
#pragma unroll
        for (int i = 0; i < EL; ++i)
          if (x[i] > at) mask |= 1u << i;
        return bound < okey(-INFINITY) ? valid : mask & valid;
      };
      if (n > kKeep) cut();
      const uint32_t bound = max(search(key), 1u);
      const uint32_t reach = key >= bound ? from(bound) : 0u, over = key >= bound ? above(bound) : 0u;
      const int w_reach = __reduce_add_sync(0xffffffffu, __popc(reach));
      __syncthreads();
      if (lane == 0) s_scan[warp] = w_reach;
      __syncthreads();
      int reached = 0;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) reached += s_scan[w];
      const bool all = reached <= kAdd;            // else too many equal the bound: the first of them are taken in order
      add(first, all ? reach : over);
      __syncthreads();
      const int added = s_n - n;
      n = s_n;
      if (!all && added < a.k) {
        const int need = a.k - added;
        int before = 0;                            // equal ones in front of this piece
#pragma unroll 1
        for (int v = 0; v < NV; ++v) {
          uint32_t eq = ((reach & ~over) >> (v * VN)) & ((1u << VN) - 1u);
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
          int at = before + s - cnt, total = 0;
#pragma unroll
          for (int w = 0; w < kWarps; ++w) {
            at += w < warp ? s_scan[w] : 0;
            total += s_scan[w];
          }
          for (; eq; eq &= eq - 1, ++at)
            if (at < need) s_list[n + at] = make_uint2(bound, (uint32_t)(first + v * kThreads * VN + __ffs(eq) - 1));
          before += total;
          if (before >= need) break;               // (the same in all threads)
        }
        n += min(before, need);
        __syncthreads();
        if (tid == 0) s_n = n;
      }
      if (reached >= a.k) least = max(least, bound);
      else if (n >= a.k) cut();                    // (short chunks: their entries' k-th best)
      __syncthreads();
    }
    ++c;
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

// One CTA per group.  The rows' normalisers, then all lists as 64-bit scores in shared memory where they fit, then k rounds in which every
// lane knows the best of the lists list = thread, thread + threads, ...; a single warp does the rounds where 32 lanes have few lists each.
// Lists are in the order of (beam, token): the slices of a row hold disjoint, ascending ranges of tokens, and a list is sorted.  So of
// equal scores the lower list goes first.
constexpr int kPickCached = 3400;                  // entries in shared memory
__global__ void __launch_bounds__(kThreads) beam_pick_kernel(const __grid_constant__ BeamArgs a, const int cached) {
  chain_wait();
  extern __shared__ __align__(16) unsigned char smem_pick[];
  uint64_t* s_key = reinterpret_cast<uint64_t*>(smem_pick);              // [lists * k] if cached
  int32_t* s_tok = reinterpret_cast<int32_t*>(s_key + cached);           // [lists * k] if cached
  uint8_t* s_at = reinterpret_cast<uint8_t*>(s_tok + cached);            // [lists]: entries taken of each
  uint8_t* s_cnt = s_at + a.n_beams * a.n_slices;                        // [lists]: entries of each
  __shared__ double s_off[RTP_MAX_BEAMS];                  // score of a token with the row's largest logit
  __shared__ float s_max[RTP_MAX_BEAMS];                   // that logit
  __shared__ int s_state[RTP_MAX_BEAMS];                   // 1: ended, 2: no token has a probability
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
      s_state[b] = ended ? 1 : m == -INFINITY ? 2 : 0;
      if (!ended && m != -INFINITY) off -= log(z);
      s_off[b] = off;
      s_max[b] = m;
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
    auto keep = [&](int e, const Cand& c) {
      const int l = e / a.k;
      if (e - l * a.k < s_cnt[l]) s_key[e] = entry(l, c, s_tok[e]);
    };
#pragma unroll
    for (int j = 0; j < kEarly; ++j)
      if (tid + j * kThreads < cached) keep(tid + j * kThreads, early[j]);
    for (int e = tid + kEarly * kThreads; e < cached; e += kThreads) keep(e, cand[e]);
    __syncthreads();
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
      const uint64_t u = ((uint64_t)won.x << 32) | won.y;
      const double score = __longlong_as_double((long long)((u >> 63) ? u & 0x7fffffffffffffffull : ~u));
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

// How a row is cut: chunks of 4096 logits, of 2048 if they are 32-bit or in calls that would leave SMs idle; and as many slices as make one wave of four CTAs
// per SM, each of whole chunks.
struct BeamCut {
  int el, chunks, slices;                          // logits per thread and chunk, chunks per slice, slices per row
};
BeamCut beam_cut(int64_t rows, int64_t vocab, bool wide, int sm_count) {
  BeamCut c;
  c.el = !wide && rows * vocab >= (int64_t)sm_count * kThreads * 32 ? 16 : 8;
  const int64_t chunks = (vocab + (int64_t)kThreads * c.el - 1) / ((int64_t)kThreads * c.el);
  const int64_t want = std::max<int64_t>(1, std::min(chunks, (int64_t)4 * sm_count / rows));
  c.chunks = (int)((chunks + want - 1) / want);
  c.slices = (int)((chunks + c.chunks - 1) / c.chunks);
  return c;
}

template <class T>
cudaError_t launch_slices(const BeamArgs& a, int el, int64_t rows, cudaStream_t st) {
  const dim3 grid((unsigned)(rows * a.n_slices)), block(kThreads);
  auto kernel = beam_slice_kernel<T, 8>;
  if constexpr (sizeof(T) == 2)
    if (el == 16) kernel = beam_slice_kernel<T, 16>;
  (void)launch_chained(kernel, grid, block, 0, st, a);
  return cudaGetLastError();
}

}  // namespace

size_t beam_workspace_bytes(int64_t rows, int64_t vocab, int k, int sm_count) {
  const int64_t lists = rows * std::max(beam_cut(rows, vocab, false, sm_count).slices, beam_cut(rows, vocab, true, sm_count).slices);
  return (size_t)lists * (k * sizeof(Cand) + sizeof(float2) + sizeof(int32_t)) + 2 * 256;
}

cudaError_t launch_beam_select(const void* logits, int format, int64_t row_stride, int64_t n_groups, int n_beams, int64_t vocab,
                               const float* scores, const int32_t* finished, int pad_token, int k, int32_t* parent, int32_t* token,
                               float* scores_out, void* ws, int32_t* status, int sm_count, cudaStream_t st) {
  const int64_t rows = n_groups * n_beams;
  const BeamCut cut = beam_cut(rows, vocab, format == RTP_LOGITS_F32, sm_count);
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
  cudaError_t e = format == RTP_LOGITS_F32 ? launch_slices<float>(a, cut.el, rows, st)
                  : format == RTP_LOGITS_BF16 ? launch_slices<__nv_bfloat16>(a, cut.el, rows, st) : launch_slices<__half>(a, cut.el, rows, st);
  if (e != cudaSuccess) return e;
  const int cached = group_lists * k <= kPickCached ? (int)(group_lists * k) : 0;
  (void)launch_chained(beam_pick_kernel, dim3((unsigned)n_groups), dim3(kThreads), (size_t)cached * 12 + 2 * group_lists, st, a, cached);
  return cudaGetLastError();
}

}  // namespace rtp
