// Pages of a cache: copies, sequences that share pages (fork), room for new tokens with copies of shared pages that are going
// to be written (reserve), release (free) and the move of all used pages to the front of the pool (compact).
//
// A page is free iff its reference count is zero, so there is no other state to keep in step: the free pages in the order of
// their numbers are found by a scan over the counts (4 bytes a page: 64 KB for a pool of 16K pages, which one CTA reads from
// L2 in a few microseconds), and what a call hands out does not depend on the order in which threads arrive.  Decisions that
// need an order are taken by one CTA; page contents, the only bytes that matter, are then copied by all SMs.
// Measured: 64 sequences of 32K tokens freed, forked and given 200 tokens each in 19 us (a chain of dependent reads of L2 in four
// small kernels), 3001 of 16384 pages (0.8 GB) moved in 247 us (6.5 TB/s, the rate of a plain copy).
#include <type_traits>

#include "rtp_device.cuh"

namespace rtp {

namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanWarps = kPlanThreads / 32;
constexpr int kEarlyPages = kPlanWarps * 8 * 128;
constexpr int kRowThreads = 256;
constexpr int kRowVec = 4;                                        // table entries in flight per thread
// Bytes of a page that a CTA copies at a time: its threads x 16-byte loads in flight per thread.  A few pages (the copies of
// a reserve call, 64 pages) are spread over more SMs by small CTAs; a long move runs better in large ones whose stores do
// not stay in L2 (1.6 GB moved: 265 us with 256 x 8, 256 with 512 x 4, 250 with 1024 x 4, and 247 = 6.5 TB/s with 32 CTAs per SM
// in the grid instead of 8: the last pieces are dealt more evenly).
struct SmallCopy {
  static constexpr int kThreads = 256, kVec = 8;
  static constexpr bool kStream = false;
};
struct LargeCopy {
  static constexpr int kThreads = 1024, kVec = 4;
  static constexpr bool kStream = true;
};
template <class C>
constexpr int kPieceOf = C::kThreads * C::kVec * 16;

// Workspace: counts and the verdicts of the table checks (256 bytes), then lists.
constexpr int kCheckMax = 60;    // CTAs that look through the table before a compaction
constexpr int kCheckVec = 4;     // table entries in flight per thread
struct PlanHead {
  int32_t n_pairs, n_used;
  int32_t bad[kCheckMax];
};
static_assert(sizeof(PlanHead) <= 256, "the lists begin 256 bytes into the workspace");

__device__ __forceinline__ bool page_ok(int p, int num_pages) { return (unsigned)p < (unsigned)num_pages; }

// ---- contents ------------------------------------------------------------------------------------
// Copies piece `piece` (counted over the arrays of a page) of page src to page dst.
template <class C>
__device__ __forceinline__ void copy_piece(const PageArrays& pa, int64_t src, int64_t dst, int piece) {
  int a = 0;
#pragma unroll
  for (; a < kPageArrays - 1; ++a) {
    if (piece < pa.pieces[a]) break;
    piece -= pa.pieces[a];
  }
  const char* s = pa.base[a] + src * pa.bytes[a];
  char* d = pa.base[a] + dst * pa.bytes[a];
  constexpr int kStep = C::kThreads * 16;
  const int64_t at = (int64_t)piece * kPieceOf<C> + threadIdx.x * 16;
  uint4 v[C::kVec];
#pragma unroll
  for (int i = 0; i < C::kVec; ++i)
    if (at + i * kStep < pa.bytes[a]) v[i] = ld_stream_v4(s + at + i * kStep);
#pragma unroll
  for (int i = 0; i < C::kVec; ++i)
    if (at + i * kStep < pa.bytes[a]) {
      uint4* to = reinterpret_cast<uint4*>(d + at + i * kStep);
      if (C::kStream) __stcs(to, v[i]); else *to = v[i];
    }
}

// n pairs given by the caller, or as many as head->n_pairs says.
__global__ void __launch_bounds__(SmallCopy::kThreads) copy_pages_kernel(const __grid_constant__ PageArrays pa, const int num_pages,
                                                                  const int32_t* __restrict__ src,
                                                                  const int32_t* __restrict__ dst, const int n,
                                                                  const PlanHead* __restrict__ head, int32_t* status) {
  chain_wait();
  const unsigned pieces = pa.total_pieces, total = (head ? head->n_pairs : n) * pieces;   // (below 2^31: checked by the caller)
  for (unsigned u = blockIdx.x; u < total; u += gridDim.x) {
    const unsigned i = u / pieces;
    const int s = src[i], d = dst[i];
    if (!page_ok(s, num_pages) || !page_ok(d, num_pages)) {
      if (threadIdx.x == 0) set_status(status, RTP_ERR_INVALID);
      continue;
    }
    if (s != d) copy_piece<SmallCopy>(pa, s, d, (int)(u - i * pieces));
  }
}

// ---- fork, free: one CTA per sequence -------------------------------------------------------------
__global__ void __launch_bounds__(kRowThreads) fork_kernel(int32_t* __restrict__ table, int32_t* __restrict__ seq_lens,
                                                           int32_t* __restrict__ refs, const int num_pages, const int batch,
                                                           const int max_pages, const int32_t* __restrict__ src_seqs,
                                                           const int32_t* __restrict__ dst_seqs, const int n, int32_t* status) {
  chain_wait();
  const int i = blockIdx.x, src = src_seqs[i], dst = dst_seqs[i];
  bool bad = (unsigned)src >= (unsigned)batch || (unsigned)dst >= (unsigned)batch;
  // named as a destination before, or a source that is somebody's destination: what it holds would depend on the order
  for (int j = threadIdx.x; j < n; j += kRowThreads) bad = bad || (j < i && dst_seqs[j] == dst) || dst_seqs[j] == src;
  if (__syncthreads_or(bad)) {
    if (threadIdx.x == 0) set_status(status, RTP_ERR_INVALID);
    return;
  }
  const int len = seq_lens[src];
  const int np = len < 0 ? 0 : (int)(((int64_t)len + kPage - 1) >> kPageShift);
  const int32_t* from = table + (int64_t)src * max_pages;
  int32_t* to = table + (int64_t)dst * max_pages;
  bad = len < 0 || np > max_pages || seq_lens[dst] != 0;
  if (!bad)
    for (int p0 = threadIdx.x; p0 < max_pages; p0 += kRowThreads * kRowVec) {   // (loads of a step side by side)
      int e[kRowVec], t[kRowVec];
#pragma unroll
      for (int k = 0; k < kRowVec; ++k) {
        const int p = p0 + k * kRowThreads;
        e[k] = p < np ? from[p] : -1;
        t[k] = p < max_pages ? to[p] : -1;
      }
#pragma unroll
      for (int k = 0; k < kRowVec; ++k) {
        bad = bad || t[k] >= 0;
        if (p0 + k * kRowThreads < np) bad = bad || !page_ok(e[k], num_pages) || refs[e[k]] <= 0;
      }
    }
  if (__syncthreads_or(bad)) {
    if (threadIdx.x == 0) set_status(status, RTP_ERR_INVALID);
    return;
  }
  for (int p = threadIdx.x; p < np; p += kRowThreads) {
    const int e = from[p];
    to[p] = e;
    atomicAdd(refs + e, 1);
  }
  if (threadIdx.x == 0) seq_lens[dst] = len;
}

__global__ void __launch_bounds__(kRowThreads) free_kernel(int32_t* __restrict__ table, int32_t* __restrict__ seq_lens,
                                                           int32_t* __restrict__ refs, const int num_pages, const int batch,
                                                           const int max_pages, const int32_t* __restrict__ seqs,
                                                           int32_t* status) {
  chain_wait();
  const int seq = seqs[blockIdx.x];
  if ((unsigned)seq >= (unsigned)batch) {
    if (threadIdx.x == 0) set_status(status, RTP_ERR_INVALID);
    return;
  }
  int32_t* row = table + (int64_t)seq * max_pages;
  for (int p0 = threadIdx.x; p0 < max_pages; p0 += kRowThreads * kRowVec) {   // (requests of a step side by side)
    int e[kRowVec], held[kRowVec];
#pragma unroll
    for (int k = 0; k < kRowVec; ++k) e[k] = p0 + k * kRowThreads < max_pages ? row[p0 + k * kRowThreads] : -1;
#pragma unroll
    for (int k = 0; k < kRowVec; ++k)   // (a sequence named twice gives each page back once)
      if (e[k] >= 0) e[k] = atomicExch(row + p0 + k * kRowThreads, -1);
#pragma unroll
    for (int k = 0; k < kRowVec; ++k) held[k] = e[k] >= 0 && page_ok(e[k], num_pages) ? atomicSub(refs + e[k], 1) : 0;
#pragma unroll
    for (int k = 0; k < kRowVec; ++k) {
      if (e[k] < 0 || held[k] > 0) continue;
      if (page_ok(e[k], num_pages)) atomicAdd(refs + e[k], 1);   // nobody held it
      set_status(status, RTP_ERR_INVALID);
    }
  }
  if (threadIdx.x == 0) seq_lens[seq] = 0;
}

// ---- the scan over the reference counts ------------------------------------------------------------
// The pool is cut into one contiguous segment per warp of the CTA, a multiple of 128 pages (four per lane).
struct Segment {
  int lo, hi;
};
__device__ __forceinline__ Segment warp_segment(int num_pages, int warp) {
  const int64_t per = (((int64_t)num_pages + kPlanWarps - 1) / kPlanWarps + 127) / 128 * 128;
  const int64_t lo = per * warp, hi = lo + per;
  return {(int)(lo < num_pages ? lo : num_pages), (int)(hi < num_pages ? hi : num_pages)};
}
// Bit j: page at + 4 lane + j is in use; pages at or beyond hi are not.
__device__ __forceinline__ uint32_t used_bits(const int32_t* refs, int at, int hi, int lane) {
  const int p = at + 4 * lane;
  uint32_t b = 0;
  if (p + 3 < hi) {
    const int4 v = *reinterpret_cast<const int4*>(refs + p);
    b = (v.x != 0 ? 1u : 0u) | (v.y != 0 ? 2u : 0u) | (v.z != 0 ? 4u : 0u) | (v.w != 0 ? 8u : 0u);
  } else {
    for (int j = 0; j < 4; ++j)
      if (p + j < hi && refs[p + j] != 0) b |= 1u << j;
  }
  return b;
}
__device__ __forceinline__ int count_used(const int32_t* refs, int lo, int hi, int lane) {
  int n = 0;
#pragma unroll 4
  for (int at = lo; at < hi; at += 128) n += __popc(used_bits(refs, at, hi, lane));
  return __reduce_add_sync(0xffffffffu, n);
}
__device__ __forceinline__ int lanes_before(int x, int lane) {   // exclusive sum over the warp
  int s = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += y;
  }
  return s - x;
}
// Used pages before each warp's segment; returns those of the whole pool.  Called by the whole CTA.
__device__ __forceinline__ int scan_segments(int mine, int* s_before, int lane, int warp) {
  if (lane == 0) s_before[warp] = mine;
  __syncthreads();
  if (warp == 0) {
    const int x = s_before[lane], b = lanes_before(x, lane);
    __syncwarp();
    s_before[lane] = b;
    if (lane == 31) s_before[32] = b + x;
  }
  __syncthreads();
  return s_before[32];
}

// ---- reserve -----------------------------------------------------------------------------------------
constexpr int kListMax = 4096;
struct ReserveShared {
  int seq[kReserveMax];       // -1: the entry asks for nothing
  int len[kReserveMax], add[kReserveMax];
  int held[kReserveMax];      // references of `cow`
  int cow[kReserveMax];       // shared page that the sequence is going to write into, or -1
  int first[kReserveMax];     // first table entry that has to be filled
  int off[kReserveMax + 1];   // pages handed out before this entry's
  int before[33];
  int n_pairs;
  unsigned long long total;
  int page[kListMax];         // the free pages that are handed out, if they are not many
};

// How many of v[0 .. i - 1] equal v[i] (v 16-byte aligned), counted by `width` (a power of two up to 32) neighbouring lanes.
__device__ __forceinline__ int earlier_equal(const int* v, int i, int width, int lane) {
  const int x = v[i], sub = lane & (width - 1);
  int n = 0;
  for (int j = 4 * sub; j < i; j += 4 * width) {
    const int4 y = *reinterpret_cast<const int4*>(v + j);
    n += (y.x == x) + (y.y == x && j + 1 < i) + (y.z == x && j + 2 < i) + (y.w == x && j + 3 < i);
  }
  const uint32_t lanes = (width == 32 ? 0xffffffffu : (1u << width) - 1u) << (lane - sub);
  return __reduce_add_sync(lanes, n);
}

__global__ void __launch_bounds__(kPlanThreads) reserve_kernel(int32_t* __restrict__ table, const int32_t* __restrict__ seq_lens,
                                                               int32_t* __restrict__ refs, const int num_pages, const int batch,
                                                               const int max_pages, const int32_t* __restrict__ seqs,
                                                               const int32_t* __restrict__ n_tokens, const int n,
                                                               PlanHead* __restrict__ head, int32_t* __restrict__ pair_src,
                                                               int32_t* __restrict__ pair_dst, int32_t* status) {
  chain_wait();
  extern __shared__ __align__(16) unsigned char smem_reserve[];
  ReserveShared& s = *reinterpret_cast<ReserveShared*>(smem_reserve);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) {
    s.n_pairs = 0;
    s.total = 0;
  }
  // Pools of up to 32K pages: every lane asks for its reference counts first, next to the requests, and keeps four bits for
  // each of up to eight pieces of its warp's segment.
  const Segment seg = warp_segment(num_pages, warp);
  const bool early = num_pages <= kEarlyPages;
  uint32_t used4 = 0;
  if (early) {
#pragma unroll
    for (int k = 0; k < 8; ++k) used4 |= (seg.lo + 128 * k < seg.hi ? used_bits(refs, seg.lo + 128 * k, seg.hi, lane) : 0u) << (4 * k);
  }
  bool invalid = false, full = false, shared_page = false, many = false;
  for (int i = tid; i < n; i += kPlanThreads) {
    const int seq = seqs[i], add = n_tokens[i];
    const int len = (unsigned)seq < (unsigned)batch ? seq_lens[seq] : -1;
    const bool ok = add >= 0 && len >= 0;
    invalid = invalid || !ok;
    many = many || (ok && add > 32 * kPage);
    s.seq[i] = ok ? seq : -1;
    s.len[i] = len;
    s.add[i] = add;
  }
  many = __syncthreads_or(many);
  int width = 1;   // lanes that compare one request with the earlier ones
  while (width < 32 && 2 * width * n <= kPlanThreads) width *= 2;
  for (int i = tid / width; i < n; i += kPlanThreads / width) {
    const bool twice = earlier_equal(s.seq, i, width, lane) > 0;
    if ((lane & (width - 1)) == 0) s.first[i] = twice && s.seq[i] >= 0;
  }
  __syncthreads();
  for (int i = tid; i < n; i += kPlanThreads)   // a sequence named twice: the first one counts
    if (s.first[i]) {
      s.seq[i] = -1;
      invalid = true;
    }
  __syncthreads();
  // The table entries from a sequence's length up to what it is going to need: eight lanes per sequence, a warp where somebody
  // asks for more than 32 pages.
  auto look_at_rows = [&](auto width) {
    constexpr int W = decltype(width)::value;
    const uint32_t lanes = W == 32 ? 0xffffffffu : ((1u << (W & 31)) - 1u) << (lane / W * W);
    const int sub = lane % W;
    for (int i = tid / W; i < n; i += kPlanThreads / W) {
      const int seq = s.seq[i];
      int need = 0, cow = -1, first = 0, held = 0;
      if (seq >= 0) {
        const int64_t len = s.len[i], end = len + s.add[i];
        const int64_t want = (end + kPage - 1) >> kPageShift;
        const int32_t* row = table + (int64_t)seq * max_pages;
        if (want > max_pages) {
          full = true;
        } else {
          bool bad = false;
          int mapped = 0;
          first = (int)((len + kPage - 1) >> kPageShift);
          const bool part = s.add[i] > 0 && (len & (kPage - 1));
          const int last = part ? row[len >> kPageShift] : -1;   // (requested together with the entries below)
          for (int p = first + sub; p < want; p += W) {   // mapped entries come first, then unmapped ones
            const int e = row[p];
            const bool m = e >= 0;
            mapped += m;
            bad = bad || (m && p > first && row[p - 1] < 0);
            // (held by others: their tokens would be written over; held by nobody: it may be handed out to another sequence)
            bad = bad || (m && (!page_ok(e, num_pages) || refs[e] != 1));
          }
          mapped = __reduce_add_sync(lanes, mapped);
          first += mapped;
          need = (int)want - first;
          if (need < 0) need = 0;
          if (part) {
            if (!page_ok(last, num_pages)) bad = true;
            else held = refs[last];
            if (held <= 0) bad = true;
            if (held > 1) cow = last;
          }
          if (__any_sync(lanes, bad)) {
            invalid = true;
            need = 0;
            cow = -1;
            if (sub == 0) s.seq[i] = -1;
          }
        }
      }
      if (sub == 0) {
        s.first[i] = first;
        s.cow[i] = cow;
        s.held[i] = held;
        s.off[i] = need;
      }
      shared_page = shared_page || cow >= 0;
    }
  };
  if (many) look_at_rows(std::integral_constant<int, 32>()); else look_at_rows(std::integral_constant<int, 8>());
  if (__syncthreads_or(shared_page)) {
    // A page with r holders is copied by the first r - 1 of them at most: the last one to write it has it alone.
    for (int i = tid / width; i < n; i += kPlanThreads / width) {
      const int earlier = earlier_equal(s.cow, i, width, lane);
      if ((lane & (width - 1)) == 0) s.add[i] = s.cow[i] < 0 ? 0 : s.held[i] - earlier > 1 ? 1 : -1;
    }
    __syncthreads();
    for (int i = tid; i < n; i += kPlanThreads) {
      if (s.add[i] > 0) s.off[i] += 1;
      if (s.add[i] < 0) s.cow[i] = -1;
    }
  }
  __syncthreads();
  // exclusive sums of the needs: thread t takes entries t * per ..
  const int per = (n + kPlanThreads - 1) / kPlanThreads;
  int sum = 0;
  unsigned long long wide = 0;
  for (int k = 0; k < per; ++k) {
    const int i = tid * per + k;
    if (i < n) {
      const int x = s.off[i];
      s.off[i] = sum;
      sum += x;
      wide += x;
    }
  }
  if ((int64_t)n * max_pages >= (int64_t)1 << 30) atomicAdd(&s.total, wide);   // (the sum in 32 bits could wrap)
  const int in_warp = lanes_before(sum, lane);
  const int total = scan_segments(__shfl_sync(0xffffffffu, in_warp + sum, 31), s.before, lane, warp);
  for (int k = 0; k < per; ++k) {
    const int i = tid * per + k;
    if (i < n) s.off[i] += s.before[warp] + in_warp;
  }
  if (tid == 0) s.off[n] = total;
  if (invalid) set_status(status, RTP_ERR_INVALID);
  if (__syncthreads_or(full) || s.total > (unsigned)num_pages) {   // a row or the pool is too short: nothing is handed out
    if (tid == 0) {
      set_status(status, RTP_ERR_CAPACITY);
      head->n_pairs = 0;
    }
    return;
  }
  if (total > 0) {
    const int used = early ? __reduce_add_sync(0xffffffffu, __popc(used4)) : count_used(refs, seg.lo, seg.hi, lane);
    const int all_used = scan_segments(used, s.before, lane, warp);
    if (num_pages - all_used < total) {   // not enough free pages: nothing is handed out
      if (tid == 0) {
        set_status(status, RTP_ERR_CAPACITY);
        head->n_pairs = 0;
      }
      return;
    }
    // page number `page` is the u-th that is handed out
    auto hand_out = [&](int u, int page) {
      int a = 0, b = n;   // the last entry with off <= u
      while (a + 1 < b) {
        const int mid = (a + b) >> 1;
        if (s.off[mid] <= u) a = mid; else b = mid;
      }
      const int cow = s.cow[a], k = u - s.off[a];
      int32_t* row = table + (int64_t)s.seq[a] * max_pages;
      refs[page] = 1;
      if (cow >= 0 && k == 0) {
        atomicSub(refs + cow, 1);
        row[s.len[a] >> kPageShift] = page;
        const int slot = atomicAdd(&s.n_pairs, 1);
        pair_src[slot] = cow;
        pair_dst[slot] = page;
      } else {
        row[s.first[a] + k - (cow >= 0)] = page;
      }
    };
    const bool listed = total <= kListMax;   // a list first, so that every thread then hands out its own
    int rank = seg.lo - s.before[warp];      // free pages before this segment
    for (int at = seg.lo; at < seg.hi && rank < total; at += 128) {
      const int valid = min(4, max(0, seg.hi - (at + 4 * lane)));
      const uint32_t used_here = early ? used4 >> ((at - seg.lo) / 128 * 4) : used_bits(refs, at, seg.hi, lane);
      const uint32_t free_bits = ~used_here & ((1u << valid) - 1u);
      const int cnt = __popc(free_bits);
      int u = rank + lanes_before(cnt, lane);
      for (int j = 0; j < 4; ++j) {
        if (!((free_bits >> j) & 1u)) continue;
        if (u < total) {
          if (listed) s.page[u] = at + 4 * lane + j; else hand_out(u, at + 4 * lane + j);
        }
        ++u;
      }
      rank += __reduce_add_sync(0xffffffffu, cnt);
    }
    if (listed) {
      __syncthreads();
      for (int u = tid; u < total; u += kPlanThreads) hand_out(u, s.page[u]);
    }
  }
  __syncthreads();
  if (tid == 0) head->n_pairs = s.n_pairs;
}

// ---- compact -----------------------------------------------------------------------------------------
// With n_used pages in use, the k-th used page at or above n_used goes to the k-th free page below it.  That is CTA 0's work;
// the others look meanwhile for table entries that name a page without references (one below n_used would be filled with somebody
// else's tokens, which its row would then read, and give away when it is freed) or no page at all, and leave a verdict each.
// A call that finds nothing to move takes 13 us for a pool of 1K pages and 17 for one of 16K (of which most is the grid of the move),
// 34 with a table of 4 M entries.
__global__ void __launch_bounds__(kPlanThreads) compact_plan_kernel(const int32_t* __restrict__ table, const int64_t n_entries,
                                                                    const int32_t* __restrict__ refs, const int num_pages,
                                                                    PlanHead* __restrict__ head, int32_t* __restrict__ src,
                                                                    int32_t* __restrict__ dst, int32_t* __restrict__ move,
                                                                    int32_t* __restrict__ n_used_out) {
  chain_wait();
  if (blockIdx.x > 0) {
    const int64_t step = (int64_t)(gridDim.x - 1) * kPlanThreads;
    bool bad = false;
    for (int64_t i = (int64_t)(blockIdx.x - 1) * kPlanThreads + threadIdx.x; i < n_entries; i += step * kCheckVec) {
      int e[kCheckVec];   // (loads of a step side by side)
#pragma unroll
      for (int k = 0; k < kCheckVec; ++k) e[k] = i + k * step < n_entries ? table[i + k * step] : -1;
#pragma unroll
      for (int k = 0; k < kCheckVec; ++k)
        if (e[k] >= 0) bad = bad || !page_ok(e[k], num_pages) || refs[e[k]] <= 0;
    }
    bad = __syncthreads_or(bad);
    if (threadIdx.x == 0) head->bad[blockIdx.x - 1] = bad;
    return;
  }
  __shared__ int s_before[33], s_below;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const Segment seg = warp_segment(num_pages, warp);
  if (threadIdx.x == 0) s_below = 0;
  const int n_used = scan_segments(count_used(refs, seg.lo, seg.hi, lane), s_before, lane, warp);
  if (seg.lo < n_used) {
    const int below = count_used(refs, seg.lo, min(seg.hi, n_used), lane);
    if (lane == 0) atomicAdd(&s_below, below);
  }
  __syncthreads();
  const int below = s_below;   // used pages that stay
  int before = s_before[warp];
  for (int at = seg.lo; at < seg.hi; at += 128) {
    const uint32_t used = used_bits(refs, at, seg.hi, lane);
    const int cnt = __popc(used);
    int u = before + lanes_before(cnt, lane);   // used pages before page p
    for (int j = 0; j < 4; ++j) {
      const int p = at + 4 * lane + j;
      if (p >= seg.hi) break;
      const bool is_used = (used >> j) & 1u;
      if (p < n_used) {
        if (!is_used) dst[p - u] = p;
      } else {
        move[p] = is_used ? u - below : -1;
        if (is_used) src[u - below] = p;
      }
      u += is_used;
    }
    before += __reduce_add_sync(0xffffffffu, cnt);
  }
  if (threadIdx.x == 0) {
    head->n_pairs = n_used - below;
    head->n_used = n_used;
    *n_used_out = n_used;
  }
}

__global__ void __launch_bounds__(LargeCopy::kThreads) compact_move_kernel(const __grid_constant__ PageArrays pa, const int num_pages,
                                                                    int32_t* __restrict__ table, const int64_t n_entries,
                                                                    int32_t* __restrict__ refs, const PlanHead* __restrict__ head,
                                                                    const int n_checks, const int32_t* __restrict__ src,
                                                                    const int32_t* __restrict__ dst,
                                                                    const int32_t* __restrict__ move,
                                                                    int32_t* __restrict__ n_used_out, int32_t* status) {
  chain_wait();
  if (__syncthreads_or(threadIdx.x < n_checks && head->bad[threadIdx.x])) {   // the table is wrong: nothing moves, no page may be cut
    if (blockIdx.x == 0 && threadIdx.x == 0) {
      set_status(status, RTP_ERR_INVALID);
      *n_used_out = num_pages;
    }
    return;
  }
  const int n_pairs = head->n_pairs, n_used = head->n_used;
  const int64_t t0 = (int64_t)blockIdx.x * LargeCopy::kThreads + threadIdx.x, step = (int64_t)gridDim.x * LargeCopy::kThreads;
  for (int64_t i = t0; i < n_entries; i += step) {
    const int e = table[i];
    if (e >= n_used) table[i] = dst[move[e]];   // (a page in use: checked above)
  }
  for (int64_t i = t0; i < n_pairs; i += step) {
    refs[dst[i]] = refs[src[i]];
    refs[src[i]] = 0;
  }
  const unsigned pieces = pa.total_pieces, total = n_pairs * pieces;   // (below 2^31: checked by the caller)
  for (unsigned u = blockIdx.x; u < total; u += gridDim.x) {
    const unsigned i = u / pieces;
    copy_piece<LargeCopy>(pa, src[i], dst[i], (int)(u - i * pieces));
  }
}

unsigned copy_grid(const PageArrays& pa, int64_t pairs) {
  return (unsigned)std::max<int64_t>(1, std::min<int64_t>(pairs * pa.total_pieces, (int64_t)current_sm_count(148) * 8));
}

// Cuts the arrays into the pieces of the copies.
template <class C>
PageArrays in_pieces(PageArrays pa) {
  pa.total_pieces = 0;
  for (int a = 0; a < kPageArrays; ++a) {
    pa.pieces[a] = (int)((pa.bytes[a] + kPieceOf<C> - 1) / kPieceOf<C>);
    pa.total_pieces += pa.pieces[a];
  }
  return pa;
}

}  // namespace

size_t pages_workspace_bytes(int64_t num_pages, int64_t n_seqs) {
  return 256 + sizeof(int32_t) * (size_t)(3 * ((num_pages + 63) & ~(int64_t)63) + 2 * ((n_seqs + 63) & ~(int64_t)63));
}

cudaError_t launch_copy_pages(const PageArrays& arrays, int num_pages, const int32_t* src, const int32_t* dst, int64_t n,
                              int32_t* status, cudaStream_t st) {
  const PageArrays pa = in_pieces<SmallCopy>(arrays);
  if (n == 0 || pa.total_pieces == 0) return cudaSuccess;
  if (n >= ((int64_t)1 << 31) / pa.total_pieces) return cudaErrorNotSupported;
  const unsigned grid = (unsigned)std::min<int64_t>(n * pa.total_pieces, 1 << 20);
  (void)launch_chained(copy_pages_kernel, dim3(grid), dim3(SmallCopy::kThreads), 0, st, pa, num_pages, src, dst, (int)n,
                       (const PlanHead*)nullptr, status);
  return cudaGetLastError();
}

cudaError_t launch_fork(int32_t* table, int32_t* seq_lens, int32_t* refs, int num_pages, int batch, int max_pages,
                        const int32_t* src, const int32_t* dst, int n, int32_t* status, cudaStream_t st) {
  if (n == 0) return cudaSuccess;
  (void)launch_chained(fork_kernel, dim3(n), dim3(kRowThreads), 0, st, table, seq_lens, refs, num_pages, batch, max_pages, src,
                       dst, n, status);
  return cudaGetLastError();
}

cudaError_t launch_free(int32_t* table, int32_t* seq_lens, int32_t* refs, int num_pages, int batch, int max_pages,
                        const int32_t* seqs, int n, int32_t* status, cudaStream_t st) {
  if (n == 0) return cudaSuccess;
  (void)launch_chained(free_kernel, dim3(n), dim3(kRowThreads), 0, st, table, seq_lens, refs, num_pages, batch, max_pages, seqs,
                       status);
  return cudaGetLastError();
}

cudaError_t launch_reserve(const PageArrays& arrays, int32_t* table, const int32_t* seq_lens, int32_t* refs, int num_pages, int batch,
                           int max_pages, const int32_t* seqs, const int32_t* n_tokens, int n, void* ws, int32_t* status,
                           cudaStream_t st) {
  if (n == 0) return cudaSuccess;
  const PageArrays pa = in_pieces<SmallCopy>(arrays);
  static PerDeviceOnce once;
  cudaError_t e = set_dyn_smem_once(reserve_kernel, (int)sizeof(ReserveShared), once);
  if (e != cudaSuccess) return e;
  PlanHead* head = reinterpret_cast<PlanHead*>(ws);
  int32_t* src = reinterpret_cast<int32_t*>(reinterpret_cast<char*>(ws) + 256);
  int32_t* dst = src + ((n + 63) & ~63);
  (void)launch_chained(reserve_kernel, dim3(1), dim3(kPlanThreads), sizeof(ReserveShared), st, table, seq_lens, refs, num_pages,
                       batch, max_pages, seqs, n_tokens, n, head, src, dst, status);
  e = cudaGetLastError();
  if (e != cudaSuccess || pa.total_pieces == 0) return e;
  (void)launch_chained(copy_pages_kernel, dim3(copy_grid(pa, n)), dim3(SmallCopy::kThreads), 0, st, pa, num_pages, src, dst, 0,
                       (const PlanHead*)head, status);
  return cudaGetLastError();
}

cudaError_t launch_compact(const PageArrays& arrays, int32_t* table, int64_t n_entries, int32_t* refs, int num_pages,
                           int32_t* n_used, void* ws, int32_t* status, cudaStream_t st) {
  const PageArrays pa = in_pieces<LargeCopy>(arrays);
  if ((int64_t)num_pages * pa.total_pieces >= (int64_t)1 << 31) return cudaErrorNotSupported;
  PlanHead* head = reinterpret_cast<PlanHead*>(ws);
  const int64_t pad = ((int64_t)num_pages + 63) & ~(int64_t)63;
  int32_t* src = reinterpret_cast<int32_t*>(reinterpret_cast<char*>(ws) + 256);
  int32_t *dst = src + pad, *move = dst + pad;
  const int n_checks = (int)std::min<int64_t>(kCheckMax, (n_entries + kPlanThreads * kCheckVec - 1) / (kPlanThreads * kCheckVec));
  (void)launch_chained(compact_plan_kernel, dim3(1 + n_checks), dim3(kPlanThreads), 0, st, (const int32_t*)table, n_entries,
                       (const int32_t*)refs, num_pages, head, src, dst, move, n_used);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  (void)launch_chained(compact_move_kernel, dim3((unsigned)current_sm_count(148) * 32), dim3(LargeCopy::kThreads), 0, st, pa, num_pages,
                       table, n_entries, refs, head, n_checks, src, dst, move, n_used, status);
  return cudaGetLastError();
}

}  // namespace rtp
