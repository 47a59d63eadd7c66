// Attention of chunks of several sequences over the paged cache (rtp_attn_chunks): a chunk is any number of consecutive rows of a
// sequence, one (a decode step), a few (tokens to verify) or thousands (a piece of a prompt), all in one call.
//
// Work.  A unit is a KV head with its query heads, over up to 2 x BMP consecutive positions of a chunk (BMP = 128 / G positions x G
// heads fill the 128 rows of an MMA).  Its cost is the number of key tiles (128 keys) that its rows see, from one to thousands,
// known on the device only.  plan_kernel counts it out: units are dealt round robin as long as there are two rounds and more of them
// (CTAs that run at the same time then walk the same keys, which come from L2), and the last one or two rounds, or all of a small call,
// are laid end to end and cut into equal pieces, one per CTA, at any key tile.  A piece that is not a whole unit leaves its rows'
// maxima, sums and unnormalised outputs in the workspace; merge_kernel joins them by log-sum-exp.
//
// Tiles.  One CTA per SM (384 threads), persistent over its list of pieces:
//   warp 9    Q (TMA, rows in the order [position][head]) and K tiles, warp 10 V tiles, into a ring of five 32 KB slots; table entries
//             are looked up 16 tiles at a time.  Keys that no row may see are zeroed in V (their pages' tails may hold anything).
//   warp 8    issues S = Q K^T (128 x 128 x 128) and O += P V on the 5th-generation tensor cores, S of a job before P V of the job
//             before it, across pieces: the next piece's tiles are on their way while this one ends.
//   warps 0-7 two groups of 128 threads, thread = row = TMEM lane: S to registers, mask, online softmax in 32 bits, P (bf16) back to
//             TMEM over the first half of S, from where the MMA takes it: shared memory holds no P and serves the ring instead.
// Jobs alternate between the groups.  A unit of more than BMP positions has two Q tiles, one per group, over the same K / V tiles
// (half the traffic); a smaller one has one, and the groups take every other key tile and are joined at the end, straight from TMEM.
// S and P of a group share 128 columns: S of its next job is issued behind the P V that reads P, and the tensor core runs them in order.
//
// Bound and measured (8 KV heads, groups of 4, device time).  Long chunks: the tensor cores, 2048 rows over 32K keys 830 us = 1283 TFLOP/s
// of 1694 that a library product reaches (1000 us by the prefill kernel of the other calls), by itself; call after call, under the 1000 W limit,
// 965 us = 1104 of the 1395 that the product sustains there.  What is missing is the chain S -> softmax ->
// P -> next S of each group, of which two cover each other but not all of it, and the shared issue slots of the issuing warp and the softmax
// warps.  Few rows: DRAM, 5 rows each of 32 sequences of 8K keys 119 us = 5.4 TB/s.  A mixture of pieces and single rows: both in turn,
// 12 chunks up to 700 rows over up to 32K keys 272 us by itself, 305 call after call.  7 rows over 200 keys: two launches and one chain of
// loads and products, 10.6 us.
// Tried and left: exponentials by polynomial on the FMA pipe (slower: one warp per scheduler is issue bound), a 56 / 224
// register split, rolled loops, the merge launched ahead (no difference).
#include "tc_common.cuh"

namespace rtp {

// 3-D tensor map of query rows [rows][n_heads][128] bf16 with a box of box_rows x box_heads x 64 (tensor_map.cu).
cudaError_t make_heads_map(CUtensorMap* map, const void* base, int64_t rows, int n_heads, int box_heads, int box_rows, int swizzle);
cudaError_t encode_rows_map(CUtensorMap* map, const void* base, int64_t rows, int row_elems, int box_cols, int box_rows, int swizzle);

namespace {

constexpr int kThreads = 384;
constexpr int kTile = 128;                     // keys per tile
constexpr int kBlk = 128 * 128;                // bytes of a [128 rows][64 elements] bf16 block
constexpr int kSlot = 2 * kBlk;                // a Q, K or V tile
constexpr int kRing = 5;
constexpr int kRingOff = 2 * kSlot;            // behind two Q tiles
constexpr int kBarOff = kRingOff + kRing * kSlot;
constexpr int kXchOff = kBarOff + 256;         // float [2 groups][2][128 rows]
constexpr int kSmem = kXchOff + 2048;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kMaxUnits = 64;                  // (KV head, pattern) pairs of a call
constexpr int kPlanThreads = 1024;

enum Bar { kQFull = 0, kQEmpty = 2, kFull = 4, kEmpty = kFull + kRing, kSFull = kEmpty + kRing, kPFull = kSFull + 2, kOFull = kPFull + 4,
           kAux = kOFull + 2, kNumBars };   // (P: first and second half of each group's)
static_assert(kNumBars * 8 + 16 <= 256, "barriers, TMEM address and abort flag");

// A KV head of the call: sinks and window or everything before the row; which of its query heads are written.
enum UnitFlags { kLocal = 1, kSkipRet = 2, kSkipOther = 4, kLocalPool = 8 };
struct HeadUnits {
  uint8_t head[kMaxUnits], flags[kMaxUnits];
  int32_t n;
  uint32_t ret_q[RTP_MAX_Q_HEADS / 32];        // retrieval query heads
  __device__ bool writes(int unit, int qh) const {
    const bool ret = (ret_q[qh >> 5] >> (qh & 31)) & 1u;
    return !((flags[unit] & kSkipRet) && ret) && !((flags[unit] & kSkipOther) && !ret);
  }
};

// A piece of a unit: key tiles tile_lo .. tile_hi - 1 of its n_tiles.
struct __align__(16) Piece {
  int32_t row0, pos0, n_pos, seq;              // rows row0 .. of q at positions pos0 ..
  int32_t unit, kt_first, n_sink_tiles, n_keys;
  int32_t tile_lo, tile_hi, slot, id;          // slot: of its partial result, or one of the two below; id: number of the unit
};
constexpr int kWhole = -1, kNothing = -2;
struct __align__(16) MergeUnit {
  int32_t row0, n_pos, unit, id;
  int32_t first_cta, last_cta, pad0, pad1;
};
struct Plan {                                  // where things lie in the workspace
  int32_t* n_merge;
  int32_t* piece_begin;                        // [n_ctas + 1]
  int32_t* part_id;                            // [2 n_ctas]: unit of the partial result in a slot, or -1
  MergeUnit* merge;                            // [n_ctas]
  Piece* pieces;
  int64_t* before;                             // [max_units + 1], of calls with many units of different costs
  float* ml;                                   // [2 n_ctas][slot_rows][2]
  float* o;                                    // [2 n_ctas][slot_rows][128]
  int32_t n_ctas, max_units, slot_rows;
};

struct ChunkArgs {
  const int32_t *seq, *start, *offsets;
  int32_t n_chunks, G, bmp;
  int64_t R;
  int64_t ring_tokens, pool_tokens;            // of the local pool, 0 if no unit reads one
};

// ---- plan --------------------------------------------------------------------------------------------
// Costs are in jobs (a key tile of a Q tile); a piece has a start and an end beside them.
constexpr int kPieceCost = 3;
constexpr int kMinJobs = 6;                    // a piece of its own (and a merge) has to be worth it
constexpr int kMinShare = 24;                  // jobs of a CTA's share of what is not dealt
constexpr int kSnap = 3;                       // key tiles that are not cut off
constexpr int kPlanUnits = 1024;               // units whose costs lie in shared memory

struct PlanShared {
  int64_t warp_sum[2][32];
  int64_t load[1024 + 1];                      // jobs dealt to each CTA, then the cuts
  int64_t before[kPlanUnits + 1];
  int32_t begin[1024], first[1024];            // of each CTA: pairs in front of its own, its first unit
  int32_t n_merge;
};

constexpr int kKeptUnits = 1024, kKeptChunks = 4096;   // units that are described once (their descriptions lie in shared memory)
// Bytes in front of them: the above, and the chunks' lists.
__host__ __device__ constexpr size_t plan_lists(int64_t n_chunks) {
  return ((sizeof(PlanShared) + 15) & ~(size_t)15) + (((size_t)n_chunks * (sizeof(int4) + sizeof(int2)) + 15) & ~(size_t)15);
}
// Exclusive sum over the block, and the total.  The two rows of warp_sum are used in turn: who writes one again has passed the barrier of
// the other, and so has everybody who read it.
__device__ __forceinline__ int64_t scan64(int64_t x, int64_t (*warp_sum)[32], int& turn, int64_t& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  int64_t s = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t y = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += y;
  }
  if (lane == 31) warp_sum[turn][warp] = s;
  __syncthreads();
  const int64_t w = lane < warps ? warp_sum[turn][lane] : 0;
  turn ^= 1;
  int64_t t = w;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t y = __shfl_up_sync(0xffffffffu, t, o);
    if (lane >= o) t += y;
  }
  total = __shfl_sync(0xffffffffu, t, 31);
  return __shfl_sync(0xffffffffu, t - w, warp) + s - x;
}
// The last i in [0, n) with v[i] <= x (v[0] <= x).
template <class V>
__device__ __forceinline__ int last_at(int n, int64_t x, V v) {
  int lo = 0, hi = n;
  while (lo + 1 < hi) {
    const int mid = (lo + hi) >> 1;
    if (v(mid) <= x) lo = mid; else hi = mid;
  }
  return lo;
}

__global__ void __launch_bounds__(kPlanThreads) plan_kernel(const __grid_constant__ ChunkArgs a, const __grid_constant__ CacheView cv,
                                                            const __grid_constant__ HeadUnits hu, const __grid_constant__ Plan plan,
                                                            const int n_sink, const int window, int32_t* status) {
  chain_wait();
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // (the attention kernel sets itself up and waits for this one)
  extern __shared__ __align__(16) unsigned char smem_plan[];
  PlanShared& s = *reinterpret_cast<PlanShared*>(smem_plan);
  int4* chunk = reinterpret_cast<int4*>(smem_plan + ((sizeof(PlanShared) + 15) & ~15));   // [n_chunks]: units before, rows, start, keys
  int2* where = reinterpret_cast<int2*>(chunk + a.n_chunks);                              // [n_chunks]: row in q, sequence
  Piece* kept = reinterpret_cast<Piece*>(smem_plan + plan_lists(a.n_chunks));                // [kKeptUnits] of calls with at most kKeptChunks chunks
  const int tid = threadIdx.x, nt = blockDim.x;
  const int N = plan.n_ctas, H = hu.n, span = 2 * a.bmp;
  int turn = 0;
  // chunks, with what is wrong in them
  int64_t mine = 0;
  const int per = (a.n_chunks + nt - 1) / nt, c0 = min(tid * per, a.n_chunks), c1 = min(c0 + per, a.n_chunks);
  bool bad = false;
  for (int c = c0; c < c1; ++c) {
    const int64_t lo = a.offsets[c], hi = a.offsets[c + 1];
    const int seq = a.seq[c];
    int start = a.start[c], rows = (int)(hi - lo);
    if (lo < 0 || hi < lo || hi > a.R) {       // no rows of the call
      rows = 0;
      bad = true;
    }
    int keys = (unsigned)seq < (unsigned)cv.batch ? max(0, min(cv.seq_lens[seq], cv.cap_tokens)) : 0;
    if (start < 0) keys = 0;
    if (rows > 0 && (int64_t)start + rows > keys) bad = true;
    // positions, those of a tile's unused rows included, stay within 32 bits (rows that far behind the end see the same keys in front of it)
    start = max(0, min(start, 0x7fffffff - rows - 2 * span));
    // a ring has to hold the window of the chunk's first row when the sequence's last token has been appended, be it of this chunk or not
    if (rows > 0 && a.ring_tokens && keys > a.pool_tokens && a.ring_tokens < (int64_t)window + ((int64_t)keys - start) + kPage) {
      rows = 0;
      set_status(status, RTP_ERR_CAPACITY);
    }
    chunk[c] = make_int4(0, rows, start, keys);
    where[c] = make_int2((int)lo, seq);
    mine += (int64_t)((rows + span - 1) / span) * H;
  }
  if (bad) set_status(status, RTP_ERR_INVALID);
  for (int i = tid; i < 2 * N; i += nt) plan.part_id[i] = -1;
  for (int i = tid; i < N; i += nt) s.load[i] = 0;
  if (tid == 0) s.n_merge = *plan.n_merge = 0;
  int64_t total_units;
  int64_t at = scan64(mine, s.warp_sum, turn, total_units);
  if (total_units > plan.max_units) {          // offsets that run back and forth: nothing is done
    if (tid == 0) set_status(status, RTP_ERR_INVALID);
    for (int i = tid; i <= N; i += nt) plan.piece_begin[i] = 0;
    return;
  }
  for (int c = c0; c < c1; ++c) {
    chunk[c].x = (int)at;
    at += (int64_t)((chunk[c].y + span - 1) / span) * H;
  }
  __syncthreads();
  const int U = (int)total_units;
  // unit u: chunk by chunk, head by head, the last positions first; returns its key tiles
  auto make = [&](int u, Piece& p) -> int {
    const int i = last_at(a.n_chunks, u, [&](int j) { return chunk[j].x; });
    const int4 c = chunk[i];
    const int2 w = where[i];
    const int nq = (c.y + span - 1) / span, r = u - c.x, h = r / nq, t = nq - 1 - (r - h * nq);
    p.pos0 = c.z + t * span;
    p.n_pos = min(span, c.y - t * span);
    p.row0 = w.x + t * span;
    p.seq = w.y;
    p.unit = h;
    p.n_keys = min(c.w, p.pos0 + p.n_pos);
    p.id = u;
    const int n_all = p.n_keys > 0 ? (p.n_keys - 1) / kTile + 1 : 0;
    p.kt_first = p.n_sink_tiles = 0;
    if (hu.flags[h] & kLocal) {
      p.kt_first = min(max(0, p.pos0 - window + 1) / kTile, n_all);
      p.n_sink_tiles = min(min((n_sink + kTile - 1) / kTile, p.kt_first), n_all);
    }
    return p.n_sink_tiles + n_all - p.kt_first;
  };
  const bool keep = U <= kKeptUnits && a.n_chunks <= kKeptChunks;
  if (keep) {
    for (int u = tid; u < U; u += nt) {
      Piece p;
      p.tile_hi = make(u, p);
      kept[u] = p;
    }
    __syncthreads();
  }
  auto describe = [&](int u, Piece& p) -> int {
    if (!keep) return make(u, p);
    p = kept[u];
    return p.tile_hi;
  };
  // A CTA each for few and short units: a cut of less than two shares each would not end sooner, and nothing has to be summed up (7 rows over
  // 200 keys: 10 us against 17 by the general way below, over 1000 keys 17 against 24, over 1500 with 12 tiles 25 either way).
  if (U <= N) {
    Piece p;
    if (tid < U) {
      p.tile_hi = describe(tid, p);
      p.tile_lo = 0;
      p.slot = kWhole;
    }
    if (!__syncthreads_or(tid < U && (int64_t)p.tile_hi * (p.n_pos > a.bmp ? 2 : 1) > 2 * kMinJobs)) {
      if (tid < U) plan.pieces[tid] = p;
      for (int i = tid; i <= N; i += nt) plan.piece_begin[i] = min(i, U);
      return;
    }
  }
  // Costs: the dealt units' go to their CTAs, the others' into a list.
  int rounds = U / N;
  int64_t* before = s.before;
  int64_t W_dealt = 0, W_cut = 0;
  for (;;) {
    const int D = rounds * N, M = U - D;
    before = M <= kPlanUnits ? s.before : plan.before;
    for (int u = tid; u < U; u += nt) {
      Piece p;
      const int n = describe(u, p);
      const int64_t w = kPieceCost + (int64_t)n * (p.n_pos > a.bmp ? 2 : 1);
      if (u < D) atomicAdd(reinterpret_cast<unsigned long long*>(&s.load[u % N]), (unsigned long long)w);
      else before[u - D] = w;
    }
    __syncthreads();
    const int each = (M + nt - 1) / nt, j0 = min(tid * each, M), j1 = min(j0 + each, M);
    int64_t sum = 0;
    for (int j = j0; j < j1; ++j) sum += before[j];
    int64_t run = scan64(sum, s.warp_sum, turn, W_cut);
    for (int j = j0; j < j1; ++j) {
      const int64_t w = before[j];
      before[j] = run;
      run += w;
    }
    if (tid == 0) before[M] = W_cut;
    if (rounds == 0) break;
    // Whole units only where no CTA gets more than its share of them (a few that cost more than the others are cut instead), and one
    // round less where the rest would be cut into crumbs.
    scan64(tid < N ? s.load[tid] : 0, s.warp_sum, turn, W_dealt);
    const bool uneven = __syncthreads_or(tid < N && s.load[tid] * N > W_dealt + W_cut);
    const bool crumbs = W_cut > 0 && W_cut < (int64_t)N * kMinShare;
    if (!uneven && !(crumbs && rounds == U / N)) break;
    rounds = uneven ? 0 : rounds - 1;
    __syncthreads();
    for (int i = tid; i < N; i += nt) s.load[i] = 0;
    __syncthreads();
  }
  __syncthreads();
  const int D = rounds * N, M = U - D;
  // What each CTA takes of the cut part: up to the mean; with nothing dealt, equal shares for as many as are worth it.
  if (rounds) {
    // (the mean in double precision, and one more, so that there is room in any case)
    const int64_t mean = (int64_t)((double)(W_dealt + W_cut) * (1.0 / N)) + 2, room = tid < N ? max((int64_t)0, mean - s.load[tid]) : 0;
    int64_t rooms;
    const int64_t room_before = scan64(room, s.warp_sum, turn, rooms);
    if (tid < N) s.load[tid] = min(W_cut, (int64_t)((double)room_before * ((double)W_cut / (double)rooms)));
  } else {
    const int takers = max(1, (int)min((int64_t)N, W_cut / (kMinJobs + kPieceCost)));
    if (tid < N) s.load[tid] = tid < takers ? (int64_t)((double)W_cut * tid / takers) : W_cut;
  }
  if (tid == 0) s.load[N] = W_cut;
  __syncthreads();
  // CTA i takes the units j that meet [load[i], load[i + 1])
  const bool taker = tid < N && s.load[tid] < s.load[tid + 1];
  auto at_unit = [&](int j) { return before[j]; };
  const int j_first = taker ? last_at(M, s.load[tid], at_unit) : 0, j_end = taker ? last_at(M, s.load[tid + 1] - 1, at_unit) + 1 : 0;
  int64_t pairs64;
  const int cut_before = (int)scan64(j_end - j_first, s.warp_sum, turn, pairs64), pairs = (int)pairs64;
  if (tid < N) {
    s.begin[tid] = cut_before;
    s.first[tid] = j_first;
    plan.piece_begin[tid] = tid * rounds + cut_before;
  }
  if (tid == 0) plan.piece_begin[N] = N * rounds + pairs;
  __syncthreads();
  for (int u = tid; u < D; u += nt) {
    Piece p;
    p.tile_hi = describe(u, p);
    p.tile_lo = 0;
    p.slot = kWhole;
    plan.pieces[(u % N) * rounds + s.begin[u % N] + u / N] = p;
  }
  // the key tile of a unit (u0 < x < its end) at which a cut at x falls
  auto cut_at = [&](int64_t x, int64_t u0, int n, int per_tile) -> int {
    const int t = x <= u0 + kPieceCost ? 0 : (int)((x - u0 - kPieceCost + per_tile - 1) >> (per_tile - 1));
    return t < kSnap ? 0 : n - t < kSnap ? n : t;
  };
  for (int q = tid; q < pairs; q += nt) {      // a thread per (CTA, unit) pair
    const int i = last_at(N, q, [&](int c) { return s.begin[c]; }), j = s.first[i] + q - s.begin[i];
    Piece p;
    const int64_t from = s.load[i], to = s.load[i + 1], u0 = before[j], u1 = before[j + 1];
    const int n = describe(D + j, p), per_tile = p.n_pos > a.bmp ? 2 : 1;
    p.tile_lo = from <= u0 ? 0 : cut_at(from, u0, n, per_tile);
    p.tile_hi = to >= u1 ? n : cut_at(to, u0, n, per_tile);
    p.slot = kWhole;
    if (p.tile_lo >= p.tile_hi && !(n == 0 && u0 >= from)) {
      p.slot = kNothing;                       // (less than is cut off of a unit: its neighbours have it)
    } else if (p.tile_lo > 0 || p.tile_hi < n) {
      p.slot = 2 * i + (p.tile_lo == 0);       // (a CTA has one piece that begins inside a unit, and one that only ends there)
      plan.part_id[p.slot] = p.id;
      if (p.tile_lo == 0) {                    // up to the last CTA whose share begins before the unit's end
        const int last = last_at(N, u1 - 1, [&](int c) { return s.load[c]; });
        plan.merge[atomicAdd(&s.n_merge, 1)] = MergeUnit{p.row0, p.n_pos, p.unit, p.id, i, last, 0, 0};
      }
    }
    plan.pieces[(i + 1) * rounds + q] = p;
  }
  __syncthreads();
  if (tid == 0) *plan.n_merge = s.n_merge;
}

// ---- attention ----------------------------------------------------------------------------------------
__device__ __forceinline__ uint64_t desc128(uint32_t saddr, uint32_t lbo) { return smem_desc_sw(saddr, lbo, 1024, 2); }
// The products are single statements of few instructions: the issuing thread shares its scheduler with two softmax warps that seldom
// leave it a slot.  (A probe: an issuer of twice the instructions next to two warps of FMAs took 1.5 to 5 times as long.)
// D (TMEM) = A B^T over 128 channels, both from shared memory: eight steps of 16 channels, 32 bytes each, four to a block.
__device__ __forceinline__ void mma_ss8(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc) {
  asm volatile(
      "{\n.reg .pred t, f;\n.reg .b64 a, b;\nsetp.ne.b32 t, 1, 0;\nsetp.ne.b32 f, 0, 0;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, f;\n"
      "add.s64 a, %1, 2;\nadd.s64 b, %2, 2;\ntcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, t;\n"
      "add.s64 a, %1, 4;\nadd.s64 b, %2, 4;\ntcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, t;\n"
      "add.s64 a, %1, 6;\nadd.s64 b, %2, 6;\ntcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, t;\n"
      "add.s64 a, %1, 1024;\nadd.s64 b, %2, 1024;\ntcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, t;\n"
      "add.s64 a, %1, 1026;\nadd.s64 b, %2, 1026;\ntcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, t;\n"
      "add.s64 a, %1, 1028;\nadd.s64 b, %2, 1028;\ntcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, t;\n"
      "add.s64 a, %1, 1030;\nadd.s64 b, %2, 1030;\ntcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, t;\n}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc)
      : "memory");
}
static_assert(kBlk >> 4 == 1024, "the distance of two blocks in a descriptor");
// D (TMEM) += A (TMEM: two bf16 per column, lane = row) B over 64 keys: four steps of 16 keys, 8 columns of A and 2 KB of B each.
__device__ __forceinline__ void mma_ts4(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n.reg .pred t, p;\n.reg .b64 b;\n.reg .b32 a;\nsetp.ne.b32 t, 1, 0;\nsetp.ne.b32 p, %4, 0;\n"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n"
      "add.u32 a, %1, 8;\nadd.s64 b, %2, 128;\ntcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, t;\n"
      "add.u32 a, %1, 16;\nadd.s64 b, %2, 256;\ntcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, t;\n"
      "add.u32 a, %1, 24;\nadd.s64 b, %2, 384;\ntcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, t;\n}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
// A wait that is usually over already: asked once without parking the thread.
__device__ __forceinline__ void wait_for(uint32_t bar, uint32_t parity, volatile int* abort_flag, int32_t* status, unsigned long long limit_ns) {
  uint32_t ok;
  asm volatile("{\n.reg .pred p;\nmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  if (!ok) mbar_wait(bar, parity, abort_flag, status, limit_ns);
}
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(p));
  return p != 0;
}
// a * b + c on two numbers at a time
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 r;
  asm("{\n.reg .b64 a, b, c, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nmov.b64 c, {%6, %7};\nfma.rn.f32x2 d, a, b, c;\nmov.b64 {%0, %1}, d;\n}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return r;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 r;
  asm("{\n.reg .b64 a, b, d;\nmov.b64 a, {%2, %3};\nmov.b64 b, {%4, %5};\nadd.rn.f32x2 d, a, b;\nmov.b64 {%0, %1}, d;\n}"
      : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return r;
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
      "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
      : "memory");
}

struct __align__(64) Maps {
  CUtensorMap q, k, v, lk, lv;                 // queries; pages of the main and of the local pool
};

__global__ void __launch_bounds__(kThreads, 1) attn_chunks_kernel(const __grid_constant__ Maps maps, const __grid_constant__ CacheView cv,
                                                                  const __grid_constant__ CacheView lv, const __grid_constant__ HeadUnits hu,
                                                                  const __grid_constant__ Plan plan, const __grid_constant__ Dims d,
                                                                  const int bmp, __nv_bfloat16* __restrict__ out,
                                                                  float* __restrict__ lse, int32_t* status) {
  extern __shared__ __align__(1024) unsigned char smem[];
  const uint32_t sbase = s_u32(smem);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + kBarOff + kNumBars * 8);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(smem + kBarOff + kNumBars * 8 + 8);
  auto bar = [&](int i) { return sbase + kBarOff + i * 8; };
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int G = d.group;
  if (tid == 0) {
    for (int i = 0; i < kNumBars; ++i) mbar_init(bar(i), i >= kPFull && i < kPFull + 4 ? 128 : 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(s_u32(tmem_slot)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  chain_wait();                                // (what is above touches nothing but the block's own memory)
  const int p_lo = __ldcg(plan.piece_begin + blockIdx.x), p_hi = __ldcg(plan.piece_begin + blockIdx.x + 1);
  // All 512 columns are this block's, from address 0 on: S / P of the groups at columns 0, 128; their O at 256, 384.
  constexpr uint32_t tmem = 0;

  auto load_piece = [&](int i) -> Piece {
    Piece p;
    const int4* src = reinterpret_cast<const int4*>(plan.pieces + i);
    int4* dst = reinterpret_cast<int4*>(&p);
#pragma unroll
    for (int x = 0; x < 3; ++x) dst[x] = __ldcg(src + x);
    return p;
  };

  // 256 x 232 + 128 x 40 = 384 x 168 registers
  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 40;");
    if (warp == 9 || warp == 10) {
      // ================================ loaders: Q and K, V ================================
      const bool is_v = warp == 10;
      unsigned fill = 0, n_aux = 0;
      int slot = is_v ? 1 : 0, phase = 1;      // (a wait for the phase before the first passes at once)
      bool drop = d.wait_test && !is_v;        // (the test hook drops the first signal)
      for (int i = p_lo; i < p_hi; ++i) {
        const Piece p = load_piece(i);
        if (p.slot == kNothing) continue;
        const int flags = hu.flags[p.unit], kvh = hu.head[p.unit];
        const bool local_pool = flags & kLocalPool;
        const CacheView& view = local_pool ? lv : cv;
        const CUtensorMap* map = is_v ? (local_pool ? &maps.lv : &maps.v) : (local_pool ? &maps.lk : &maps.k);
        const int kslot = view.kv_slot[kvh], n_kv = view.n_kv;
        const int64_t bt_base = (int64_t)p.seq * view.max_pages;
        // Row in the pool of the pages of 16 tiles (lane: tile base + lane / 2, first or second page; -1: no key there), looked up while
        // the tiles before them are loaded.
        auto tile_of = [&](int x) { return x < p.n_sink_tiles ? x : p.kt_first + (x - p.n_sink_tiles); };
        auto look_up = [&](int base) {
          const int y = base + (lane >> 1), page = 2 * tile_of(y) + (lane & 1);
          return y < p.tile_hi && page * kPage < p.n_keys ? (safe_phys(view, bt_base + page_entry(view, page), status) * n_kv + kslot) * kPage : -1;
        };
        int next = look_up(p.tile_lo), rows = 0;
        if (!is_v && p.tile_lo < p.tile_hi) {
          for (int t = 0; t < (p.n_pos > bmp ? 2 : 1); ++t, ++fill) {
            const int b = fill & 1;
            if (fill >= 2) wait_for(bar(kQEmpty + b), ((fill >> 1) - 1) & 1, abort_flag, status, d.wait_ns);
            if (elect_one()) {
              mbar_expect_tx(bar(kQFull + b), (uint32_t)(G * bmp) * 256u);
              tma_load_3d(sbase + b * kSlot, &maps.q, 0, kvh * G, p.row0 + t * bmp, bar(kQFull + b));
              tma_load_3d(sbase + b * kSlot + kBlk, &maps.q, 64, kvh * G, p.row0 + t * bmp, bar(kQFull + b));
            }
            __syncwarp();
          }
        }
        for (int x = p.tile_lo; x < p.tile_hi; ++x) {
          const int rel = (x - p.tile_lo) & 15;
          if (rel == 0) {
            rows = next;
            next = look_up(x + 16);
          }
          const int y0 = __shfl_sync(0xffffffffu, rows, 2 * rel), y1 = __shfl_sync(0xffffffffu, rows, 2 * rel + 1);
          wait_for(bar(kEmpty + slot), phase, abort_flag, status, d.wait_ns);
          const uint32_t dst = sbase + kRingOff + slot * kSlot;
          const int n_ok = p.n_keys - tile_of(x) * kTile;   // keys of the tile that rows may see
          const bool part = is_v && n_ok < kTile;
          const uint32_t fb = part ? bar(kAux) : bar(kFull + slot);
          if (elect_one() && !drop) {
            mbar_expect_tx(fb, y1 >= 0 ? 2 * kBlk : kBlk);
            tma_load_2d(dst, map, 0, y0, fb);
            tma_load_2d(dst + kBlk, map, 64, y0, fb);
            if (y1 >= 0) {
              tma_load_2d(dst + kPage * 128, map, 0, y1, fb);
              tma_load_2d(dst + kBlk + kPage * 128, map, 64, y1, fb);
            }
          }
          __syncwarp();
          drop = false;
          if (part) {                          // what lies behind the last key is not read: 0 x NaN is no 0
            wait_for(bar(kAux), n_aux & 1, abort_flag, status, d.wait_ns);
            ++n_aux;
            unsigned char* v = smem + kRingOff + slot * kSlot;
            for (int z = n_ok * 8 + lane; z < kTile * 8; z += 32) {
              *reinterpret_cast<uint4*>(v + z * 16) = make_uint4(0, 0, 0, 0);
              *reinterpret_cast<uint4*>(v + kBlk + z * 16) = make_uint4(0, 0, 0, 0);
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(kFull + slot));
          }
          slot += 2;
          if (slot >= kRing) {
            slot -= kRing;
            phase ^= 1;
          }
        }
      }
    } else if (warp == 8) {
      // ================================ MMA issuer ================================
      // One thread.  The tensor core holds about four products that are issued and not done: as long as the thread is back within their
      // time (256 cycles) it does not run dry, which would cost 400 cycles.
      if (elect_one()) {
        const uint32_t idesc_s = instr_desc_mn(128, 128, false), idesc_o = instr_desc_mn(128, 128, true);
        const uint64_t q_desc = desc128(sbase, 16), k_desc = desc128(sbase + kRingOff, 16), v_desc = desc128(sbase + kRingOff, kBlk);
        unsigned fill = 0, p_phase = 0;        // p_phase: a bit for each group
        int g = 0, slot = 0, phase = 0;        // group of the next job; ring slot of the next tile's K (its V is in the one behind)
        // the P V that is still to be issued, of group g ^ 1: bits 0 there, 1 its tile's first, 2 its piece's first, 3 its tile's last,
        // 4 its piece's last, 5 phase of its V's slot
        unsigned pv = 0;
        int pv_slot = 0;
        auto issue_pv = [&]() {
          if (!(pv & 1u)) return;
          const int pg = g ^ 1;
          const uint32_t p_bar = bar(kPFull) + pg * 16, v_bar = pv_slot * 8, par = (p_phase >> pg) & 1u;
          const uint64_t v = v_desc + (uint32_t)(pv_slot * (kSlot >> 4));
          p_phase ^= 1u << pg;
          if (pv & 2u) wait_for(bar(kFull) + v_bar, (pv >> 5) & 1u, abort_flag, status, d.wait_ns);
          wait_for(p_bar, par, abort_flag, status, d.wait_ns);
          tc_fence_after();
          mma_ts4(256u + pg * 128u, pg * 128u, v, idesc_o, ~pv & 4u);
          wait_for(p_bar + 8, par, abort_flag, status, d.wait_ns);
          tc_fence_after();
          mma_ts4(256u + pg * 128u, pg * 128u + 32u, v + (4 * 2048 >> 4), idesc_o, 1u);
          if (pv & 8u) tc_commit(bar(kEmpty) + v_bar);
          if (pv & 16u) tc_commit(bar(kOFull) + pg * 8);
        };
        for (int i = p_lo; i < p_hi; ++i) {
          const Piece p = load_piece(i);
          const int n = p.tile_hi - p.tile_lo;
          const bool two = p.n_pos > bmp;
          if (p.slot == kNothing || n == 0) continue;
          const int b0 = fill & 1, b1 = b0 ^ 1, jobs = two ? 2 * n : n;
          wait_for(bar(kQFull + b0), (fill >> 1) & 1, abort_flag, status, d.wait_ns);
          if (two) wait_for(bar(kQFull + b1), ((fill + 1) >> 1) & 1, abort_flag, status, d.wait_ns);
          fill += two ? 2 : 1;
#pragma unroll 1
          for (int x = 0; x < jobs; ++x) {
            const int second = two ? x & 1 : 0;
            if (!second) wait_for(bar(kFull) + slot * 8, phase, abort_flag, status, d.wait_ns);
            tc_fence_after();
            mma_ss8(g * 128u, q_desc + (uint32_t)((b0 ^ second) * (kSlot >> 4)), k_desc + (uint32_t)(slot * (kSlot >> 4)), idesc_s);
            tc_commit(bar(kSFull) + g * 8);
            const bool done = !two || second;  // with this tile
            if (done) tc_commit(bar(kEmpty) + slot * 8);
            if (x + (two ? 2 : 1) >= jobs) tc_commit(bar(kQEmpty) + (b0 ^ second) * 8);
            issue_pv();
            g ^= 1;
            const bool wrap = slot + 1 == kRing;
            pv_slot = wrap ? 0 : slot + 1;
            pv = 1u | (second ? 0u : 2u) | (x < 2 ? 4u : 0u) | (done ? 8u : 0u) | (x + 2 >= jobs ? 16u : 0u) | ((unsigned)(phase ^ (int)wrap) << 5);
            if (done) {
              slot += 2;
              if (slot >= kRing) {
                slot -= kRing;
                phase ^= 1;
              }
            }
          }
        }
        issue_pv();
      }
      __syncwarp();
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
    // ================================ softmax (thread = row) ================================
    const int grp = tid >> 7, row = tid & 127, po = row / G, hs = row - po * G;
    const uint32_t lane_addr = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t tmem_s = tmem + grp * 128u + lane_addr, tmem_o = tmem + 256u + grp * 128u + lane_addr;
    const uint32_t tmem_o2 = tmem + 256u + (grp ^ 1) * 128u + lane_addr;
    float* xch = reinterpret_cast<float*>(smem + kXchOff);
    const float sc2 = d.sm_scale * kLog2e;
    unsigned job0 = 0, n_s = 0, n_o = 0;
    for (int i = p_lo; i < p_hi; ++i) {
      const Piece p = load_piece(i);
      if (p.slot == kNothing) continue;
      const int n = p.tile_hi - p.tile_lo, nq = p.n_pos > bmp ? 2 : 1, jobs = n * nq;
      const int x0 = jobs ? (int)((grp ^ job0) & 1) : grp;          // this group's first job; without keys, group = Q tile
      job0 += jobs;
      const int qt = nq == 2 ? x0 : 0;
      const bool row_ok = po < bmp && qt * bmp + po < p.n_pos;
      const int pos = p.pos0 + qt * bmp + po, lim = min(pos, p.n_keys - 1);
      const bool local = hu.flags[p.unit] & kLocal;
      const bool warp_on = __any_sync(0xffffffffu, row_ok);
      float m_ref = -INFINITY, l_run = 0.f;
      for (int x = x0; x < jobs; x += 2, ++n_s) {
        const int tt = p.tile_lo + (nq == 2 ? x >> 1 : x);
        const int n_base = (tt < p.n_sink_tiles ? tt : p.kt_first + (tt - p.n_sink_tiles)) * kTile;
        wait_for(bar(kSFull + grp), n_s & 1, abort_flag, status, d.wait_ns);
        if (warp_on) {
          tc_fence_after();
          float s[kTile];
          uint32_t* s_lo = reinterpret_cast<uint32_t*>(s);
          uint32_t* s_hi = s_lo + 64;
          RTP_TMEM_LD64(s_lo, tmem_s);
          tc_wait_ld();
          RTP_TMEM_LD64(s_hi, tmem_s + 64);
          const bool masked = n_base + kTile - 1 > lim || (local && n_base <= pos - d.window);
          const int hi = lim - n_base, lo = local ? pos - d.window - n_base : -1, sink = local ? d.n_sink - n_base : 0;
          if (masked) {
#pragma unroll
            for (int e = 0; e < 64; ++e)
              if (!(e <= hi && (e > lo || e < sink))) s[e] = -INFINITY;
          }
          float t0 = s[0], t1 = s[1], t2 = s[2], t3 = s[3];
#pragma unroll
          for (int e = 4; e + 8 <= 64; e += 8) {
            t0 = fmaxf(fmaxf(t0, s[e]), s[e + 1]); t1 = fmaxf(fmaxf(t1, s[e + 2]), s[e + 3]);
            t2 = fmaxf(fmaxf(t2, s[e + 4]), s[e + 5]); t3 = fmaxf(fmaxf(t3, s[e + 6]), s[e + 7]);
          }
          t0 = fmaxf(fmaxf(t0, s[60]), s[61]); t1 = fmaxf(fmaxf(t1, s[62]), s[63]);
          tc_wait_ld();
          if (masked) {
#pragma unroll
            for (int e = 64; e < kTile; ++e)
              if (!(e <= hi && (e > lo || e < sink))) s[e] = -INFINITY;
          }
#pragma unroll
          for (int e = 64; e < kTile; e += 8) {
            t0 = fmaxf(fmaxf(t0, s[e]), s[e + 1]); t1 = fmaxf(fmaxf(t1, s[e + 2]), s[e + 3]);
            t2 = fmaxf(fmaxf(t2, s[e + 4]), s[e + 5]); t3 = fmaxf(fmaxf(t3, s[e + 6]), s[e + 7]);
          }
          const float tmax = fmaxf(fmaxf(t0, t1), fmaxf(t2, t3)) * sc2;
          // the reference is raised, and O and l scaled, only when a maximum exceeds it by more than 2^8 (any reference gives the same
          // quotient); the group's P V of before is complete, since S was issued behind it
          const bool raise = tmax > m_ref + 8.0f;
          if (__any_sync(0xffffffffu, raise)) {
            if (x >= 2) {
              const float f = raise ? ((m_ref == -INFINITY) ? 0.f : fast_ex2(m_ref - tmax)) : 1.f;
#pragma unroll 1
              for (int c4 = 0; c4 < 4; ++c4) {
                uint32_t r[32];
                RTP_TMEM_LD32(r, tmem_o + c4 * 32);
                tc_wait_ld();
#pragma unroll
                for (int e = 0; e < 32; ++e) r[e] = __float_as_uint(__uint_as_float(r[e]) * f);
                RTP_TMEM_ST32(tmem_o + c4 * 32, r);
              }
              l_run *= f;
            }
            if (raise) m_ref = tmax;
          }
          const float mb = (m_ref == -INFINITY) ? 0.f : m_ref;
          const float2 sc22 = make_float2(sc2, sc2), mb2 = make_float2(-mb, -mb);
          float2 rs0 = make_float2(0.f, 0.f), rs1 = rs0;
#pragma unroll
          // P is rounded to bf16, V's type, which the product's other operand has to have (with the output's own rounding the result is 0.0021 to
          // 0.0024 off 64 bits, relative and in the mean; 0.0017 without); the sum is of the 32-bit values
          for (int h = 0; h < 2; ++h) {
            uint32_t pk[32];
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              const float2 z = fma2(make_float2(s[h * 64 + 2 * e], s[h * 64 + 2 * e + 1]), sc22, mb2);
              const float2 pr = make_float2(fast_ex2(z.x), fast_ex2(z.y));
              if (e & 1) rs1 = add2(rs1, pr); else rs0 = add2(rs0, pr);
              const __nv_bfloat162 v = __floats2bfloat162_rn(pr.x, pr.y);
              pk[e] = *reinterpret_cast<const uint32_t*>(&v);
            }
            RTP_TMEM_ST32(tmem_s + h * 32, pk);
            tc_wait_st();
            tc_fence_before();
            mbar_arrive(bar(kPFull + 2 * grp + h));
          }
          l_run += (rs0.x + rs0.y) + (rs1.x + rs1.y);
        } else {
          mbar_arrive(bar(kPFull + 2 * grp));
          mbar_arrive(bar(kPFull + 2 * grp + 1));
        }
      }
      // ---- end of the piece ----
      const bool mine = x0 < jobs;             // this group has an accumulator
      const bool joined = nq == 1 && jobs >= 2;
      if (mine) {
        mbar_wait(bar(kOFull + grp), n_o & 1, abort_flag, status, d.wait_ns);
        ++n_o;
        tc_fence_after();
      }
      float m_tot = m_ref, l_tot = l_run, w_me = 1.f, w_ot = 0.f;
      if (joined) {                            // both groups have seen this row: each takes half of the channels
        xch[(grp * 2 + 0) * 128 + row] = m_ref;
        xch[(grp * 2 + 1) * 128 + row] = l_run;
        tc_fence_before();
        asm volatile("bar.sync 1, 256;" ::: "memory");
        tc_fence_after();
        const float m_ot = xch[((grp ^ 1) * 2 + 0) * 128 + row], l_ot = xch[((grp ^ 1) * 2 + 1) * 128 + row];
        m_tot = fmaxf(m_ref, m_ot);
        w_me = (m_ref == -INFINITY) ? (l_run == 0.f ? 0.f : l_run) : fast_ex2(m_ref - m_tot);
        w_ot = (m_ot == -INFINITY) ? (l_ot == 0.f ? 0.f : l_ot) : fast_ex2(m_ot - m_tot);
        l_tot = l_run * w_me + l_ot * w_ot;
      }
      const bool writer = joined || mine || (jobs == 0 && grp < nq);
      if (writer && warp_on) {
        const int c_lo = joined ? grp * 2 : 0, c_hi = joined ? c_lo + 2 : 4;   // pieces of 32 channels
        const int64_t r_out = p.row0 + qt * bmp + po;
        const int qh = hu.head[p.unit] * G + hs;
        const bool wr = row_ok && (p.slot >= 0 || hu.writes(p.unit, row_ok ? qh : 0));
        // (a sum that is no number stays one: only a row that saw nothing is 0)
        const float inv = p.slot >= 0 ? 1.f : l_tot == 0.f ? 0.f : 1.f / l_tot;
        const float f_me = w_me * inv, f_ot = w_ot * inv;
        const int64_t prow = ((int64_t)p.slot * plan.slot_rows + qt * 128 + row);
        for (int c4 = c_lo; c4 < c_hi; ++c4) {
          uint32_t r[32], r2[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) r[e] = 0u;
          if (mine) RTP_TMEM_LD32(r, tmem_o + c4 * 32);
          if (joined) RTP_TMEM_LD32(r2, tmem_o2 + c4 * 32);
          tc_wait_ld();
          float o[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = __uint_as_float(r[e]) * f_me;
          if (joined) {
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = fmaf(__uint_as_float(r2[e]), f_ot, o[e]);
          }
          if (l_tot == 0.f) {                  // (accumulators of keys that were all masked, or none)
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = 0.f;
          }
          if (wr && p.slot >= 0) {
            float4* dst = reinterpret_cast<float4*>(plan.o + prow * kHeadDim + c4 * 32);
#pragma unroll
            for (int e = 0; e < 8; ++e) dst[e] = make_float4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
          } else if (wr) {
            uint4* dst = reinterpret_cast<uint4*>(out + (r_out * d.n_q + qh) * kHeadDim + c4 * 32);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              uint32_t w[4];
#pragma unroll
              for (int y = 0; y < 4; ++y) {
                const __nv_bfloat162 v = __floats2bfloat162_rn(o[8 * e + 2 * y], o[8 * e + 2 * y + 1]);
                w[y] = *reinterpret_cast<const uint32_t*>(&v);
              }
              dst[e] = make_uint4(w[0], w[1], w[2], w[3]);
            }
          }
        }
        if (wr && c_lo == 0) {
          if (p.slot >= 0) {
            *reinterpret_cast<float2*>(plan.ml + prow * 2) = make_float2(m_tot, l_tot);
          } else if (lse) {
            lse[r_out * d.n_q + qh] = l_tot == 0.f ? -INFINITY : (m_tot + log2f(l_tot)) * kLn2;
          }
        }
      }
      if (joined) {                            // the other group's accumulator is no longer read
        tc_fence_before();
        asm volatile("bar.sync 1, 256;" ::: "memory");
        tc_fence_after();
      }
    }
  }

  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {                           // copies that are still under way land before the block's memory is given up
    const unsigned long long t0 = global_ns();
    while (global_ns() - t0 < 1000000ull) __nanosleep(1000);
  }
  if (warp == 8) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(*tmem_slot), "r"(512) : "memory");
  }
}

// ---- merge: a warp per row of a cut unit ---------------------------------------------------------------
// The first CTA's last piece and the others' first ones, in their order.  What the first two left is requested before it is known
// how much it counts: most units are cut once.
constexpr int kMergeWarps = 8;
__global__ void __launch_bounds__(kMergeWarps * 32) merge_kernel(const __grid_constant__ HeadUnits hu, const __grid_constant__ Plan plan,
                                                                 const int G, const int bmp, const int n_q, const int rows,
                                                                 __nv_bfloat16* __restrict__ out, float* __restrict__ lse) {
  chain_wait();
  const int lane = threadIdx.x & 31, n = __ldcg(plan.n_merge) * rows;
  for (int item = (int)(blockIdx.x * kMergeWarps + (threadIdx.x >> 5)); item < n; item += (int)gridDim.x * kMergeWarps) {
    const int u = item / rows, y = item - u * rows;
    const int4* src = reinterpret_cast<const int4*>(plan.merge + u);
    const int4 a = __ldcg(src), b = __ldcg(src + 1);   // row0, n_pos, unit, id; first and last CTA
    const int po = y / G, hs = y - po * G, qt = po / bmp, row = qt * 128 + (po - qt * bmp) * G + hs;
    const int qh = hu.head[a.z] * G + hs;
    if (po >= a.y || !hu.writes(a.z, qh)) continue;
    auto part = [&](int slot) { return __ldcg(reinterpret_cast<const float4*>(plan.o + ((int64_t)slot * plan.slot_rows + row) * kHeadDim) + lane); };
    const float4 o0 = part(2 * b.x + 1), o1 = part(2 * min(b.x + 1, plan.n_ctas - 1));
    float m = -INFINITY, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int c0 = b.x; c0 <= b.y; c0 += 32) {
      const int c = c0 + lane, slot = 2 * c + (c == b.x);
      float2 ml = make_float2(-INFINITY, 0.f);
      int id = -1;
      if (c <= b.y) {
        id = __ldcg(plan.part_id + slot);
        ml = __ldcg(reinterpret_cast<const float2*>(plan.ml) + (int64_t)slot * plan.slot_rows + row);
      }
      const bool there = id == a.w;
      if (!there) ml = make_float2(-INFINITY, 0.f);
      const float m_new = fmaxf(m, warp_max(ml.x));
      const float mb = m_new == -INFINITY ? 0.f : m_new;
      // (a sum without a maximum is 0, or no number, which it has to stay)
      const float f = m == -INFINITY ? 1.f : fast_ex2(m - mb), w = ml.x == -INFINITY ? ml.y : fast_ex2(ml.x - mb);
      m = m_new;
      l = l * f + warp_sum(ml.y * w);
      o.x *= f; o.y *= f; o.z *= f; o.w *= f;
      uint32_t todo = __ballot_sync(0xffffffffu, there);
      while (todo) {
        const int j = __ffs(todo) - 1;
        todo &= todo - 1;
        const float wj = __shfl_sync(0xffffffffu, w, j);
        const int at = c0 + j;
        const float4 v = at == b.x ? o0 : at == b.x + 1 ? o1 : part(2 * at);
        o.x = fmaf(v.x, wj, o.x); o.y = fmaf(v.y, wj, o.y); o.z = fmaf(v.z, wj, o.z); o.w = fmaf(v.w, wj, o.w);
      }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const __nv_bfloat162 p = __floats2bfloat162_rn(o.x * inv, o.y * inv), q = __floats2bfloat162_rn(o.z * inv, o.w * inv);
    const int64_t at = (int64_t)(a.x + po) * n_q + qh;
    reinterpret_cast<uint2*>(out + at * kHeadDim)[lane] = make_uint2(*reinterpret_cast<const uint32_t*>(&p), *reinterpret_cast<const uint32_t*>(&q));
    if (lse && lane == 0) lse[at] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
  }
}

Plan carve(void* ws, int G, int n_units, int64_t n_chunks, int64_t R, int sm_count, size_t* bytes) {
  Plan p = {};
  p.n_ctas = std::min(sm_count, 1024);
  const int bmp = kTile / G;
  const int64_t units = (R / (2 * bmp) + n_chunks) * n_units;
  p.max_units = (int)std::min<int64_t>(units, 0x7fffffff);
  p.slot_rows = R > bmp ? 256 : (int)(R * G);
  char* base = reinterpret_cast<char*>(ws);
  size_t off = 0;
  auto take = [&](size_t n) {
    char* r = base + off;
    off += (n + 255) & ~(size_t)255;
    return r;
  };
  p.n_merge = reinterpret_cast<int32_t*>(take(4));
  p.piece_begin = reinterpret_cast<int32_t*>(take((size_t)(p.n_ctas + 1) * 4));
  p.part_id = reinterpret_cast<int32_t*>(take((size_t)p.n_ctas * 8));
  p.merge = reinterpret_cast<MergeUnit*>(take((size_t)p.n_ctas * sizeof(MergeUnit)));
  p.pieces = reinterpret_cast<Piece*>(take((size_t)(units + p.n_ctas) * sizeof(Piece)));
  p.before = reinterpret_cast<int64_t*>(take((size_t)(units + 1) * 8));
  p.ml = reinterpret_cast<float*>(take((size_t)2 * p.n_ctas * p.slot_rows * 8));
  p.o = reinterpret_cast<float*>(take((size_t)2 * p.n_ctas * p.slot_rows * kHeadDim * 4));
  *bytes = off;
  return p;
}

size_t plan_smem(int64_t n_chunks) { return plan_lists(n_chunks) + (n_chunks <= kKeptChunks ? kKeptUnits * sizeof(Piece) : 0); }

}  // namespace

size_t attn_chunks_workspace_bytes(const Dims& d, int64_t n_chunks, int64_t R, int sm_count) {
  size_t bytes = 0;
  carve(nullptr, d.group, std::min(2 * d.n_kv, kMaxUnits), n_chunks, R, sm_count, &bytes);
  return bytes;
}

cudaError_t launch_attn_chunks(const CacheView& cv, const CacheView& lv, const Dims& d, const ChunkHeads& ch, const __nv_bfloat16* q,
                               const int32_t* chunk_seq, const int32_t* chunk_start, const int32_t* row_offsets, int64_t n_chunks,
                               int64_t R, __nv_bfloat16* out, float* lse, void* ws, size_t ws_bytes, int32_t* status, int sm_count,
                               cudaStream_t st) {
  if (n_chunks == 0 || R == 0 || ch.n == 0) return cudaSuccess;
  HeadUnits hu = {};
  for (int i = 0; i < RTP_MAX_Q_HEADS / 32; ++i) hu.ret_q[i] = ch.ret_q[i];
  for (int i = 0; i < ch.n; ++i) {
    hu.head[i] = ch.head[i];
    hu.flags[i] = (uint8_t)((ch.local[i] ? kLocal : 0) | (ch.skip_ret[i] ? kSkipRet : 0) | (ch.skip_other[i] ? kSkipOther : 0) |
                            (ch.local[i] && lv.n_kv > 0 ? kLocalPool : 0));
  }
  hu.n = ch.n;
  const int bmp = kTile / d.group;
  size_t need = 0;
  Plan plan = carve(ws, d.group, ch.n, n_chunks, R, sm_count, &need);
  if (need > ws_bytes) return cudaErrorMemoryAllocation;
  if ((int64_t)plan.max_units + plan.n_ctas >= ((int64_t)1 << 31) - 1) return cudaErrorNotSupported;
  Maps maps = {};
  const int swz = (int)CU_TENSOR_MAP_SWIZZLE_128B;
  cudaError_t e = make_heads_map(&maps.q, q, R, d.n_q, d.group, bmp, swz);
  if (e == cudaSuccess && cv.n_kv > 0) e = encode_rows_map(&maps.k, cv.k, (int64_t)cv.num_pages * cv.n_kv * kPage, kHeadDim, 64, kPage, swz);
  if (e == cudaSuccess && cv.n_kv > 0) e = encode_rows_map(&maps.v, cv.v, (int64_t)cv.num_pages * cv.n_kv * kPage, kHeadDim, 64, kPage, swz);
  if (e == cudaSuccess && lv.n_kv > 0) e = encode_rows_map(&maps.lk, lv.k, (int64_t)lv.num_pages * lv.n_kv * kPage, kHeadDim, 64, kPage, swz);
  if (e == cudaSuccess && lv.n_kv > 0) e = encode_rows_map(&maps.lv, lv.v, (int64_t)lv.num_pages * lv.n_kv * kPage, kHeadDim, 64, kPage, swz);
  if (e != cudaSuccess) return e;
  static PerDeviceOnce once_plan, once_attn;
  e = set_dyn_smem_once(plan_kernel, (int)std::max(plan_smem(kMaxChunks), plan_smem(kKeptChunks)), once_plan);
  if (e == cudaSuccess) e = set_dyn_smem_once(attn_chunks_kernel, kSmem, once_attn);
  if (e != cudaSuccess) return e;
  bool ring = false;
  for (int i = 0; i < ch.n; ++i) ring = ring || (hu.flags[i] & kLocalPool);
  const ChunkArgs a = {chunk_seq, chunk_start, row_offsets, (int32_t)n_chunks, d.group, bmp, R,
                       ring ? (int64_t)lv.ring_pages * kPage : 0, ring ? (int64_t)lv.max_pages * kPage : 0};
  (void)launch_chained(plan_kernel, dim3(1), dim3(plan.n_ctas <= 512 ? 512 : kPlanThreads), plan_smem(n_chunks), st, a, cv, hu, plan, d.n_sink, d.window, status);
  e = cudaGetLastError();
  if (e != cudaSuccess) return e;              // (without its plan the attention would take what the workspace holds for one)
  (void)launch_chained(attn_chunks_kernel, dim3(plan.n_ctas), dim3(kThreads), (size_t)kSmem, st, maps, cv, lv, hu, plan, d, bmp, out, lse, status);
  e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  // sequences that are too short to be cut need no merge
  if (((int64_t)std::max(cv.max_pages, lv.max_pages) * kPage + kTile - 1) / kTile >= 2 * kSnap) {
    const int rows = (int)std::min<int64_t>(R, 2 * bmp) * d.group;
    const int64_t blocks = std::min<int64_t>(((int64_t)plan.n_ctas * rows + kMergeWarps - 1) / kMergeWarps, (int64_t)8 * sm_count);
    (void)launch_chained(merge_kernel, dim3((unsigned)blocks), dim3(kMergeWarps * 32), 0, st, hu, plan, d.group, bmp, d.n_q, rows, out, lse);
    return cudaGetLastError();
  }
  return cudaSuccess;
}

}  // namespace rtp
