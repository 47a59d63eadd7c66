// Decode attention (the sets of attn_rows.cu) on a 4-bit K/V cache: o = softmax(sm_scale q K^T) V with K and V taken
// as codes and scales, 144 bytes per (token, KV head) where the bf16 cache has 512.
//
// Layout of the work: a (row, KV head or listed query head) is split over CTAs, a CTA over four warps, a warp takes tiles
// of 32 tokens.  Tiles are copied to a ring in shared memory by 16-byte cp.async, two tiles ahead.
//
// The contractions run with the TOKENS as the 16 rows of the MMA (m16n8k16, fp16 -> fp32) and the up to eight query heads
// of the group as its columns:
//   S^T = K Q^T   A = 16 tokens x 16 channels.  The channels of a k-step may be any as long as Q has the same, so lane
//                 (g, c) of the fragment takes channels 32 c .. 32 c + 31 of its two tokens: one 16-byte read each.
//   O^T = V^T P^T A = 16 channels x 16 tokens.  Lane (g, c) takes channels 16 g .. 16 g + 15 (one scale group) of four
//                 tokens.  P^T comes from S^T by movmatrix.  An MMA register holds two values of the contracted index, a
//                 conversion gives two channels of one token:
//     groups of 8   the nibbles of two tokens are interleaved into bytes first, so that the pair is (token, token');
//     groups <= 4   half of the eight columns would be idle.  The pair is (even channel, odd channel) of one token, columns
//                   0 .. 3 have P of the heads in the even place and 0 in the odd one, columns 4 .. 7 the reverse: they
//                   come out as the sums of the even and of the odd channels.  As many MMAs, no interleaving, and half
//                   the accumulators.
// A single head (lists and pages of one query head) has eight columns to itself: column n of S^T gets the channels of scale
// group 2 n (or 2 n - 7) alone, K goes in without its scales, and eight products per token bring them in afterwards.
// What is decoded is exact in fp16 (kv4.cuh).  Queries are scaled by a power of two per head, so that
// their largest channel is near 2^9: the rounding to fp16 then costs 2^-34 of it at most, for any bf16 input.
// Probabilities are relative to a reference that trails the running maximum by at most 2^8 and are shifted up by 2^7: they
// fit fp16 (11 bits; bf16 has 8), down to 2^-21 of the reference without a loss.  Sums are fp32.
//
// What bounds it: 484 warp instructions per 32 tokens and KV head (128 conversions, 128 products with scales, 32 MMAs, 32 shared
// reads, 9 copies; an issue slot in two of three cycles) next to 4.6 KB.  4 x 512K tokens, 8 KV heads, groups of 4 (2.4 GB):
// 367 to 390 us = 6.2 to 6.6 TB/s from a cold card, 430 to 470 at its power limit; a tenth of the tokens in lists per head, random rows:
// 74 us, bound by DRAM's 64-byte pieces (192 bytes for each of 1.63 M list entries, 4.2 TB/s; a token that two heads list is gathered twice).
#include "kv4.cuh"

namespace rtp {

namespace {

constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr int kPartial = kHeadDim + 2;                       // a split's result: acc[128], m, l
constexpr int kMaxSplits = 512;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr int kTileTok = 32;                                 // two MMA tiles of 16 tokens
constexpr int kTilesPerPage = kPage / kTileTok;
constexpr int kStages = 3;                                   // tiles of a warp in shared memory
constexpr int kTileV = kTileTok * kKv4TokBytes;              // K codes, V codes (from here), scales (from kTileS)
constexpr int kTileS = 2 * kTileV;
constexpr int kTileBytes = kTileS + kTileTok * kKv4ScaleBytes;   // 4608
constexpr int kSmemBytes = kWarps * kStages * kTileBytes;    // 54 KB: four CTAs per SM
constexpr uint32_t kFull = 0xffffffffu;
constexpr float kLag = 8.f;    // the reference of the softmax may trail the maximum by this much (log2)
constexpr float kLift = 7.f;   // probabilities are multiplied by 2^kLift: at most 2^15 < 65504

__device__ __forceinline__ void cp16z(uint32_t dst, const void* src, bool valid) {
  const int sz = valid ? 16 : 0;
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(sz) : "memory");
}
__device__ __forceinline__ void cp16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ uint4 lds_v4(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint2 lds_v2(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t lds_u8(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b) {
  const __half2 r = __hmul2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  const __half2 r = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
__device__ __forceinline__ void mma_acc(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <int G, int SET>
__global__ void __launch_bounds__(kThreads, 4) attn_rows4_kernel(
    const __grid_constant__ CacheView cv, const __grid_constant__ Dims d, const __grid_constant__ HeadMaps hm,
    const __grid_constant__ Rows rows, const int n_units,
    const __nv_bfloat16* __restrict__ q, const int32_t* __restrict__ sel_idx, const int64_t sel_stride,
    const int32_t* __restrict__ sel_count, __nv_bfloat16* __restrict__ out, float* __restrict__ lse,
    float* __restrict__ partial, const int n_splits, int32_t* status) {
  chain_wait();
  static_assert(G >= 1 && G <= 8, "the query heads of a KV group are the eight columns of the MMA");
  extern __shared__ __align__(128) unsigned char smem_rows4[];

  const int64_t r = blockIdx.x / n_units;
  const int u = blockIdx.x % n_units;
  const int split = blockIdx.y;
  const int lane = threadIdx.x & 31, warp = __shfl_sync(kFull, (int)(threadIdx.x >> 5), 0);   // (uniform for the compiler)
  const int g = lane >> 2, c = lane & 3;

  int qh0, kvh;
  if (SET == kSetList || SET == kSetPages) {
    qh0 = hm.ret_q_head[u];
    kvh = qh0 / d.group;
  } else {
    kvh = hm.kv_list[u];
    qh0 = kvh * d.group;
  }
  // Head of column n of the MMAs: n, or n % 4 in groups of up to four.  head_b: of column g (queries), head: of this lane's
  // columns 2 c and 2 c + 1 in the results.
  constexpr bool kPairs = G <= 4, kSingle = G == 1;
  constexpr int H = kSingle ? 1 : 2;     // heads per lane
  constexpr int kTilesO = kPairs ? 4 : 8;
  const int head_b = kSingle ? 0 : kPairs ? g & 3 : g;
  const int head[2] = {kSingle ? 0 : kPairs ? (2 * c) & 3 : 2 * c, kSingle ? 0 : kPairs ? (2 * c + 1) & 3 : 2 * c + 1};
  uint4 qv[4];   // requested now, looked at when the first tiles are on their way
#pragma unroll
  for (int i = 0; i < 4; ++i)
    qv[i] = head_b < G ? __ldg(reinterpret_cast<const uint4*>(q + ((int64_t)r * d.n_q + qh0 + head_b) * kHeadDim + 32 * c) + i)
                       : make_uint4(0u, 0u, 0u, 0u);
  const int seq = rows.row_seq(r);
  int n_keys = rows.row_pos(r) + 1;
  {
    const int sl = (seq >= 0 && seq < cv.batch) ? min(cv.seq_lens[seq], cv.cap_tokens) : 0;   // (never beyond the block table)
    if (n_keys > sl) {
      if (threadIdx.x == 0) set_status(status, RTP_ERR_INVALID);
      n_keys = sl;
    }
    if (n_keys < 0) n_keys = 0;
  }

  // The set as tiles of 32: entries of the list, or half a page (of which the tokens outside the set are masked).
  int n_ent = 0, ns = 0, wlo = 0, sink_tiles = 0, n_total;
  const int32_t* ids = nullptr;
  if (SET == kSetList || SET == kSetPages || SET == kSetUnion) {
    const int64_t at = r * (SET == kSetUnion ? n_units : d.n_ret) + u;
    n_ent = (int)max(min((int64_t)sel_count[at], sel_stride), (int64_t)0);
    ids = sel_idx + at * sel_stride;
    n_total = SET == kSetList ? (n_ent + kTileTok - 1) / kTileTok : n_ent * kTilesPerPage;
  } else if (SET == kSetLocal) {
    ns = min(d.n_sink, n_keys);
    wlo = max(ns, n_keys - d.window);
    sink_tiles = (ns + kTileTok - 1) / kTileTok;
    n_total = sink_tiles + (n_keys > wlo ? (n_keys + kTileTok - 1) / kTileTok - wlo / kTileTok : 0);
  } else {
    n_total = (n_keys + kTileTok - 1) / kTileTok;
  }
  const int per = ((n_total + n_splits - 1) / n_splits + kTilesPerPage - 1) / kTilesPerPage * kTilesPerPage;
  const int first = min(n_total, split * per);
  const int n_tiles = min(n_total, first + per) - first;
  const int n_mine = n_tiles > warp ? (n_tiles - warp + kWarps - 1) / kWarps : 0;   // tiles first + warp, + 4, ...

  // O^T, rows of tile i: byte 8 g + 2 i (elements 0, 1: columns 2 c, 2 c + 1) and byte 8 g + 2 i + 1 (2, 3), the column's half
  // of either; in groups of 8: channels 16 g + 2 i and 16 g + 2 i + 1
  float o[kTilesO][4];
#pragma unroll
  for (int i = 0; i < kTilesO; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
  // Reference of the softmax, less the lift, for the lane's heads; none before a head's first token.  While a column of
  // the warp has none, every tile goes through the branch that sets it (limit = -inf).
  float base[H], l[H], limit = head[0] < G ? -INFINITY : kLift + kLag;
  bool empty[H];   // (columns beyond the group count as set)
#pragma unroll
  for (int j = 0; j < H; ++j) {
    base[j] = l[j] = 0.f;
    empty[j] = head[j] < G;
  }

  const int kslot = cv.kv_slot[kvh];
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem_rows4) + warp * kStages * kTileBytes;
  const uint8_t* kp = reinterpret_cast<const uint8_t*>(cv.k);
  const uint8_t* vp = reinterpret_cast<const uint8_t*>(cv.v);
  const int tok_k = (g >> 1) + 4 * (g & 1);   // token of MMA row g (row g + 8: tok_k + 8)
  // groups of up to four: the first or second of two packed probabilities into the half that column g multiplies
  const uint32_t place[2] = {g < 4 ? 0x4410u : 0x1044u, g < 4 ? 0x4432u : 0x3244u};

  // Where a tile lives is found in steps, each a tile after the one that requested it: entry -> token -> page -> row.
  // List sets: lane t looks after token t of the tile.  Other sets: all lanes look after the tile's page.
  auto raw_entry = [&](int i) -> int {
    if (i >= n_mine) return -1;
    const int tile = first + warp + i * kWarps;
    if (SET == kSetList) return tile * kTileTok + lane < n_ent ? __ldg(ids + tile * kTileTok + lane) : -1;
    if (SET == kSetPages || SET == kSetUnion) return __ldg(ids + tile / kTilesPerPage);
    return 0;
  };
  // the token of this lane (list), or the first token of the tile; -1: none
  auto token_of = [&](int i, int entry) -> int {
    if (i >= n_mine) return -1;
    const int tile = first + warp + i * kWarps;
    if (SET == kSetList) {
      if (entry >= 0 && entry < n_keys) return entry;
      if (tile * kTileTok + lane < n_ent) set_status(status, RTP_ERR_INVALID);
      return -1;
    }
    if (SET == kSetPages || SET == kSetUnion) {
      const int page = SET == kSetUnion ? entry & 0xffffff : entry;
      if (page < 0 || n_keys == 0 || page > ((n_keys - 1) >> kPageShift)) {
        set_status(status, RTP_ERR_INVALID);
        return -1;
      }
      return page * kPage + (tile % kTilesPerPage) * kTileTok;
    }
    if (SET == kSetLocal) return tile < sink_tiles ? tile * kTileTok : (wlo / kTileTok + tile - sink_tiles) * kTileTok;
    return tile * kTileTok;
  };
  const int32_t* table = cv.block_table + (int64_t)seq * cv.max_pages;
  auto raw_phys = [&](int tok) -> int {   // (only the local heads' pool can be a ring)
    const int page = tok >> kPageShift;
    return tok >= 0 ? __ldg(table + (SET == kSetLocal ? page_entry(cv, page) : page)) : 0;
  };
  // tokens of the tile that belong to the set, one bit each
  auto valid_mask = [&](int i, int tok) -> uint32_t {
    if (SET == kSetList) return __ballot_sync(kFull, tok >= 0);
    if (tok < 0) return 0u;
    int lo = 0, hi = n_keys;
    if (SET == kSetLocal) {
      if (first + warp + i * kWarps < sink_tiles) hi = ns; else lo = wlo;
    }
    const int a = lo - tok, b = tok + kTileTok - hi;   // tokens missing at the front and at the end
    uint32_t m = kFull;
    if (SET == kSetLocal && a > 0) m = a < kTileTok ? m << a : 0u;
    if (b > 0) m = b < kTileTok ? m & (kFull >> b) : 0u;
    return m;
  };
  // Copies a tile to its stage.  Lane (t, chunk) = (lane / 4, lane % 4) takes chunk `chunk` of tokens t, t + 8, ..; lane t the
  // scales of token t.  The K rows of 16 tokens lie in the order of the MMA rows, the chunks of a V row are exchanged in pairs
  // by bit 1 of the token number: either way the reads below touch every bank once.  Tokens outside the set are filled with
  // zeros.  (A row number fits 32 bits: 2^32 rows of 144 bytes are more than the device's memory.)
  const uint32_t dk = ring + (2 * (g & 3) + (g >> 2)) * kKv4TokBytes + c * 16;
  const uint32_t dv = ring + kTileV + g * kKv4TokBytes + ((c ^ (g & 2)) << 4);
  const uint32_t ds = ring + kTileS + lane * kKv4ScaleBytes;
  auto issue = [&](uint32_t at, int tok, int phys, uint32_t mask) {
    if ((unsigned)phys >= (unsigned)cv.num_pages) {
      set_status(status, RTP_ERR_INVALID);
      phys = 0;
    }
    const uint32_t row = ((uint32_t)phys * cv.n_kv + kslot) * kPage + (tok & (kPage - 1));
    if (SET == kSetList) {
      const uint32_t mine = mask >> lane & 1u ? row : 0u;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bool ok = (mask >> (g + 8 * j)) & 1u;
        const int64_t off = (int64_t)__shfl_sync(kFull, mine, g + 8 * j) * kKv4TokBytes + c * 16;
        cp16z(dk + at + j * 8 * kKv4TokBytes, kp + off, ok);
        cp16z(dv + at + j * 8 * kKv4TokBytes, vp + off, ok);
      }
      cp16z(ds + at, cv.kv_scales + (int64_t)mine * kKv4ScaleBytes, mask >> lane & 1u);
      return;
    }
    const int64_t off = (int64_t)row * kKv4TokBytes + lane * 16, off_s = (int64_t)(row + lane) * kKv4ScaleBytes;
    if (mask == kFull) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        cp16(dk + at + j * 8 * kKv4TokBytes, kp + off + j * 8 * kKv4TokBytes);
        cp16(dv + at + j * 8 * kKv4TokBytes, vp + off + j * 8 * kKv4TokBytes);
      }
      cp16(ds + at, cv.kv_scales + off_s);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bool ok = (mask >> (g + 8 * j)) & 1u;
        const int64_t o_j = ok ? off + j * 8 * kKv4TokBytes : 0;
        cp16z(dk + at + j * 8 * kKv4TokBytes, kp + o_j, ok);
        cp16z(dv + at + j * 8 * kKv4TokBytes, vp + o_j, ok);
      }
      const bool ok = (mask >> lane) & 1u;
      cp16z(ds + at, cv.kv_scales + (ok ? off_s : 0), ok);
    }
  };

  uint32_t mask_st[kStages - 1], flag_st[kStages - 1];   // of the tiles in the ring
#pragma unroll
  for (int x = 0; x < kStages - 1; ++x) {
    const int e = raw_entry(x), tok = token_of(x, e);
    mask_st[x] = valid_mask(x, tok);
    flag_st[x] = (uint32_t)e >> 24;
    issue(x * kTileBytes, tok, raw_phys(tok), mask_st[x]);
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
  // B fragments of the queries: channels 32 c + 4 ks .. + 3 of column g's head in k-step ks
  uint32_t qb[8][2];
  float sc[H];   // logits in log2 units: factors of the lane's heads
  {
    const uint32_t w[16] = {qv[0].x, qv[0].y, qv[0].z, qv[0].w, qv[1].x, qv[1].y, qv[1].z, qv[1].w,
                            qv[2].x, qv[2].y, qv[2].z, qv[2].w, qv[3].x, qv[3].y, qv[3].z, qv[3].w};
    float mx = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i)
      mx = fmaxf(mx, fmaxf(fabsf(__uint_as_float(w[i] << 16)), fabsf(__uint_as_float(w[i] & 0xffff0000u))));
    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
    const int e = max((int)(__float_as_uint(mx) >> 23), 27) - 127;            // floor(log2 mx), at least -100
    const float up = __uint_as_float((uint32_t)(9 - e + 127) << 23);          // 2^(9 - e)
    const float down = d.sm_scale * kLog2e * __uint_as_float((uint32_t)max(e - 9 + 127, 1) << 23);
#pragma unroll
    for (int i = 0; i < 16; ++i)
      qb[i >> 1][i & 1] = pack_f16x2(__uint_as_float(w[i] << 16) * up, __uint_as_float(w[i] & 0xffff0000u) * up);
#pragma unroll
    for (int j = 0; j < H; ++j) sc[j] = __shfl_sync(0xffffffffu, down, 8 * c + 4 * j);   // (from the lane of column 2 c + j)
    if (kSingle) {   // column n < 4: group 2 n, the first half of lane n's channels; column 4 + n: group 2 n + 1
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (g != c + (i < 8 ? 0 : 4)) qb[i >> 1][i & 1] = 0u;
    }
  }
  int ent_a = raw_entry(kStages - 1);                       // the next tile to be copied: its entry, token and page
  int tok_a = token_of(kStages - 1, ent_a), phys_a = raw_phys(tok_a);
  int ent_b = raw_entry(kStages);
  uint32_t rd = 0, wr = (kStages - 1) * kTileBytes;         // stage that is read, stage that is filled

#pragma unroll 1
  for (int i = 0; i < n_mine; ++i) {
    asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
    __syncwarp();
    const uint32_t vm = mask_st[0], flags = flag_st[0];
    {   // tile i + 2 goes where tile i - 1 was
#pragma unroll
      for (int x = 0; x + 1 < kStages - 1; ++x) {
        mask_st[x] = mask_st[x + 1];
        flag_st[x] = flag_st[x + 1];
      }
      const uint32_t m_next = valid_mask(i + kStages - 1, tok_a);
      mask_st[kStages - 2] = m_next;
      flag_st[kStages - 2] = (uint32_t)ent_a >> 24;
      if (i + kStages - 1 < n_mine) issue(wr, tok_a, phys_a, m_next);
      asm volatile("cp.async.commit_group;" ::: "memory");
      ent_a = ent_b;
      tok_a = token_of(i + kStages, ent_a);
      phys_a = raw_phys(tok_a);
      ent_b = raw_entry(i + kStages + 1);
      wr = rd;
    }
    const uint32_t tile = ring + rd;
    rd = rd == (kStages - 1) * kTileBytes ? 0u : rd + kTileBytes;
    // ---- S^T = K Q^T, as exponents relative to the reference: t[x][h][j] = head j of token 16 x + 8 h + tok_k ----
    float t[2][2][H];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      float s[4] = {0.f, 0.f, 0.f, 0.f};
      const uint32_t kt = tile + x * 16 * kKv4TokBytes + lane * 16, st = tile + kTileS + (16 * x + tok_k) * kKv4ScaleBytes;
      const uint4 kk[2] = {lds_v4(kt), lds_v4(kt + 8 * kKv4TokBytes)};
      const int grp = kSingle ? 4 * (c & 1) + (c >> 1) : 2 * c;   // scale groups: of columns 2 c and 2 c + 1, or of the lane's channels
      uint32_t f[2][2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        f[h][0] = lds_u8(st + 8 * h * kKv4ScaleBytes + grp);
        f[h][1] = lds_u8(st + 8 * h * kKv4ScaleBytes + grp + (kSingle ? 2 : 1));
        if (!kSingle) {   // fp16 pairs (scale, scale): code << 7 in both halves, by a product (the ALU is the busiest unit here)
          f[h][0] *= 0x00800080u;
          f[h][1] *= 0x00800080u;
        }
      }
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        uint32_t a[4], b[4];
        e2m1x8_to_f16x2(w == 0 ? kk[0].x : w == 1 ? kk[0].y : w == 2 ? kk[0].z : kk[0].w, a);
        e2m1x8_to_f16x2(w == 0 ? kk[1].x : w == 1 ? kk[1].y : w == 2 ? kk[1].z : kk[1].w, b);
        if (!kSingle) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            a[j] = mul_f16x2(a[j], f[0][w >> 1]);
            b[j] = mul_f16x2(b[j], f[1][w >> 1]);
          }
        }
        mma_acc(s, a[0], b[0], a[1], b[1], qb[2 * w][0], qb[2 * w][1]);
        mma_acc(s, a[2], b[2], a[3], b[3], qb[2 * w + 1][0], qb[2 * w + 1][1]);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (kSingle) {   // the two groups of this lane's columns, then the other lanes' (a code << 20 is scale * 2^-112 in fp32)
          float v = s[2 * h] * (__uint_as_float(f[h][0] << 20) * 0x1p112f);
          v = fmaf(s[2 * h + 1], __uint_as_float(f[h][1] << 20) * 0x1p112f, v);
          v += __shfl_xor_sync(kFull, v, 1);
          v += __shfl_xor_sync(kFull, v, 2);
          s[2 * h] = v;
        }
#pragma unroll
        for (int j = 0; j < H; ++j) t[x][h][j] = fmaf(s[2 * h + j], sc[j], -base[j]);
      }
    }
    if (SET == kSetUnion || vm != kFull) {
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int j = 0; j < H; ++j) {
            bool on = (vm >> (16 * x + 8 * h + tok_k)) & 1u;
            if (SET == kSetUnion) on = on && ((flags >> head[j]) & 1u);
            if (!on) t[x][h][j] = -INFINITY;
          }
    }
    // (V of the first 16 tokens is read here, so that the loads have arrived behind the branch)
    const uint32_t va = tile + kTileV + c * kKv4TokBytes + (((g >> 1) ^ (c & 2)) << 4) + (g & 1) * 8;
    const uint32_t vs = tile + kTileS + c * kKv4ScaleBytes + kKv4ScaleBytes / 2 + g;
    uint2 w[4];
    uint32_t f[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      w[j] = lds_v2(va + j * 4 * kKv4TokBytes);
      f[j] = lds_u8(vs + j * 4 * kKv4ScaleBytes);
    }
    float top[H];
#pragma unroll
    for (int j = 0; j < H; ++j) top[j] = fmaxf(fmaxf(t[0][0][j], t[0][1][j]), fmaxf(t[1][0][j], t[1][1][j]));
    if (__any_sync(kFull, fmaxf(top[0], top[H - 1]) > limit)) {
      // a score lies further above the reference than it may (or there is none yet): the maximum becomes the reference
      limit = kLift + kLag;
#pragma unroll
      for (int j = 0; j < H; ++j) {
#pragma unroll
        for (int x = 4; x <= 16; x <<= 1) top[j] = fmaxf(top[j], __shfl_xor_sync(kFull, top[j], x));
        // (a column without a token so far has the reference -inf, for which `base` holds 0)
        const float above = empty[j] ? (top[j] == -INFINITY ? 0.f : top[j] - kLift) : fmaxf(top[j] - kLift, 0.f);
        const float raised = base[j] + above, rise = raised - base[j];   // (what the sum's rounding leaves of it)
        const float corr = empty[j] ? 0.f : fast_ex2(-rise);
        if (top[j] == -INFINITY && empty[j]) limit = -INFINITY; else empty[j] = false;
#pragma unroll
        for (int x = 0; x < kTilesO; ++x) {
          o[x][j] *= corr;
          o[x][2 + j] *= corr;
          if (kSingle) {
            o[x][1] *= corr;
            o[x][3] *= corr;
          }
        }
        l[j] *= corr;
        base[j] = raised;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          t[x][0][j] -= rise;
          t[x][1][j] -= rise;
        }
      }
    }
    uint32_t pb[2][2];   // P^T of 16 tokens: rows 2 c, 2 c + 1 (and + 8) of column g
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float p[H];
#pragma unroll
        for (int j = 0; j < H; ++j) {
          p[j] = fast_ex2(t[x][h][j]);
          l[j] += p[j];
        }
        pb[x][h] = transpose8x8(pack_f16x2(p[0], p[H - 1]));
      }
    // ---- O^T += V^T P^T: tokens c, c + 4, c + 8, c + 12 of each 16 ----
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      if (x > 0) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          w[j] = lds_v2(va + (16 * x + 4 * j) * kKv4TokBytes);
          f[j] = lds_u8(vs + (16 * x + 4 * j) * kKv4ScaleBytes);
        }
      }
      if constexpr (kPairs) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {   // tokens c + 4 k and c + 4 k + 8
          const uint32_t b0 = __byte_perm(pb[x][0], 0u, place[k]), b1 = __byte_perm(pb[x][1], 0u, place[k]);
          const uint32_t s0 = f[k] * 0x00800080u, s1 = f[k + 2] * 0x00800080u;
#pragma unroll
          for (int hh = 0; hh < 2; ++hh) {
            uint32_t a[4], b[4];
            e2m1x8_to_f16x2(hh ? w[k].y : w[k].x, a);
            e2m1x8_to_f16x2(hh ? w[k + 2].y : w[k + 2].x, b);
#pragma unroll
            for (int i = 0; i < 2; ++i)
              mma_acc(o[2 * hh + i], mul_f16x2(a[2 * i], s0), mul_f16x2(a[2 * i + 1], s0), mul_f16x2(b[2 * i], s1),
                      mul_f16x2(b[2 * i + 1], s1), b0, b1);
          }
        }
      } else {
        const uint32_t f01 = f[1] * 0x00800000u + f[0] * 0x80u, f23 = f[3] * 0x00800000u + f[2] * 0x80u;
        constexpr uint32_t kLow = 0x0f0f0f0fu;
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
          const uint32_t w0 = hh ? w[0].y : w[0].x, w1 = hh ? w[1].y : w[1].x, w2 = hh ? w[2].y : w[2].x, w3 = hh ? w[3].y : w[3].x;
          uint32_t e01[4], d01[4], e23[4], d23[4];   // even and odd channels of the token pairs
          e2m1x8_to_f16x2((w0 & kLow) | ((w1 << 4) & ~kLow), e01);
          e2m1x8_to_f16x2(((w0 >> 4) & kLow) | (w1 & ~kLow), d01);
          e2m1x8_to_f16x2((w2 & kLow) | ((w3 << 4) & ~kLow), e23);
          e2m1x8_to_f16x2(((w2 >> 4) & kLow) | (w3 & ~kLow), d23);
#pragma unroll
          for (int j = 0; j < 4; ++j)
            mma_acc(o[4 * hh + j], mul_f16x2(e01[j], f01), mul_f16x2(d01[j], f01), mul_f16x2(e23[j], f23), mul_f16x2(d23[j], f23),
                    pb[x][0], pb[x][1]);
        }
      }
    }
  }
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // the merge may be set up meanwhile (it waits, too)
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();   // the rings are free: they now hold the warps' partial results

  float* red = reinterpret_cast<float*>(smem_rows4);   // [kWarps][G][kPartial]
#pragma unroll
  for (int j = 0; j < H; ++j) {
#pragma unroll
    for (int x = 4; x <= 16; x <<= 1) l[j] += __shfl_xor_sync(0xffffffffu, l[j], x);
    // (the column is the head's first, or of a pair that counts; a single head's columns are all alike: 0 and 4 count)
    if (head[j] < G && !(kSingle && (c & 1))) {
      float* rw = red + (warp * G + head[j]) * kPartial;
#pragma unroll
      for (int i = 0; i < kTilesO; ++i) {
        if (kPairs) {
          rw[16 * g + 4 * i + (c >> 1)] = o[i][j];
          rw[16 * g + 4 * i + 2 + (c >> 1)] = o[i][2 + j];
        } else {
          rw[16 * g + 2 * i] = o[i][j];
          rw[16 * g + 2 * i + 1] = o[i][2 + j];
        }
      }
      if (g == 0 && (!kPairs || c < 2)) {
        // (scores that are not numbers leave no reference behind, but a sum that is none either: that has to reach the output)
        rw[kHeadDim] = l[j] != l[j] ? 0.f : empty[j] ? -INFINITY : base[j];
        rw[kHeadDim + 1] = l[j];
      }
    }
  }
  __syncthreads();
  // a warp for each head (the next four heads after that), four channels per lane: 2 lane, 2 lane + 1 and 64 more of each
#pragma unroll
  for (int gg0 = 0; gg0 < G; gg0 += kWarps) {
    const int gg = gg0 + warp;
    if (gg >= G) break;
    // (a retrieval head inside a local group is not a local call's; a local head inside a retrieval group not a union call's)
    if ((SET == kSetLocal || SET == kSetUnion) && hm.skips(qh0 + gg)) continue;
    float2 ml[kWarps];
    float mt = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      ml[w] = *reinterpret_cast<const float2*>(red + (w * G + gg) * kPartial + kHeadDim);
      mt = fmaxf(mt, ml[w].x);
    }
    float lt = 0.f;
    float2 a0 = {0.f, 0.f}, a1 = {0.f, 0.f};
    if (mt != -INFINITY) {
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float2* rw = reinterpret_cast<const float2*>(red + (w * G + gg) * kPartial) + lane;
        const float wgt = fast_ex2(ml[w].x - mt);
        const float2 x = rw[0], y = rw[32];
        lt += ml[w].y * wgt;
        a0.x += x.x * wgt;
        a0.y += x.y * wgt;
        a1.x += y.x * wgt;
        a1.y += y.y * wgt;
      }
    }
    if (n_splits == 1) {
      const int64_t oh = (int64_t)r * d.n_q + qh0 + gg;
      const float inv = lt == 0.f ? 0.f : 1.f / lt;   // (a sum that is not a number gives such an output)
      __nv_bfloat162* to = reinterpret_cast<__nv_bfloat162*>(out + oh * kHeadDim) + lane;
      to[0] = __floats2bfloat162_rn(a0.x * inv, a0.y * inv);
      to[32] = __floats2bfloat162_rn(a1.x * inv, a1.y * inv);
      if (lse && lane == 0) lse[oh] = lt == 0.f ? -INFINITY : (mt + log2f(lt)) * kLn2;
    } else {
      float2* p = reinterpret_cast<float2*>(partial + (((int64_t)blockIdx.x * G + gg) * n_splits + split) * kPartial);
      p[lane] = a0;
      p[32 + lane] = a1;
      if (lane == 0) p[kHeadDim / 2] = make_float2(mt, lt);
    }
  }
}

// One CTA per (row, head): log-sum-exp merge of the splits' results.  First the weights of all splits, one thread each,
// then the sums, a warp for every fourth (below eight splits) or eighth split, 32 lanes x four channels each, so that the
// loads of a merge of 74 splits do not follow one another: 17.5 -> 7.4 us for 32 (row, head) pairs with four warps, 2 us less with eight.
template <int SET, int W>
__global__ void __launch_bounds__(32 * W) attn_merge4_kernel(
    const __grid_constant__ Dims d, const __grid_constant__ HeadMaps hm, const int n_units, const int G,
    const float* __restrict__ partial, const int n_splits, __nv_bfloat16* __restrict__ out, float* __restrict__ lse) {
  chain_wait();
  constexpr int kPer = kMaxSplits / (32 * W);
  __shared__ float wgt[kMaxSplits], red[W][kHeadDim], red_m[W], red_l[W];
  const int64_t unit = blockIdx.x / G;
  const int g = blockIdx.x % G;
  const int64_t r = unit / n_units;
  const int u = unit % n_units;
  const int qh = (SET == kSetList || SET == kSetPages) ? hm.ret_q_head[u] : hm.kv_list[u] * d.group + g;
  if ((SET == kSetLocal || SET == kSetUnion) && hm.skips(qh)) return;
  const float* p = partial + ((unit * G + g) * (int64_t)n_splits) * kPartial;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  // the warp's first four results are requested together with the maxima
  constexpr int kAhead = 4;
  float2 x0[kAhead], y0[kAhead];
#pragma unroll
  for (int k = 0; k < kAhead; ++k) {
    const int s = warp + k * W;
    const float2* row = reinterpret_cast<const float2*>(p + (int64_t)s * kPartial) + lane;
    x0[k] = s < n_splits ? row[0] : make_float2(0.f, 0.f);
    y0[k] = s < n_splits ? row[32] : make_float2(0.f, 0.f);
  }
  float m[kPer], l[kPer], mt = -INFINITY;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int s = tid + k * 32 * W;
    const float2 ml = s < n_splits ? *reinterpret_cast<const float2*>(p + (int64_t)s * kPartial + kHeadDim) : make_float2(-INFINITY, 0.f);
    m[k] = ml.x;
    l[k] = ml.y;
    mt = fmaxf(mt, ml.x);
  }
  mt = warp_max(mt);
  if (lane == 0) red_m[warp] = mt;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < W; ++k) mt = fmaxf(mt, red_m[k]);
  float lt = 0.f;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int s = tid + k * 32 * W;
    if (s >= n_splits) break;
    const float w = m[k] == -INFINITY ? 0.f : fast_ex2(m[k] - mt);
    wgt[s] = w;
    lt += l[k] * w;
  }
  lt = warp_sum(lt);
  if (lane == 0) red_l[warp] = lt;
  __syncthreads();
  lt = 0.f;
#pragma unroll
  for (int k = 0; k < W; ++k) lt += red_l[k];
  float2 a0 = {0.f, 0.f}, a1 = {0.f, 0.f};
#pragma unroll
  for (int k = 0; k < kAhead; ++k) {
    const float w = warp + k * W < n_splits ? wgt[warp + k * W] : 0.f;
    a0.x = fmaf(x0[k].x, w, a0.x);
    a0.y = fmaf(x0[k].y, w, a0.y);
    a1.x = fmaf(y0[k].x, w, a1.x);
    a1.y = fmaf(y0[k].y, w, a1.y);
  }
#pragma unroll 4
  for (int s = warp + kAhead * W; s < n_splits; s += W) {
    const float w = wgt[s];
    const float2* q = reinterpret_cast<const float2*>(p + (int64_t)s * kPartial) + lane;
    const float2 x = q[0], y = q[32];
    a0.x = fmaf(x.x, w, a0.x);
    a0.y = fmaf(x.y, w, a0.y);
    a1.x = fmaf(y.x, w, a1.x);
    a1.y = fmaf(y.y, w, a1.y);
  }
  *reinterpret_cast<float2*>(&red[warp][2 * lane]) = a0;
  *reinterpret_cast<float2*>(&red[warp][64 + 2 * lane]) = a1;
  __syncthreads();
  if (tid >= kHeadDim) return;
  float a = 0.f;
#pragma unroll
  for (int k = 0; k < W; ++k) a += red[k][tid];
  const int64_t oh = r * d.n_q + qh;
  out[oh * kHeadDim + tid] = __float2bfloat16_rn(lt == 0.f ? 0.f : a / lt);
  if (lse && tid == 0) lse[oh] = lt == 0.f ? -INFINITY : (mt + log2f(lt)) * kLn2;
}

template <int G, int SET>
cudaError_t launch_typed4(const CacheView& cv, const Dims& d, const HeadMaps& hm, const Rows& rows, int n_units,
                          const __nv_bfloat16* q, const int32_t* sel_idx, int64_t sel_stride, const int32_t* sel_count,
                          __nv_bfloat16* out, float* lse, float* partial, int n_splits, int32_t* status, cudaStream_t st) {
  const dim3 grid((unsigned)(rows.R * n_units), n_splits);
  static PerDeviceOnce once;   // (one per instantiation)
  const cudaError_t attr = set_dyn_smem_once(attn_rows4_kernel<G, SET>, kSmemBytes, once, true);
  if (attr != cudaSuccess) return attr;
  (void)launch_chained(attn_rows4_kernel<G, SET>, grid, dim3(kThreads), kSmemBytes, st, cv, d, hm, rows, n_units, q, sel_idx,
                       sel_stride, sel_count, out, lse, partial, n_splits, status);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess || n_splits == 1) return e;
  const dim3 heads((unsigned)(rows.R * n_units * G));
  if (n_splits < 8)
    (void)launch_chained(attn_merge4_kernel<SET, 4>, heads, dim3(128), 0, st, d, hm, n_units, G, partial, n_splits, out, lse);
  else
    (void)launch_chained(attn_merge4_kernel<SET, 8>, heads, dim3(256), 0, st, d, hm, n_units, G, partial, n_splits, out, lse);
  return cudaGetLastError();
}

}  // namespace

// No plan has more splits than this.
int max_splits4(int64_t units, int64_t max_set, int sm_count) {
  if (units <= 0) return 1;
  const int64_t tiles = (max_set + kTileTok - 1) / kTileTok, cap = (tiles + kWarps - 1) / kWarps;
  return (int)std::max<int64_t>(1, std::min<int64_t>({4LL * sm_count / units, cap, kMaxSplits}));
}

// Split count of a call.  Long sets get one round of the four resident CTAs per SM.  Shorter ones get one or two CTAs per SM:
// they finish as early, with fewer partial results to merge (8 KV heads, us with 1 / 2 / 4 CTAs per SM: 4K tokens 5.8 / 6.7 /
// 8.2, 8K 7.1 / 7.5 / 8.6, 32K 14.2 / 12.3 / 13.1, 64K and more best with 4), as long as a CTA has at most 512 tokens (four
// tiles per warp) per resident CTA; a list, whose tokens come one by one, 128.  `max_set` is what the block table (or the
// list's stride) has room for: a set of that size gives every CTA at least 128 tokens (a tile per warp), and the four warps equally
// many tiles where the count is free.  A shorter one in a wide table is dealt out in pairs of tiles, over fewer of the CTAs.
int plan_splits4(int64_t units, int64_t max_set, int sm_count, bool list) {
  if (units <= 0) return 1;
  const int64_t tiles = (max_set + kTileTok - 1) / kTileTok, cap = std::max<int64_t>(1, (tiles + kWarps - 1) / kWarps);
  const int64_t limit = (list ? 1 : 4) * kWarps;   // tiles
  int64_t s = 1, step = kTilesPerPage;
  for (int k : {1, 2, 4}) {
    s = std::min<int64_t>(std::max<int64_t>(1, k * (int64_t)sm_count / units), cap);
    step = k < 4 ? kWarps : kTilesPerPage;
    if (tiles <= s * k * limit * (s == 1 ? 2 : 1)) break;   // (a single split needs no merge)
  }
  const int64_t per = std::max<int64_t>(1, (tiles + s * step - 1) / (s * step)) * step;
  return (int)std::min<int64_t>(std::max<int64_t>(1, (tiles + per - 1) / per), kMaxSplits);
}

cudaError_t launch_attn_rows4(const CacheView& cv, const Dims& d, const HeadMaps& hm, const Rows& rows, int set, int n_units,
                              const __nv_bfloat16* q, const int32_t* sel_idx, int64_t sel_stride,
                              const int32_t* sel_count, __nv_bfloat16* out, float* lse, float* partial, int n_splits,
                              int32_t* status, cudaStream_t st) {
#define RTP_LAUNCH4(GG, SS)                                                                                               \
  return launch_typed4<GG, SS>(cv, d, hm, rows, n_units, q, sel_idx, sel_stride, sel_count, out, lse, partial, n_splits, \
                               status, st)
#define RTP_GROUPS4(SS)                 \
  switch (d.group) {                    \
    case 1: RTP_LAUNCH4(1, SS);         \
    case 2: RTP_LAUNCH4(2, SS);         \
    case 4: RTP_LAUNCH4(4, SS);         \
    case 8: RTP_LAUNCH4(8, SS);         \
    default: return cudaErrorInvalidValue; \
  }
  switch (set) {
    case kSetList: RTP_LAUNCH4(1, kSetList);
    case kSetPages: RTP_LAUNCH4(1, kSetPages);
    case kSetUnion: RTP_GROUPS4(kSetUnion)
    case kSetLocal: RTP_GROUPS4(kSetLocal)
    default: RTP_GROUPS4(kSetDense)
  }
#undef RTP_GROUPS4
#undef RTP_LAUNCH4
}

}  // namespace rtp
