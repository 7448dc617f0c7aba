// Integer-only attention of ONE new token per sequence over a paged int8 key-value cache.
//
// Per (sequence, query head): s_j = q k_j over the visible keys, M = max s_j, e_j = i-exp(M - s_j) (Algorithm 3),
//   w_j = (e_j b_w + 2^23) >> 24, b_w = floor(p_max 2^24 / i-exp(0)): the weights in u8 (or 7 bits), p_max at the maximum,
//   O = sum w_j v_j, W = sum w_j (exact in 32 bits for 65536 keys),  out = round(O / W S_v / S_ctx)
// with the last quotient as a dyadic multiplier per row, R = floor(b 2^(l-1) / W), l the bit length of W, b / 2^c =
// dyadic(S_v / S_ctx).  The weights are not divided by their sum before the product as in attention_i8.cu: past a few
// hundred keys of similar score every floor(e p_max / sum) would be 0.
//
// i-exp is defined from the row's maximum and its shifts do not commute with a later, larger one, so the sequence is
// split over a CLUSTER of CTAs instead of over independent blocks: every CTA finds the maximum of its keys' scores, the
// maxima meet through distributed shared memory, then every CTA weights its values, and the partial O and W (whole
// numbers, so no order matters) are summed by the CTAs of the cluster, each a part of the results.  Nothing but the result
// is written.
//
// The products run on mma.sync m16n8k32 (s8 x s8, s8 x u8): up to eight query heads of a group, and the kernel is bound by
// the 128 bytes per key and the latency of getting them, not by the tensor pipe (15 % busy).  S^T = Q K^T leaves a lane with one head
// and the very keys whose weights it needs as the B operand of O^T = V^T w; the 16 bytes of a key that a lane copies are
// the operand of both K steps as they come (any order of the 64 dimensions will do if Q has the same); the values are
// transposed on their way out of shared memory (ldmatrix of bytes), four keys to a register.
// Measured, with what one pass leaves in L2 for the next / with nothing there: 64 sequences of up to 2048 keys, 16 heads of their own 28 / 29 us
// (5.2 TB/s, 0.79 of the copy rate); 16 of up to 32768, 32 heads over 4: 33 / 39 us (3.0 TB/s), where neither issue (47 % of the slots) nor
// HBM (39 %) is full: warps wait for loads and barriers, and the CTAs of the long sequences, as many as the short ones have, run on alone
// (SMs are active for 69 % of the time); one of 1000: 5.0 us, a chain of five dependent loads and the barriers of its cluster.
#include <algorithm>

#include "device_utils.cuh"
#include "sm100_ptx.cuh"

namespace ibert {
namespace {

constexpr int kTile = 32;                // keys a warp takes at a time
constexpr int kTileBytes = kTile * kHeadDim;
constexpr int kMaxGroup = 8;             // query heads per CTA
constexpr int kMaxCluster = 8;           // (larger ones find no place on the GPU for long: 16 x 32768 x 32 heads 55 us at 16 where 8 took 38, now 33)
constexpr int kDecMaxSmem = 160 * 1024;

struct DecodeArgs {
  const int8_t *q, *k_cache, *v_cache;
  const int32_t *tables, *lens, *cu;     // cu: null, or [B + 1]: the row of sequence b is cu[b + 1] - 1
  int64_t rows;
  int8_t* out;
  int32_t* status;
  int32_t heads, kv_heads, group, tiles_of_group;     // query heads per kv head, and in pieces of kMaxGroup
  int32_t log_page, max_pages, n_pages, max_len, window, sinks;
  int32_t score_pitch;                   // words of scores per head in shared memory, = 16 mod 32
  LongAttnConsts k;
};

// the same on accumulators of zeros
__device__ __forceinline__ void mma_s8_first(int32_t (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                             uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
               : "=r"(c[0]), "=r"(c[1]), "=r"(c[2]), "=r"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "r"(0));
}
__device__ __forceinline__ void mma_s8(int32_t (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                       uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_s8u8(int32_t (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.u8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// W warps with STAGES tiles of each in flight.  KEEP: the scores stay in shared memory from the maximum to the weights, and the
// exponentials of a head are spread over all threads; else the keys are read a second time (out of L2) and every lane computes
// the weights that it needs itself.  For one or two heads the eight weights per lane and tile would be those of an eighth or a
// quarter of the lanes; for more, the scores' 4 bytes per head and key take the shared memory that the loads in flight need.  Kept / read
// again, us: 8 heads, 64 x 2048 26 / 14, 128 with a window of 1024 33 / 17; 3 heads, 16 x 32768 41 / 33, 4 heads 44 / 33, one of 1000
// 6.6 / 5.5.  Where 3 or 4 heads see few keys and sequences are many, the rule by heads alone loses some: 64 x 2048 12 / 14 and 13 / 14,
// 128 with a window of 1024 13 / 16 and 14 / 16.
template <int W, int STAGES, bool KEEP>
__global__ void __launch_bounds__(32 * W, KEEP ? 5 : 4)
attention_decode_kernel(const __grid_constant__ DecodeArgs a) {
  constexpr int kThreads = 32 * W;
  extern __shared__ __align__(16) uint8_t smem[];
  int32_t* s_score = reinterpret_cast<int32_t*>(smem + W * STAGES * kTileBytes);               // KEEP: [heads][score_pitch]
  __shared__ int32_t s_all_max[kMaxCluster][kMaxGroup];       // by CTA of the cluster
  __shared__ int32_t s_warp_max[W][kMaxGroup];
  __shared__ int32_t s_out[16][32];      // partial O: [4 i + c][lane] holds head 2 t + (c & 1), dimension 16 i + 8 (c >> 1) + g
  __shared__ int32_t s_sum[kMaxGroup];                        // partial W

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const uint32_t rank = ptx::cluster_ctarank();
  int cl;
  asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(cl));
  // (The shared memory of a CTA may be written by another one only once it runs: every CTA says so here and waits for the others
  // before its first store to them, behind its keys.)
  if (cl > 1) ptx::cluster_arrive();
  const int item = (int)blockIdx.x / cl;
  const int piece = item % a.tiles_of_group, pair = item / a.tiles_of_group;
  const int kvh = pair % a.kv_heads;
  const int batch = pair / a.kv_heads;

  for (int i = tid; i < kMaxGroup * kHeadDim; i += kThreads) (&s_out[0][0])[i] = 0;
  if (tid < kMaxGroup) s_sum[tid] = 0;
  ptx::grid_dep_wait();

  // ---- visible keys: j < first and start <= j < len, in tiles of 32: `lead` tiles in front of the window's first one
  int32_t len = ptx::ld_dep(a.lens + batch);
  bool bad = len < 0 || len > a.max_len;
  len = min(max(len, 0), a.max_len);
  int64_t q_row = batch;                 // < 0: no new token, nothing to do
  if (a.cu) {
    const int32_t c0 = ptx::ld_dep(a.cu + batch), c1 = ptx::ld_dep(a.cu + batch + 1);
    q_row = c1 > c0 ? c1 - 1 : -1;
    if (q_row >= a.rows || (c1 > c0 && q_row < 0)) { bad = true; q_row = -1; }
    if (q_row < 0) len = 0;
  }
  const int start = a.window > 0 ? max(len - a.window, 0) : 0, first = min(a.sinks, start);
  const int tile_w = start / kTile, lead = min((first + kTile - 1) / kTile, tile_w);
  const int tiles = len > 0 ? lead + (len + kTile - 1) / kTile - tile_w : 0;
  const int per = (tiles + cl - 1) / cl, i0 = min((int)rank * per, tiles), i1 = min(i0 + per, tiles);
  const int head0 = kvh * a.group + piece * kMaxGroup;
  const int G = min(a.group - piece * kMaxGroup, kMaxGroup);  // query heads of this CTA
  auto first_key = [&](int i) { return (i < lead ? i : i - lead + tile_w) * kTile; };
  auto seen = [&](int key) { return key < len && (key >= start || key < first); };
  // Byte offsets in either cache of keys 0 and 16 of every tile of this CTA.  A page holds whole halves of tiles, and rows of
  // it past the sequence's end may be read as well as any.  Bit 0: some of the half's keys are not visible; -1: none is, or
  // there is no such page: nothing is copied, and whatever the ring holds gets masked scores and weights of 0.
  int64_t* s_place = reinterpret_cast<int64_t*>(s_score + (KEEP ? G * a.score_pitch : 0));
  for (int i = tid; i < 2 * (i1 - i0); i += kThreads) {
    const int key0 = first_key(i0 + (i >> 1)) + 16 * (i & 1);
    int64_t place = -1;
    if (key0 < len && (key0 + 15 >= start || key0 < first)) {
      const int32_t page = ptx::ld_dep(a.tables + (int64_t)batch * a.max_pages + (key0 >> a.log_page));
      if ((uint32_t)page < (uint32_t)a.n_pages) {
        const bool whole = key0 + 16 <= len && (key0 >= start || key0 + 16 <= first);
        place = ((((int64_t)page * a.kv_heads + kvh) << a.log_page) + (key0 & ((1 << a.log_page) - 1))) * kHeadDim + (whole ? 0 : 1);
      } else bad = true;
    }
    s_place[i] = place;
  }
  uint4 q = make_uint4(0, 0, 0, 0);      // 16 bytes of head g, the A operand's rows 0 to 7 (rows 8 to 15 are zeros)
  if (g < G && q_row >= 0) q = ptx::ld_dep(reinterpret_cast<const uint4*>(a.q + (q_row * a.heads + head0 + g) * kHeadDim) + t);
  __syncthreads();                       // s_place, s_out and s_sum are filled

  // ---- a warp's stream of tiles, copied into a ring of its own: its keys, then its values (KEEP), or its keys, then a tile of
  // keys and its values in turn.  The first of the second part are on their way while the CTAs meet.
  uint8_t* ring = smem + warp * STAGES * kTileBytes;
  const int n_tiles = i0 + warp < i1 ? (i1 - i0 - warp + W - 1) / W : 0, n_stream = (KEEP ? 2 : 3) * n_tiles;
  // In a tile of keys, row n of the j-th eight is key 16 (j / 2) + 2 (j & 1) + 4 (n / 2) + (n & 1): a lane's two scores of the
  // eights 2 p and 2 p + 1 are then those of keys 16 p + 4 t .. + 3, the four that a register of transposed values holds.  A
  // tile of values lies in the ring with its 16-byte chunks swizzled: eight rows of a chunk are eight different bank groups.
  const int k_lane = (((g >> 1) << 2) + (g & 1)) * kHeadDim + t * 16, v_lane = lane * 16;
  const uint32_t k_dst = lane * 16, v_dst = g * kHeadDim + ((t ^ ((g >> 1) & 3)) << 4);
  auto issue = [&](int n) {              // tile n of the stream; a lane copies 16 bytes of each of its eight rows
    if (n < n_stream) {
      const int m = n - n_tiles, i = n < n_tiles ? n : (KEEP ? m : m >> 1);
      const bool keys = n < n_tiles || (!KEEP && !(m & 1));
      const longlong2 p = *reinterpret_cast<const longlong2*>(s_place + 2 * (warp + i * W));
      const int8_t* base = keys ? a.k_cache + k_lane : a.v_cache + v_lane;
      const int8_t *lo = base + (p.x & ~int64_t(1)), *hi = base + (p.y & ~int64_t(1));
      const uint32_t dst = ptx::smem_addr(ring + (n & (STAGES - 1)) * kTileBytes) + (keys ? k_dst : v_dst);
      const int second = keys ? 2 * kHeadDim : 8 * kHeadDim;             // from one eight rows of a half to the other
      if (p.x >= 0) {
        ptx::cp_async_16(dst, lo);
        ptx::cp_async_16(dst + 512, lo + second);
      }
      if (p.y >= 0) {
        ptx::cp_async_16(dst + 1024, hi);
        ptx::cp_async_16(dst + 1536, hi + second);
      }
    }
    ptx::cp_async_commit();
  };
  constexpr int32_t kNone = INT32_MIN;
  // scores c[j][e] of head g against keys 16 (j / 2) + 4 t + 2 (j & 1) + e of a tile of keys that this lane copied itself,
  // and whether some of them are masked
  auto scores = [&](int n, int i, int32_t (&c)[4][4]) {
    const uint8_t* tile = ring + (n & (STAGES - 1)) * kTileBytes + lane * 16;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint4 r = *reinterpret_cast<const uint4*>(tile + j * 512);
      mma_s8_first(c[j], q.x, 0u, q.y, 0u, r.x, r.y);
      mma_s8(c[j], q.z, 0u, q.w, 0u, r.z, r.w);
    }
    const int2 flags = make_int2((int)s_place[2 * (warp + i * W)], (int)s_place[2 * (warp + i * W) + 1]);
    const bool masked = (flags.x | flags.y) & 1;              // (-1 has bit 0, too)
    if (masked) {
      const int key0 = first_key(i0 + warp + i * W) + 4 * t;
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e)
          if ((j < 2 ? flags.x : flags.y) == -1 || !seen(key0 + 16 * (j >> 1) + 2 * (j & 1) + e)) c[j][e] = kNone;
    }
    return masked;
  };
#pragma unroll
  for (int n = 0; n < STAGES; ++n) issue(n);

  // ---- the largest score of every head
  int32_t mx = kNone;                    // of head g
  for (int n = 0; n < n_tiles; ++n) {
    ptx::cp_async_wait<STAGES - 1>();
    int32_t c[4][4];
    scores(n, n, c);
    issue(n + STAGES);
#pragma unroll
    for (int j = 0; j < 4; ++j) mx = __vimax3_s32(mx, c[j][0], c[j][1]);
    if (KEEP && g < G) {                 // (in the order of the keys)
      int32_t* s_tile = s_score + g * a.score_pitch + (warp + n * W) * kTile + 4 * t;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<int2*>(s_tile + 16 * (j >> 1) + 2 * (j & 1)) = make_int2(c[j][0], c[j][1]);
    }
  }
  mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
  mx = max(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
  if (t == 0) s_warp_max[warp][g] = mx;
  __syncthreads();
  if (cl > 1) ptx::cluster_wait();       // (every CTA of the cluster runs)
  for (int i = tid; i < cl * kMaxGroup; i += kThreads) {      // this CTA's maxima into every CTA of the cluster
    const int h = i & (kMaxGroup - 1), to = i / kMaxGroup;
    int32_t m = s_warp_max[0][h];
    for (int w = 1; w < W; ++w) m = max(m, s_warp_max[w][h]);
    ptx::st_cluster_s32(ptx::map_to_cta(ptx::smem_addr(&s_all_max[rank][h]), (uint32_t)to), m);
  }
  if (cl > 1) ptx::cluster_sync(); else __syncthreads();

  // ---- weights and O = sum w v
  const LongAttnConsts& k = a.k;
  int32_t acc[4][4] = {};                                     // dims 16 i + g (c < 2) and 16 i + 8 + g x heads 2t, 2t + 1
  auto accumulate = [&](int n, uint32_t w0, uint32_t w1) {    // a tile of values; lane l addresses row l
    const uint32_t row = ptx::smem_addr(ring + (n & (STAGES - 1)) * kTileBytes) + lane * kHeadDim;
    uint32_t v[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) ptx::ldmatrix_b8_t(v[i], row + ((i ^ ((lane >> 1) & 3)) << 4));
    __syncwarp();                        // every lane has read the tile
    issue(n + STAGES);
#pragma unroll
    for (int i = 0; i < 4; ++i) mma_s8u8(acc[i], v[i][0], v[i][1], v[i][2], v[i][3], w0, w1);
  };
  auto pack = [](const uint32_t* e) {    // the upper bytes of four words
    return __byte_perm(__byte_perm(e[0], e[1], 0x0073), __byte_perm(e[2], e[3], 0x0073), 0x5410);
  };
  auto second_part = [&](auto exp_of) {  // exp_of(score, maximum, offset of the folded form)
    if constexpr (KEEP) {
      const int quads = (i1 - i0) * (kTile / 4);
      for (int h = 0; h < G; ++h) {
        int32_t top = kNone;
        for (int c = 0; c < cl; ++c) top = max(top, s_all_max[c][h]);
        const int32_t wk = iexp_folded_offset(k.e, top);
        int32_t* row = s_score + h * a.score_pitch;
        uint32_t sum = 0;
        for (int i = tid; i < quads; i += kThreads) {         // the word takes the place of the first of its four scores
          const int4 s4 = *reinterpret_cast<const int4*>(row + 4 * i);
          const int32_t s[4] = {s4.x, s4.y, s4.z, s4.w};
          uint32_t e[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) e[j] = s[j] == kNone ? 0u : exp_of(s[j], top, wk) * k.b_w + (1u << 23);
          const uint32_t w = pack(e);
          row[4 * i] = (int32_t)w;
          sum = __dp4a(w, 0x01010101u, sum);
        }
        sum = __reduce_add_sync(0xffffffffu, sum);
        if (lane == 0 && sum != 0) atomicAdd(&s_sum[h], (int32_t)sum);
      }
      __syncthreads();
      for (int n = n_tiles; n < n_stream; ++n) {
        ptx::cp_async_wait<STAGES - 1>();
        __syncwarp();                    // every lane's copies of the tile have landed
        const int32_t* s_tile = s_score + g * a.score_pitch + (warp + (n - n_tiles) * W) * kTile + 4 * t;
        accumulate(n, g < G ? (uint32_t)s_tile[0] : 0u, g < G ? (uint32_t)s_tile[16] : 0u);
      }
    } else {
      int32_t top = kNone;               // of head g
      for (int c = 0; c < cl; ++c) top = max(top, s_all_max[c][g]);
      const int32_t wk = iexp_folded_offset(k.e, top);
      uint32_t sum = 0;
      for (int i = 0; i < n_tiles; ++i) {
        const int n = n_tiles + 2 * i;
        ptx::cp_async_wait<STAGES - 1>();
        int32_t c[4][4];
        const bool masked = scores(n, i, c);
        issue(n + STAGES);
        uint32_t w[2];
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          uint32_t e[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            e[j] = exp_of(c[2 * p + (j >> 1)][j & 1], top, wk) * k.b_w + (1u << 23);
          }
          if (masked) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (c[2 * p + (j >> 1)][j & 1] == kNone) e[j] = 0u;
          }
          w[p] = g < G ? pack(e) : 0u;
          sum = __dp4a(w[p], 0x01010101u, sum);
        }
        ptx::cp_async_wait<STAGES - 1>();
        __syncwarp();
        accumulate(n + 1, w[0], w[1]);
      }
      sum += __shfl_xor_sync(0xffffffffu, sum, 1);
      sum += __shfl_xor_sync(0xffffffffu, sum, 2);
      if (t == 0 && sum != 0) atomicAdd(&s_sum[g], (int32_t)sum);
    }
  };
  if (iexp_takes_folded(k.e)) {
    const int64_t mk = iexp_folded_addend(k.e);
    const int32_t neg_m = -(int32_t)k.e.fold_m;
    if (k.e.s_in == 0)
      second_part([&](int32_t s, int32_t, int32_t wk) { return iexp_folded((int32_t)((uint32_t)s + (uint32_t)wk), mk, neg_m, k.e.q_ln2, k.e.q_c); });
    else
      second_part([&](int32_t s, int32_t, int32_t wk) {
        return iexp_folded((int32_t)((uint32_t)s + (uint32_t)wk) >> k.e.s_in, mk, neg_m, k.e.q_ln2, k.e.q_c);
      });
  } else {
    second_part([&](int32_t s, int32_t top, int32_t) { return iexp_dist_wide((uint32_t)top - (uint32_t)s, k.e); });
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int c = 0; c < 4; ++c)
      if (2 * t + (c & 1) < G) atomicAdd(&s_out[4 * i + c][lane], acc[i][c]);
  if (cl > 1) ptx::cluster_sync(); else __syncthreads();

  ptx::grid_dep_launch();                // (not earlier: CTAs of the next kernel would wait in the slots of this one's last ones)
  // ---- every CTA joins and divides its part of the G x 64 results
  for (int i = (int)rank * kThreads + tid; i < G * kHeadDim; i += cl * kThreads) {
    const int h = i / kHeadDim, d = i % kHeadDim;
    const int32_t* part = &s_out[(d >> 4) * 4 + ((d >> 3) & 1) * 2 + (h & 1)][(d & 7) * 4 + (h >> 1)];
    int32_t o = 0;
    uint32_t total = 0;
    for (int c = 0; c < cl; ++c) {
      o += ptx::ld_cluster_s32(ptx::map_to_cta(ptx::smem_addr(part), (uint32_t)c));
      total += (uint32_t)ptx::ld_cluster_s32(ptx::map_to_cta(ptx::smem_addr(&s_sum[h]), (uint32_t)c));
    }
    if (q_row >= 0) a.out[(q_row * a.heads + head0 + h) * kHeadDim + d] = (int8_t)weighted_mean(o, row_share(total, k));
  }
  if (bad) atomicCAS(a.status, 0, IBERT_ERR_VALUE_RANGE);
  if (cl > 1) ptx::cluster_sync();       // nobody leaves while a peer may still read its shared memory
}

}  // namespace

int launch_attention_decode(ibert_ctx* ctx, const int8_t* q, const int8_t* k_cache, const int8_t* v_cache,
                            const int32_t* tables, const int32_t* lens, const int32_t* cu, int64_t rows, int B, int max_pages, int n_pages, int log_page,
                            int max_len, int heads, int kv_heads, int window, int sinks, const LongAttnConsts& k,
                            int8_t* out) {
  DecodeArgs a{};
  a.q = q; a.k_cache = k_cache; a.v_cache = v_cache; a.tables = tables; a.lens = lens; a.cu = cu; a.rows = rows; a.out = out; a.status = ctx->d_status;
  a.heads = heads; a.kv_heads = kv_heads; a.group = heads / kv_heads;
  a.tiles_of_group = (a.group + kMaxGroup - 1) / kMaxGroup;
  a.log_page = log_page; a.max_pages = max_pages; a.n_pages = n_pages; a.max_len = max_len; a.window = window; a.sinks = sinks;
  a.k = k;
  const int64_t items = (int64_t)B * kv_heads * a.tiles_of_group;
  // Tiles of 32 keys that a sequence can have: one more where the window starts inside a tile, and the sinks' own.  The lengths are on the
  // device, so the plan is max_len's, and kept scores take shared memory for that many keys: 64 sequences of up to 2048, 16 heads of
  // their own, 29 us with a max_len of 2048, 31 with 8192, 56 with 32768 and 91 with 65536 (read again: the same with each).
  int64_t tiles = ((int64_t)max_len + kTile - 1) / kTile;
  if (window > 0) tiles = std::min<int64_t>(tiles, ((int64_t)window + kTile - 1) / kTile + 1 + ((int64_t)sinks + kTile - 1) / kTile);
  const bool keep = a.group <= 2;
  const int warps = keep ? 4 : 8, stages = keep ? 4 : 2;
  const int kept = keep ? a.group : 0;
  // (rings, scores, then the places of the tiles' halves)
  auto smem_of = [&](int c) {
    const int64_t n = (tiles + c - 1) / c;
    return (int64_t)warps * stages * kTileBytes + kept * (n * kTile + 16) * 4 + n * 16;
  };
  int cl = 1;
  while (cl < kMaxCluster && items * cl < 2 * ctx->num_sms && (tiles + cl - 1) / cl > warps) cl <<= 1;
  while (cl < kMaxCluster && smem_of(cl) > 112 * 1024) cl <<= 1;
  const int64_t smem = smem_of(cl);
  if (smem > kDecMaxSmem || items * cl > INT32_MAX) return IBERT_ERR_SHAPE;
  a.score_pitch = (int32_t)((tiles + cl - 1) / cl * kTile + 16);
  auto kernel = keep ? attention_decode_kernel<4, 4, true> : attention_decode_kernel<8, 2, false>;
  static bool set[kMaxDevices][2] = {{false}};
  bool& done = set[ctx->device % kMaxDevices][keep ? 1 : 0];
  if (!done) {
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kDecMaxSmem) != cudaSuccess) {
      cudaGetLastError();
      return IBERT_ERR_CUDA;
    }
    done = true;
  }
  return launch_pdl(kernel, dim3((unsigned)(items * cl)), dim3(32 * warps), (size_t)smem, ctx->stream, cl, a);
}

}  // namespace ibert
