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
// split over a CLUSTER of CTAs instead of over independent blocks: every CTA keeps the scores of its keys in shared
// memory, the maxima meet through distributed shared memory, then every CTA weights its values, and the partial
// O and W (whole numbers, so no order matters) are summed by the CTAs of the cluster, each a part of the 64 dimensions.
// K and V are read once; nothing but the result is written.
//
// The products run on mma.sync m16n8k32 (s8 x s8, s8 x u8): eight query heads of a group are the n of a tile, and the
// kernel is bound by the 128 bytes per key, not by the tensor pipe.  A lane's 16 bytes of a key are the A operand of
// both k steps as they come (any order of the 64 dimensions will do if Q has the same); the values of four keys are
// transposed in registers by byte permutes.
#include <algorithm>

#include "device_utils.cuh"
#include "sm100_ptx.cuh"

namespace ibert {
namespace {

constexpr int kDecThreads = 256, kDecWarps = kDecThreads / 32;
constexpr int kTile = 32;                // keys a warp takes at a time
constexpr int kMaxGroup = 8;             // query heads per CTA

struct DecodeArgs {
  const int8_t *q, *k_cache, *v_cache;
  const int32_t *tables, *lens;
  int8_t* out;
  int32_t* status;
  int32_t heads, kv_heads, group, tiles_of_group;     // query heads per kv head, and in pieces of kMaxGroup
  int32_t log_page, max_pages, n_pages, max_len, window, sinks;
  int32_t score_pitch;                   // 32-bit words per head in shared memory, = 16 mod 32
  LongAttnConsts k;
};

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
// bytes of four words, transposed: o[i] = byte i of w[0], w[1], w[2], w[3]
__device__ __forceinline__ void transpose4(const uint32_t* w, uint32_t* o) {
  const uint32_t a = __byte_perm(w[0], w[1], 0x5140), b = __byte_perm(w[0], w[1], 0x7362);
  const uint32_t c = __byte_perm(w[2], w[3], 0x5140), d = __byte_perm(w[2], w[3], 0x7362);
  o[0] = __byte_perm(a, c, 0x5410);
  o[1] = __byte_perm(a, c, 0x7632);
  o[2] = __byte_perm(b, d, 0x5410);
  o[3] = __byte_perm(b, d, 0x7632);
}

// Where key 4 j + t of a tile lies in its 32 scores: a lane then finds the eight keys t, 4 + t, .. of its weights as two
// runs of four words
__device__ __forceinline__ int score_place(int key) {
  const int t = key & 3, j = key >> 2;
  return ((j >> 2) << 4) + (t << 2) + (j & 3);
}

__global__ void __launch_bounds__(kDecThreads)
attention_decode_kernel(const __grid_constant__ DecodeArgs a) {
  extern __shared__ int32_t s_score[];                        // [heads of this CTA][score_pitch]
  __shared__ int32_t s_all_max[16][kMaxGroup];                // by CTA of the cluster
  __shared__ int32_t s_warp_max[kDecWarps][kMaxGroup];
  __shared__ int32_t s_out[kMaxGroup][kHeadDim];              // partial O
  __shared__ int32_t s_sum[kMaxGroup];                        // partial W

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const uint32_t rank = ptx::cluster_ctarank();
  int cl;
  asm("mov.u32 %0, %%cluster_nctaid.x;" : "=r"(cl));
  const int item = (int)blockIdx.x / cl;
  const int piece = item % a.tiles_of_group, pair = item / a.tiles_of_group;
  const int kvh = pair % a.kv_heads, batch = pair / a.kv_heads;
  const int head0 = kvh * a.group + piece * kMaxGroup;
  const int G = min(a.group - piece * kMaxGroup, kMaxGroup);  // query heads of this CTA

  for (int i = tid; i < kMaxGroup * kHeadDim; i += kDecThreads) (&s_out[0][0])[i] = 0;
  if (tid < kMaxGroup) s_sum[tid] = 0;
  ptx::grid_dep_launch();
  ptx::grid_dep_wait();

  // ---- visible keys: j < first and start <= j < len, in tiles of 32: `lead` tiles in front of the window's first one
  int32_t len = ptx::ld_dep(a.lens + batch);
  bool bad = len < 0 || len > a.max_len;
  len = min(max(len, 0), a.max_len);
  const int start = a.window > 0 ? max(len - a.window, 0) : 0, first = min(a.sinks, start);
  const int tile_w = start / kTile, lead = min((first + kTile - 1) / kTile, tile_w);
  const int tiles = len > 0 ? lead + (len + kTile - 1) / kTile - tile_w : 0;
  const int per = (tiles + cl - 1) / cl, i0 = min((int)rank * per, tiles), i1 = min(i0 + per, tiles);
  const int32_t* table = a.tables + (int64_t)batch * a.max_pages;
  const int64_t head_bytes = (int64_t)kHeadDim << a.log_page;
  auto first_key = [&](int i) { return (i < lead ? i : i - lead + tile_w) * kTile; };
  // offset of row `key` of this kv head in either cache; -1: no such page
  auto row_at = [&](int key) -> int64_t {
    const int32_t page = ptx::ld_dep(table + (key >> a.log_page));
    if ((uint32_t)page >= (uint32_t)a.n_pages) return -1;
    return ((int64_t)page * a.kv_heads + kvh) * head_bytes + (int64_t)(key & ((1 << a.log_page) - 1)) * kHeadDim;
  };
  auto seen = [&](int key) { return key < len && (key >= start || key < first); };

  uint4 q = make_uint4(0, 0, 0, 0);
  if (g < G) q = ptx::ld_dep(reinterpret_cast<const uint4*>(a.q + ((int64_t)batch * a.heads + head0 + g) * kHeadDim) + t);

  // ---- scores of this CTA's tiles, and their maximum
  constexpr int32_t kNone = INT32_MIN;
  int32_t mx0 = kNone, mx1 = kNone;                           // of heads 2t and 2t + 1
  for (int i = i0 + warp; i < i1; i += kDecWarps) {
    const int key0 = first_key(i);
    int32_t* s_tile = s_score + (i - i0) * kTile;
    uint4 r[4];
    uint32_t ok = 0;
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const int key = key0 + 8 * m + g;
      r[m] = make_uint4(0, 0, 0, 0);
      if (seen(key)) {
        const int64_t at = row_at(key);
        if (at >= 0) {
          r[m] = __ldcs(reinterpret_cast<const uint4*>(a.k_cache + at) + t);
          ok |= 1u << m;
        } else bad = true;
      }
    }
#pragma unroll
    for (int m = 0; m < 2; ++m) {
      int32_t c[4] = {0, 0, 0, 0};
      mma_s8(c, r[2 * m].x, r[2 * m + 1].x, r[2 * m].y, r[2 * m + 1].y, q.x, q.y);
      mma_s8(c, r[2 * m].z, r[2 * m + 1].z, r[2 * m].w, r[2 * m + 1].w, q.z, q.w);
#pragma unroll
      for (int h = 0; h < 2; ++h) {                           // keys 16 m + g and 16 m + 8 + g
        const int place = score_place(16 * m + 8 * h + g);
        const bool there = (ok >> (2 * m + h)) & 1;
        const int32_t v0 = there ? c[2 * h] : kNone, v1 = there ? c[2 * h + 1] : kNone;
        mx0 = max(mx0, v0);
        mx1 = max(mx1, v1);
        if (2 * t < G) s_tile[2 * t * a.score_pitch + place] = v0;
        if (2 * t + 1 < G) s_tile[(2 * t + 1) * a.score_pitch + place] = v1;
      }
    }
  }
#pragma unroll
  for (int d = 4; d < 32; d <<= 1) {
    mx0 = max(mx0, __shfl_xor_sync(0xffffffffu, mx0, d));
    mx1 = max(mx1, __shfl_xor_sync(0xffffffffu, mx1, d));
  }
  if (g == 0) {
    s_warp_max[warp][2 * t] = mx0;
    s_warp_max[warp][2 * t + 1] = mx1;
  }
  __syncthreads();
  for (int i = tid; i < cl * kMaxGroup; i += kDecThreads) {   // this CTA's maxima into every CTA of the cluster
    const int h = i & (kMaxGroup - 1), to = i / kMaxGroup;
    int32_t m = s_warp_max[0][h];
    for (int w = 1; w < kDecWarps; ++w) m = max(m, s_warp_max[w][h]);
    ptx::st_cluster_s32(ptx::map_to_cta(ptx::smem_addr(&s_all_max[rank][h]), (uint32_t)to), m);
  }
  ptx::cluster_sync();
  int32_t mx = kNone;                                         // of head g
  for (int c = 0; c < cl; ++c) mx = max(mx, s_all_max[c][g]);

  // ---- weights and O = sum w v
  const LongAttnConsts& k = a.k;
  int32_t acc[4][4] = {};                                     // dims 8g + 2i (+ 1) x heads 2t, 2t + 1
  uint32_t sum = 0;                                           // W of head g over this lane's keys
  const int64_t mk = iexp_folded_addend(k.e);
  const int32_t neg_m = -(int32_t)k.e.fold_m, wk = iexp_folded_offset(k.e, mx);
  const bool folded = iexp_takes_folded(k.e);
  for (int i = i0 + warp; i < i1; i += kDecWarps) {
    const int key0 = first_key(i);
    const int32_t* s_tile = s_score + (i - i0) * kTile;
    uint32_t x[8], y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int key = key0 + 4 * j + t;
      uint2 v = make_uint2(0, 0);
      if (seen(key)) {
        const int64_t at = row_at(key);
        if (at >= 0) v = __ldcs(reinterpret_cast<const uint2*>(a.v_cache + at) + g);
      }
      x[j] = v.x;
      y[j] = v.y;
    }
    uint32_t w[2] = {0, 0};
    if (g < G) {
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const int4 s4 = *reinterpret_cast<const int4*>(s_tile + g * a.score_pitch + 16 * p + 4 * t);
        const int32_t s[4] = {s4.x, s4.y, s4.z, s4.w};
        uint32_t e[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          e[j] = folded ? iexp_folded((int32_t)((uint32_t)s[j] + (uint32_t)wk) >> k.e.s_in, mk, neg_m, k.e.q_ln2, k.e.q_c)
                        : iexp_dist_wide((uint32_t)mx - (uint32_t)s[j], k.e);
          e[j] = s[j] == kNone ? 0u : e[j] * k.b_w + (1u << 23);
        }
        w[p] = __byte_perm(__byte_perm(e[0], e[1], 0x0073), __byte_perm(e[2], e[3], 0x0073), 0x5410);
        sum = __dp4a(w[p], 0x01010101u, sum);
      }
    }
    uint32_t xt[8], yt[8];
    transpose4(x, xt);
    transpose4(x + 4, xt + 4);
    transpose4(y, yt);
    transpose4(y + 4, yt + 4);
    mma_s8u8(acc[0], xt[0], xt[1], xt[4], xt[5], w[0], w[1]);
    mma_s8u8(acc[1], xt[2], xt[3], xt[6], xt[7], w[0], w[1]);
    mma_s8u8(acc[2], yt[0], yt[1], yt[4], yt[5], w[0], w[1]);
    mma_s8u8(acc[3], yt[2], yt[3], yt[6], yt[7], w[0], w[1]);
  }
  sum += __shfl_xor_sync(0xffffffffu, sum, 1);
  sum += __shfl_xor_sync(0xffffffffu, sum, 2);
  if (t == 0 && g < G) atomicAdd(&s_sum[g], (int32_t)sum);
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int h = 2 * t + (c & 1);
      if (h < G) atomicAdd(&s_out[h][8 * g + 2 * i + (c >> 1)], acc[i][c]);
    }
  ptx::cluster_sync();

  // ---- every CTA joins and divides its part of the G x 64 results
  for (int i = (int)rank * kDecThreads + tid; i < G * kHeadDim; i += cl * kDecThreads) {
    const int h = i / kHeadDim, d = i % kHeadDim;
    int32_t o = 0;
    uint32_t total = 0;
    for (int c = 0; c < cl; ++c) {
      o += ptx::ld_cluster_s32(ptx::map_to_cta(ptx::smem_addr(&s_out[h][d]), (uint32_t)c));
      total += (uint32_t)ptx::ld_cluster_s32(ptx::map_to_cta(ptx::smem_addr(&s_sum[h]), (uint32_t)c));
    }
    a.out[((int64_t)batch * a.heads + head0 + h) * kHeadDim + d] = (int8_t)weighted_mean(o, row_share(total, k));
  }
  if (bad) atomicCAS(a.status, 0, IBERT_ERR_VALUE_RANGE);
  ptx::cluster_sync();                   // nobody leaves while a peer may still read its shared memory
}

}  // namespace

int launch_attention_decode(ibert_ctx* ctx, const int8_t* q, const int8_t* k_cache, const int8_t* v_cache,
                            const int32_t* tables, const int32_t* lens, int B, int max_pages, int n_pages, int log_page,
                            int max_len, int heads, int kv_heads, int window, int sinks, const LongAttnConsts& k,
                            int8_t* out) {
  DecodeArgs a{};
  a.q = q; a.k_cache = k_cache; a.v_cache = v_cache; a.tables = tables; a.lens = lens; a.out = out; a.status = ctx->d_status;
  a.heads = heads; a.kv_heads = kv_heads; a.group = heads / kv_heads;
  a.tiles_of_group = (a.group + kMaxGroup - 1) / kMaxGroup;
  a.log_page = log_page; a.max_pages = max_pages; a.n_pages = n_pages; a.max_len = max_len; a.window = window; a.sinks = sinks;
  a.k = k;
  const int64_t items = (int64_t)B * kv_heads * a.tiles_of_group;
  // tiles of 32 keys that a sequence can have: one more where the window starts inside a tile, and the sinks' own
  int64_t tiles = ((int64_t)max_len + kTile - 1) / kTile;
  if (window > 0) tiles = std::min<int64_t>(tiles, ((int64_t)window + kTile - 1) / kTile + 1 + ((int64_t)sinks + kTile - 1) / kTile);
  int cl = 1;
  while (cl < 16 && items * cl < 2 * ctx->num_sms && (tiles + cl - 1) / cl > kDecWarps) cl <<= 1;
  const int rows = std::min(a.group, kMaxGroup);
  auto smem_of = [&](int c) { return (int64_t)rows * ((tiles + c - 1) / c * kTile + 16) * 4; };
  while (cl < 16 && smem_of(cl) > 96 * 1024) cl <<= 1;
  const int64_t smem = smem_of(cl);
  if (smem > 200 * 1024 || items * cl > INT32_MAX) return IBERT_ERR_SHAPE;
  a.score_pitch = (int32_t)((tiles + cl - 1) / cl * kTile + 16);
  if (cudaFuncSetAttribute(attention_decode_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024) != cudaSuccess ||
      cudaFuncSetAttribute(attention_decode_kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) {
    cudaGetLastError();
    return IBERT_ERR_CUDA;
  }
  return launch_pdl(attention_decode_kernel, dim3((unsigned)(items * cl)), dim3(kDecThreads), (size_t)smem, ctx->stream, cl, a);
}

}  // namespace ibert
