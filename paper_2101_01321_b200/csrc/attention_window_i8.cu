// Integer-only causal attention of packed sequences with a sliding window and first tokens that stay visible.
//
// Per (query, head), over its visible keys:  s_j = q k_j,  M = max s_j,  e_j = i-exp(M - s_j) (Algorithm 3),
//   w_j = (e_j b_w + 2^23) >> 24  (u8, p_max at the maximum),  O = sum w_j v_j,  W = sum w_j,  out = O / W at S_ctx
// -- the definition of the paged attention (attention_decode_i8.cu), so a token's context is the same whether it is
// computed here with its prompt or there alone.
//
// i-exp needs the row's maximum before the first exponential (its shifts do not commute with a later maximum), so the
// scores are computed twice: pass A takes the maximum of all score tiles, pass B recomputes them, weights them and
// multiplies with V.  The tensor pipe is idle for most of a tile's exponentials either way (16 % busy with both products and
// the second Q K^T); in exchange O is never rescaled and accumulates in tensor memory as exact integers.
//
// A CTA takes 128 consecutive ROWS of the packed tensor, whatever sequences they belong to, and one head: keys run from
// the first row's first visible key to the last row, each row with bounds of its own.  So short sequences share tiles,
// and the grid follows from the row count alone.  Four warps, a thread per query row (= TMEM lane), and one that issues
// copies and products; four CTAs per SM (128 columns of tensor memory each: 64 scores, 64 context values; pass A, which has
// no context yet, uses both halves for scores in turn) hide each other's waits.
// Bound by the instructions of the exponentials, 11.5 per 32 scores with maxima and masks.  8192 tokens, 16 heads, window 2048 + 4: 138 us,
// 2.1e12 scores a second; issue slots 70 % and the ALU pipe 66 % busy (88 and 83 us of it, multiply-adds 65), the rest are waits, instruction
// fetch and SMs that are done early.  With one barrier of the whole CTA per step, and no warp for copies and products, it was 200.
// Of prompts of unequal length the longest rows' CTAs decide: 5 of up to 1531, 560 CTAs in one wave, 50 us, SMs active for 64 % of it.
#include <cuda.h>

#include <algorithm>

#include "device_utils.cuh"
#include "sm100_ptx.cuh"

namespace ibert {
namespace {

constexpr int kKeys = 64;                          // keys per tile
constexpr int kSlot = kKeys * kHeadDim;            // 4 KB
constexpr int kKRing = 4, kVRing = 3;              // tiles in shared memory
constexpr int kP = 128 * kKeys;                    // weights of a tile: 8 KB
constexpr int kWinSmem = 128 * kHeadDim + kKRing * kSlot + kVRing * kSlot + 2 * kP + 256 + 2 * 128 * 4 + 1024;

struct WindowArgs {
  const int32_t* cu;                               // [B + 1]
  int8_t* out;                                     // [T][heads 64]
  int32_t* status;
  int32_t T, B, max_len, heads, kv_heads, window, sinks, tiles;
  int32_t int_min;                                 // INT32_MIN, as a run-time value (see add_alu)
  LongAttnConsts k;
};

// 64-bit mask of the bits [a, b) with a, b clamped to [0, 64]
__device__ __forceinline__ uint64_t bits_between(int a, int b) {
  a = min(max(a, 0), 64);
  b = min(max(b, 0), 64);
  const uint64_t below_b = b == 64 ? ~0ull : (1ull << b) - 1ull, below_a = a == 64 ? ~0ull : (1ull << a) - 1ull;
  return below_b & ~below_a;
}
// bytes of 255 where bit i of the low four is set
__device__ __forceinline__ uint32_t byte_mask(uint32_t m) { return ((m & 15u) * 0x00204081u & 0x01010101u) * 255u; }

// MODE: how i-exp is evaluated; 0: folded without a pre-shift, 1: folded with one, 2: the wide form, 3: with the quotient in 32
// bits.  On the multiply-add pipe an instruction takes two clocks per warp, four for the upper word of a product: 10.5 clocks per
// score's exponential in the folded form, 8.5 (and 7.5 on the ALU pipe) with the short quotient.
// SPLIT: threads per row, each with half of a tile's columns: while the CTAs are few, their rows' exponentials are the longest
// part of every step (4 prompts of up to 97 tokens, 12 heads, 36 CTAs: 8.6 us by one thread, 8.0 by two; 1 x 2048 x 16 heads, 256 CTAs: 40 and 37)
template <int MODE, int SPLIT>
__global__ void __launch_bounds__(128 * SPLIT + 32, SPLIT == 1 ? 4 : 2)
attention_window_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_kv,
                        const __grid_constant__ WindowArgs a) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* sQ = smem;                              // [128][64 B], 64-byte swizzle
  uint8_t* sK = sQ + 128 * kHeadDim;               // kKRing tiles [64][64 B], 64-byte swizzle
  uint8_t* sV = sK + kKRing * kSlot;                    // kVRing tiles
  uint8_t* sP = sV + kVRing * kSlot;                    // two of [128][64 B], 64-byte swizzle
  uint64_t* s_bar = reinterpret_cast<uint64_t*>(sP + 2 * kP);
  const uint32_t bar_q = ptx::smem_addr(s_bar), bar_k = bar_q + 8, bar_v = bar_k + 8 * kKRing;       // copies: Q, K and V tiles
  const uint32_t bar_s = bar_v + 8 * kVRing, bar_free = bar_s + 16;  // scores complete; scores read by the rows' warps (two buffers)
  const uint32_t bar_p = bar_free + 16, bar_pv = bar_p + 16;         // weights written (two buffers); the last product done
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(s_bar + 15);
  constexpr int kRowWarps = 4 * SPLIT;
  int32_t* s_join = reinterpret_cast<int32_t*>(s_bar + 32);    // [2][128] what the two threads of a row exchange
  int32_t* s_bounds = reinterpret_cast<int32_t*>(s_bar + 16);  // first visible key, first row of the sequence, last row's first key

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, r = tid & 127;
  const int head = (int)blockIdx.x % a.heads;
  const int q0 = (a.tiles - 1 - (int)blockIdx.x / a.heads) * 128;       // the rows with most keys first
  if (warp == 0) {
    if (ptx::elect_one()) {
      ptx::mbar_init(bar_q, 1);
      for (int i = 0; i < kKRing; ++i) ptx::mbar_init(bar_k + 8 * i, 1);
      for (int i = 0; i < kVRing; ++i) ptx::mbar_init(bar_v + 8 * i, 1);
      for (int i = 0; i < 2; ++i) {
        ptx::mbar_init(bar_s + 8 * i, 1);
        ptx::mbar_init(bar_free + 8 * i, kRowWarps);
        ptx::mbar_init(bar_p + 8 * i, kRowWarps);
      }
      ptx::mbar_init(bar_pv, 1);
      ptx::fence_mbar_init();
      ptx::tma_prefetch_desc(&map_q);
      ptx::tma_prefetch_desc(&map_kv);
    }
    __syncwarp();
    ptx::tmem_alloc(ptx::smem_addr(s_tmem), 128);
    ptx::tmem_relinquish();
  }
  ptx::grid_dep_wait();

  // ---- this row's sequence: the last b with cu[b] <= row, searched 32-fold for the warp's first row, on from there
  const int row = min(q0 + r, a.T - 1);
  int lo_b = 0, hi_b = a.B;
  const int row_w = min(q0 + (warp & 3) * 32, a.T - 1);     // (the last warp repeats the first one's)
  while (hi_b - lo_b > 1) {
    const int step = (hi_b - lo_b + 31) / 32, i = lo_b + lane * step;
    const uint32_t le = __ballot_sync(0xffffffffu, i < hi_b && (lane == 0 || ptx::ld_dep(a.cu + i) <= row_w));
    const int n = __popc(le & ~(le + 1)) ;                   // leading run of ones from lane 0
    lo_b += (n - 1) * step;
    hi_b = min(lo_b + step, hi_b);
  }
  for (int step = 1; lo_b + 1 < a.B && ptx::ld_dep(a.cu + lo_b + 1) <= row;) {           // (other rows of the warp: gallop)
    if (lo_b + step < a.B && ptx::ld_dep(a.cu + lo_b + step) <= row) { lo_b += step; step <<= 1; }
    else step = max(step >> 1, 1);
  }
  const int c0 = ptx::ld_dep(a.cu + lo_b), c1 = ptx::ld_dep(a.cu + lo_b + 1);
  const bool real = q0 + r < a.T && row >= c0 && row < c1;
  const int first = real ? max(c0, 0) : row;                 // of the sequence; a row of none sees itself and is not stored
  const int low = max(first, row - (a.window > 0 ? min(a.window, a.max_len) : a.max_len) + 1);
  const bool bad = real && tid < 128 && (c1 - c0 > a.max_len || c1 > a.T);
  if (tid == 0) { s_bounds[0] = low; s_bounds[1] = first; }
  if (tid == 127) s_bounds[2] = low;       // (of the tile's last row)
  ptx::tc_fence_before_sync();
  const bool any = __syncthreads_or(real);
  ptx::tc_fence_after_sync();
  const uint32_t tmem = *s_tmem, t_row = tmem + ((uint32_t)((warp & 3) * 32) << 16);
  const int key_w = s_bounds[0], seq0 = s_bounds[1], low_last = s_bounds[2];

  // ---- tiles of 64 keys: `lead` over the sinks of the first row's sequence, then from the first row's window on
  const int sink_end = a.window > 0 ? (int)min((int64_t)seq0 + a.sinks, (int64_t)key_w) : seq0;
  const int lead = any ? (sink_end - seq0 + kKeys - 1) / kKeys : 0;
  const int nt = any ? lead + (min(q0 + 128, a.T) - key_w + kKeys - 1) / kKeys : 0;
  auto base_of = [&](int i) { return i < lead ? seq0 + i * kKeys : key_w + (i - lead) * kKeys; };
  auto mask_of = [&](int i) {
    const int j0 = base_of(i);
    const int sinks_end = (int)min((int64_t)first + a.sinks, (int64_t)row + 1);
    if (i < lead) return bits_between(first - j0, min(sinks_end, key_w) - j0);
    uint64_t m = bits_between(low - j0, row + 1 - j0);
    if (a.window > 0) m |= bits_between(first - j0, sinks_end - j0);
    return m;
  };
  // tiles whose keys every row sees: [whole0, whole1)
  const int whole0 = lead + (low_last - key_w + kKeys - 1) / kKeys, whole1 = lead + (q0 + 1 >= key_w + kKeys ? (q0 + 1 - key_w) / kKeys : 0);
  auto whole = [&](int i) { return i >= whole0 && i < whole1; };

  const int kvh = head / (a.heads / a.kv_heads);
  const int col_k = (a.heads + kvh) * kHeadDim, col_v = col_k + a.kv_heads * kHeadDim;
  auto load_k = [&](int s) {                       // tile s of pass A, then of pass B
    const uint32_t bar = bar_k + 8 * (s % kKRing);
    ptx::mbar_arrive_expect_tx(bar, kSlot);
    ptx::tma_load_2d(ptx::smem_addr(sK) + (s % kKRing) * kSlot, &map_kv, bar, col_k, base_of(s < nt ? s : s - nt));
  };
  auto load_v = [&](int i) {
    const int at = i % kVRing;
    ptx::mbar_arrive_expect_tx(bar_v + 8 * at, kSlot);
    ptx::tma_load_2d(ptx::smem_addr(sV) + at * kSlot, &map_kv, bar_v + 8 * at, col_v, base_of(i));
  };
  auto wait = [](uint32_t bar, int use) {          // for the use-th completion of a barrier, by a whole warp
    return __all_sync(0xffffffffu, ptx::mbar_wait(bar, (uint32_t)use & 1u)) != 0;
  };
  const uint64_t dq = ptx::make_kmajor_desc(ptx::smem_addr(sQ), 512, ptx::kSwizzle64);
  const uint64_t dk0 = ptx::make_kmajor_desc(ptx::smem_addr(sK), 512, ptx::kSwizzle64);
  auto score_mma = [&](int s, int buffer) {        // S = Q K^T of tile s of the passes: 64 dimensions are two K steps
    const uint32_t idesc = ptx::make_idesc_i8(128, kKeys, true, true);
    const uint64_t dk = dk0 + (uint64_t)(s % kKRing) * (kSlot >> 4);
    ptx::mma_i8_ss(tmem + buffer * kKeys, dq, dk, idesc, 0u);
    ptx::mma_i8_ss(tmem + buffer * kKeys, dq + 2, dk + 2, idesc, 1u);
    ptx::mma_commit(bar_s + 8 * buffer);
  };
  // pass A: tile i in buffer i & 1; pass B: every tile in buffer 0, which pass A has used n0 times (buffer 1 holds the context)
  const int n0 = (nt + 1) / 2;

  bool ok = true;
  if (nt > 0 && warp == kRowWarps) {
    // ---- copies and matrix products, all by one thread.  A tile's scores may be issued when the rows have read what was in
    // its buffer; those read are complete, as are all before them, and their K tiles may be replaced.
    // Products complete in the order of their issue, and their barrier counts all that were issued before: scores that have
    // been read say that the product of weights issued before them has read its weights and values, too.  (The values need
    // three tiles, the weights two, for that; waits of their own for either cost this thread more than a step takes.)
    if (ptx::elect_one()) {
      int k_loads = min(kKRing, 2 * nt), v_loads = min(kVRing, nt);
      ptx::mbar_arrive_expect_tx(bar_q, 128 * kHeadDim);
      ptx::tma_load_2d(ptx::smem_addr(sQ), &map_q, bar_q, head * kHeadDim, q0);
      for (int s = 0; s < k_loads; ++s) load_k(s);
      for (int i = 0; i < v_loads; ++i) load_v(i);
      ok = ptx::mbar_wait(bar_q, 0);
      for (int i = 0; i < nt && ok; ++i) {
        if (i > 1) {
          if (!(ok = ptx::mbar_wait(bar_free + 8 * (i & 1), ((i >> 1) - 1) & 1))) break;
          if (k_loads < 2 * nt) load_k(k_loads++);           // tile i + 2 in the place of tile i - 2
        }
        if (!(ok = ptx::mbar_wait(bar_k + 8 * (i % kKRing), (i / kKRing) & 1))) break;
        ptx::tc_fence_after_sync();
        score_mma(i, i & 1);
      }
      const uint32_t idesc = ptx::make_idesc_i8(128, kHeadDim, false, true) | (1u << 16);        // u8 x s8, V MN-major
      const uint64_t dp = ptx::make_kmajor_desc(ptx::smem_addr(sP), 512, ptx::kSwizzle64);
      const uint64_t dv = (uint64_t)((ptx::smem_addr(sV) & 0x3FFFFu) >> 4) | ((uint64_t)(512 >> 4) << 16) |
                          ((uint64_t)(512 >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)ptx::kSwizzle64 << 61);
      int v_at = 0, v_phase = 0;                   // of tile i - 1
      for (int i = 0; i <= nt && ok; ++i) {
        if (i < nt) {                              // scores of tile i
          const int s = nt + i;
          if (!(ok = ptx::mbar_wait(bar_free, (n0 + i - 1) & 1) && ptx::mbar_wait(bar_k + 8 * (s % kKRing), (s / kKRing) & 1))) break;
          ptx::tc_fence_after_sync();
          score_mma(s, 0);
          // (the scores that buffer 0 held were those of tile s - 1, at the start of the pass s - 2 if not s - 1)
          for (const int to = min(s + (i > 0 ? 3 : 2), 2 * nt - 1); k_loads <= to;) load_k(k_loads++);
          if (i >= kVRing) { load_v(i); ++v_loads; }
        }
        if (i == 0) continue;
        const int p = i - 1;                       // O += P V of tile i - 1
        if (!(ok = ptx::mbar_wait(bar_p + 8 * (p & 1), (p >> 1) & 1) && ptx::mbar_wait(bar_v + 8 * v_at, v_phase))) break;
        ptx::tc_fence_after_sync();
        const uint64_t dpi = dp + (uint64_t)(p & 1) * (kP >> 4), dvi = dv + (uint64_t)v_at * (kSlot >> 4);
        ptx::mma_i8_ss(tmem + kKeys, dpi, dvi, idesc, p > 0 ? 1u : 0u);
        ptx::mma_i8_ss(tmem + kKeys, dpi + 2, dvi + ((32 * kHeadDim) >> 4), idesc, 1u);
        if (p == nt - 1) ptx::mma_commit(bar_pv);
        if (++v_at == kVRing) { v_at = 0; v_phase ^= 1; }
      }
      if (!ok) {                                   // copies still in flight land before the shared memory is given up
        for (int s = max(k_loads - kKRing, 0); s < k_loads; ++s) ptx::mbar_wait(bar_k + 8 * (s % kKRing), (s / kKRing) & 1);
        for (int i = max(v_loads - kVRing, 0); i < v_loads; ++i) ptx::mbar_wait(bar_v + 8 * (i % kVRing), (i / kVRing) & 1);
        ptx::mbar_wait(bar_q, 0);
      }
    }
    ok = __all_sync(0xffffffffu, ok);
  } else if (nt > 0) {
    // ---- pass A: row maxima
    const int half = warp >> 2;
    int32_t mx = INT32_MIN;
    auto join = [&](int32_t v, auto op) {          // of a row's two threads
      if constexpr (SPLIT == 1) return v;
      s_join[tid] = v;
      ptx::named_bar_sync(1, 32 * kRowWarps);
      v = op(s_join[r], s_join[128 + r]);
      ptx::named_bar_sync(1, 32 * kRowWarps);
      return v;
    };
    auto arrive = [&](uint32_t bar) {              // of this warp, after what its lanes did with tensor or shared memory
      ptx::tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(bar);
    };
    for (int i = 0; i < nt; ++i) {
      ok = wait(bar_s + 8 * (i & 1), i >> 1);
      if (!ok) break;
      ptx::tc_fence_after_sync();
      constexpr int kCols = kKeys / SPLIT;
      const int first_col = SPLIT == 1 ? 0 : half * kCols;
      uint32_t v[kCols];
      if constexpr (SPLIT == 1) ptx::tmem_ld64(t_row + (i & 1) * kKeys, v);
      else ptx::tmem_ld32(t_row + (i & 1) * kKeys + first_col, v);
      ptx::tmem_wait_ld();
      arrive(bar_free + 8 * (i & 1));
      if (!whole(i)) {
        const uint64_t m = mask_of(i) >> first_col;
        const uint32_t m0 = (uint32_t)m, m1 = (uint32_t)(m >> 32);
#pragma unroll
        for (int j = 0; j < kCols; ++j)
          if (!(((j < 32 ? m0 : m1) >> (j & 31)) & 1u)) v[j] = (uint32_t)INT32_MIN;
      }
#pragma unroll
      for (int j = 0; j < kCols; j += 2) mx = __vimax3_s32(mx, (int32_t)v[j], (int32_t)v[j + 1]);
    }
    mx = join(mx, [](int32_t x, int32_t y) { return max(x, y); });

    // ---- pass B: weights, O = sum w v
    const LongAttnConsts& k = a.k;
    const ExpConsts& ek = k.e;
    const int64_t mk = iexp_folded_addend(ek);
    const int32_t neg_m = -(int32_t)ek.fold_m, wk = iexp_folded_offset(ek, mx);
    // MODE 3: x = K - d with K = q_b - s_out q_ln2, d clamped to 9 q_ln2
    const int32_t short_k0 = ek.q_b - ek.s_out * (int32_t)ek.q_ln2, short_min = short_k0 - 9 * (int32_t)ek.q_ln2;
    const uint32_t short_neg = 0u - k.short_m, short_c = (uint32_t)(short_k0 + k.short_add) * k.short_m + ((uint32_t)ek.s_out << k.short_k);
    auto weight = [&](uint32_t s) {                // w in the upper byte
      uint32_t e;
      if constexpr (MODE == 3) {                   // (scores of masked keys may exceed the maximum; their weights are dropped)
        const int32_t x = __viaddmax_s32((int32_t)s, wk, short_min);
        const uint32_t n = ((uint32_t)x * short_neg + short_c) >> k.short_k;
        const int32_t t = (int32_t)(n * ek.q_ln2) + x;
        e = shr_clamped((uint32_t)(t * t + ek.q_c), n);
      } else if constexpr (MODE == 0) e = iexp_folded(add_alu((int32_t)s, wk, a.int_min), mk, neg_m, ek.q_ln2, ek.q_c);
      else if constexpr (MODE == 1) e = iexp_folded((int32_t)(s + (uint32_t)wk) >> ek.s_in, mk, neg_m, ek.q_ln2, ek.q_c);
      else e = iexp_dist_wide((uint32_t)mx - s, ek);
      return e * k.b_w + (1u << 23);
    };
    uint32_t sum = 0;
    for (int i = 0; i < nt && ok; ++i) {
      ok = wait(bar_s, n0 + i);
      if (!ok) break;
      ptx::tc_fence_after_sync();
      const uint64_t m = whole(i) ? ~0ull : mask_of(i);
      uint8_t* p_row = sP + (i & 1) * kP + r * kKeys;
#pragma unroll
      for (int u = 0; u < 2 / SPLIT; ++u) {
        const int h = SPLIT == 1 ? u : half;
        uint32_t v[32], w[8];
        ptx::tmem_ld32(t_row + 32 * h, v);
        ptx::tmem_wait_ld();
        if (u == 2 / SPLIT - 1) arrive(bar_free);
#pragma unroll
        for (int j = 0; j < 8; ++j)
          w[j] = __byte_perm(__byte_perm(weight(v[4 * j]), weight(v[4 * j + 1]), 0x0073),
                             __byte_perm(weight(v[4 * j + 2]), weight(v[4 * j + 3]), 0x0073), 0x5410);
        const uint32_t mh = (uint32_t)(m >> (32 * h));
        if (mh != 0xffffffffu) {
#pragma unroll
          for (int j = 0; j < 8; ++j) w[j] &= byte_mask(mh >> (4 * j));
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) sum = __dp4a(w[j], 0x01010101u, sum);
#pragma unroll
        for (int c = 0; c < 2; ++c)
          *reinterpret_cast<uint4*>(p_row + (((2 * h + c) ^ ((r >> 1) & 3)) << 4)) =
              make_uint4(w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]);
      }
      ptx::fence_proxy_async_smem();
      arrive(bar_p + 8 * (i & 1));
    }
    if (ok) ok = wait(bar_pv, 0);

    // ---- the weighted mean of this row
    sum = (uint32_t)join((int32_t)sum, [](int32_t x, int32_t y) { return x + y; });
    if (ok) {
      ptx::tc_fence_after_sync();
      const RowShare share = row_share(sum, k);
      int8_t* o = a.out + ((int64_t)row * a.heads + head) * kHeadDim;
#pragma unroll 1
      for (int h = SPLIT == 1 ? 0 : half; h < (SPLIT == 1 ? 2 : half + 1); ++h) {
        uint32_t v[32];
        ptx::tmem_ld32(t_row + kKeys + 32 * h, v);
        ptx::tmem_wait_ld();
        if (real) {
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
              w[j] = pack4_sat_s8(weighted_mean((int32_t)v[16 * c + 4 * j], share), weighted_mean((int32_t)v[16 * c + 4 * j + 1], share),
                                  weighted_mean((int32_t)v[16 * c + 4 * j + 2], share), weighted_mean((int32_t)v[16 * c + 4 * j + 3], share));
            reinterpret_cast<uint4*>(o + 32 * h)[c] = make_uint4(w[0], w[1], w[2], w[3]);
          }
        }
      }
    }
  }
  // (Not earlier: CTAs of the next kernel that wait for this one would take the slots that its own last CTAs are balanced by,
  // and be stacked on the SMs that happen to have one free.)
  ptx::grid_dep_launch();
  if (!ok) atomicCAS(a.status, 0, IBERT_ERR_TIMEOUT);
  if (bad) atomicCAS(a.status, 0, IBERT_ERR_VALUE_RANGE);
  ptx::tc_fence_before_sync();
  __syncthreads();
  if (warp == 0) {
    ptx::tc_fence_after_sync();
    ptx::tmem_dealloc(tmem, 128);
  }
}

}  // namespace

int launch_attention_window(ibert_ctx* ctx, const int8_t* qkv, const int32_t* cu, int B, int max_len, int64_t T, int heads,
                            int kv_heads, int window, int sinks, const LongAttnConsts& k, int8_t* out) {
  const uint64_t cols = (uint64_t)(heads + 2 * kv_heads) * kHeadDim;
  const uint64_t dims[2] = {cols, (uint64_t)T}, str[1] = {cols};
  const uint32_t box_q[2] = {kHeadDim, 128}, box_kv[2] = {kHeadDim, kKeys};
  CUtensorMap mq, mkv;
  if (int rc = encode_tensor_map(&mq, qkv, 2, dims, str, box_q, 64)) return rc;
  if (int rc = encode_tensor_map(&mkv, qkv, 2, dims, str, box_kv, 64)) return rc;
  WindowArgs a{};
  a.cu = cu; a.out = out; a.status = ctx->d_status;
  a.T = (int32_t)T; a.B = B; a.max_len = max_len; a.heads = heads; a.kv_heads = kv_heads; a.window = window;
  // (sequences of up to max_len lose nothing: where this cuts, they have at most 65536 keys and all of them are seen; longer
  // ones, which are reported, keep their sums in 32 bits)
  a.sinks = std::min(sinks, kMaxVisible - std::min({window, max_len, kMaxVisible}));
  a.tiles = (int32_t)((T + 127) / 128); a.int_min = INT32_MIN; a.k = k;
  const int64_t grid = (int64_t)a.tiles * heads;
  if (grid > INT32_MAX) return IBERT_ERR_SHAPE;
  const int mode = k.short_k ? 3 : (!iexp_takes_folded(k.e) ? 2 : (k.e.s_in == 0 ? 0 : 1));
  // As many CTAs as are resident so.  Split / not, us, for some 500 CTAs: rows of equal work 86 / 74 (8192 tokens with a window), 22 / 18 (60
  // prompts of up to 128; 100 of up to 80).  Where the work is unequal they would gain, 45 / 49 (5 prompts of up to 1531), 84 / 94 (one of
  // 4096), 59 / 66 (3 of up to 2000), but the host does not know the lengths.
  const bool split = grid <= 2 * (int64_t)ctx->num_sms;
  decltype(&attention_window_kernel<0, 1>) const kernels[2][4] = {
      {attention_window_kernel<0, 1>, attention_window_kernel<1, 1>, attention_window_kernel<2, 1>, attention_window_kernel<3, 1>},
      {attention_window_kernel<0, 2>, attention_window_kernel<1, 2>, attention_window_kernel<2, 2>, attention_window_kernel<3, 2>}};
  auto kernel = kernels[split ? 1 : 0][mode];
  static bool set[kMaxDevices][8] = {{false}};
  bool& done = set[ctx->device % kMaxDevices][mode + (split ? 4 : 0)];
  if (!done) {
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kWinSmem) != cudaSuccess) {
      cudaGetLastError();
      return IBERT_ERR_CUDA;
    }
    done = true;
  }
  return launch_pdl(kernel, dim3((unsigned)grid), dim3(split ? 288 : 160), (size_t)kWinSmem, ctx->stream, 1, mq, mkv, a);
}

}  // namespace ibert
