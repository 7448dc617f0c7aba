// Q | K | V of new tokens made ready for attention in one pass: norm of every query and key head, rotary positions,
// int8, and K and V written to their places in a paged cache.  Integers throughout, in the paper's (q, S) convention.
//
// Per head vector x[0..63] (the linear layer's int8 or Q16 values):
//   ss = sum x^2,  r = ISqrt(ss 2^s0)  (Algorithm 4; 2^(s0/2) sqrt(ss) keeps the root's own rounding below 2^-8),
//   rho = floor(2^(l+29) / r) with l the bit length of r,
//   u_i = clamp((x_i b_i rho + 2^(sh-1)) >> sh, +-32767),  sh = l + 26 - s0/2 + g,  b_i = round(gamma_i 128 / S_out 2^g)
// is gamma_i x_i / rms(x) at scale S_out / 128: Q16, seven bits finer than the result.  Without a norm
// u_i = requant(x_i; dyadic(128 S_in / S_out), 32767).  With cos and sin in units of 2^-14 the rotated pair
//   y_a = u_a c - u_b s,  y_b = u_a s + u_b c   (below 2^31)   leaves as  clamp((y + 2^20) >> 21, +-127).
// The 16-bit u is the one rounding in front of the last: it costs at most 2^-7 of the result's step.
#include <algorithm>

#include "device_utils.cuh"
#include "sm100_ptx.cuh"

namespace ibert {
namespace {

constexpr int kRopeThreads = 256;

__device__ __forceinline__ int bit_length(uint32_t v) { return 32 - __clz(v); }

// N consecutive elements of a head: the words they are in, and the values
template <int N, typename T>
__device__ __forceinline__ void load_run(const T* p, uint32_t (&w)[N * sizeof(T) / 4]) {
  if constexpr (N * sizeof(T) == 16) {
    const uint4 t = __ldcs(reinterpret_cast<const uint4*>(p));
    w[0] = t.x; w[1] = t.y; w[2] = t.z; w[3] = t.w;
  } else if constexpr (N * sizeof(T) == 8) {
    const uint2 t = __ldcs(reinterpret_cast<const uint2*>(p));
    w[0] = t.x; w[1] = t.y;
  } else {
    w[0] = __ldcs(reinterpret_cast<const uint32_t*>(p));
  }
}
template <int N, typename T>
__device__ __forceinline__ void unpack_run(const uint32_t (&w)[N * sizeof(T) / 4], int32_t* x) {
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = sizeof(T) == 2 ? sext_half(w[i / 2], i & 1) : sext_byte(w[i / 4], i & 3);
}
template <int N>
__device__ __forceinline__ void store_run(int8_t* p, const uint32_t* w) {
  if constexpr (N == 8) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
  else *reinterpret_cast<uint32_t*>(p) = w[0];
}

// (v b + 2^(sh-1)) >> sh for sh >= 33: the rounding constant is a whole number of upper words, so one multiply-high with an
// addend leaves nothing to be carried
__device__ __forceinline__ int32_t requant_high(int32_t v, int32_t b, int32_t add, int shift) {   // 2^(sh-33), sh - 32
  int32_t d;
  asm("mad.hi.s32 %0, %1, %2, %3;" : "=r"(d) : "r"(v), "r"(b), "r"(add));
  return d >> shift;
}
// clamp(round(x b / 2^c), +-qmax) of 16-bit values: x 2^16 fits 32 bits
template <int N>
__device__ __forceinline__ void requant_16(int32_t* x, int32_t b, int c, int32_t qmax) {
  if (c >= 17) {
    const int32_t add = 1 << (c - 17);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = clamp_sym(requant_high((int32_t)((uint32_t)x[i] << 16), b, add, c - 16), qmax);
  } else {
    const int64_t half = rounding_half(c);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = requant_add(x[i], b, half, c, qmax);
  }
}

// 32 / N lanes own one head vector, a lane two runs of N elements such that both elements of every rotated pair are its
// own: with rotated halves runs N j and rot/2 + N j in lane j, and the dimensions that stay in the lanes behind; interleaved
// (and without rotation) the 2 N elements from 2 N j.  N = 8 (16-byte loads of Q16, and the root and the reciprocal of a head
// on four lanes instead of eight) wherever rot is a multiple of 16.  The lanes take several heads of one token one after the
// other, so that position, slot, cos, sin and the gammas are loaded once for them, with the next head's elements in flight.
// The N groups of a warp take N tokens and the same heads: Q and K on one side, V on the other do different work, and mixed
// in a warp they cost half as much again.
// Bound by latencies at the 24 warps per SM that 80 registers allow: 32768 tokens of 3 x 16 heads, Q16 in, K and V cached as well 104 us
// (3.6 TB/s); issue slots 61 % busy, the ALU pipe 57 %, HBM 35 %.  4099 tokens, int8 without norm: 7.3 us, 390 CTAs of four heads in a row
// where 444 fit.
template <typename T, bool NORM, int N>
__global__ void __launch_bounds__(kRopeThreads, 3)
qkv_rope_kernel(const __grid_constant__ RopeArgs a) {
  constexpr int kLanes = 32 / N;
  const int j = threadIdx.x & (kLanes - 1);
  const int heads_all = a.heads + 2 * a.kv_heads;
  const int block_group = (int)blockIdx.x / a.chunks;       // (the parts of a token next to each other)
  const int64_t t_group = (int64_t)block_group * (kRopeThreads / 32) + (threadIdx.x >> 5);
  ptx::grid_dep_wait();
  const int64_t t_own = t_group * N + (threadIdx.x & 31) / kLanes;
  if (t_group * N >= a.T) return;                            // (whole warps)
  const bool live = t_own < a.T;                             // (the others repeat the last token and store nothing)
  const int64_t t = live ? t_own : a.T - 1;
  int chunk = (int)blockIdx.x - block_group * a.chunks;
  // chunks of heads of Q, then of K, then of V
  const int part = chunk < a.chunks_q ? 0 : (chunk < a.chunks_q + a.chunks_kv ? 1 : 2);
  chunk -= part == 0 ? 0 : (part == 1 ? a.chunks_q : a.chunks_q + a.chunks_kv);
  const int n_heads = part == 0 ? a.heads : a.kv_heads;
  const int per = part == 0 ? a.per_q : a.per_kv, h0 = chunk * per, h1 = min(h0 + per, n_heads);         // within the part
  const int head_base = part == 0 ? 0 : (part == 1 ? a.heads : a.heads + a.kv_heads);

  const int half = a.rot >> 1;
  const bool rotates = part < 2 && 2 * N * j < a.rot;        // (rot is a multiple of 2 N: all of a lane's elements or none)
  const bool halves = !a.interleaved && rotates;
  const int e0 = halves ? N * j : 2 * N * j, e1 = halves ? half + N * j : 2 * N * j + N;
  const T* x_row = static_cast<const T*>(a.x) + (t * heads_all + head_base + h0) * kHeadDim;
  constexpr int kWords = N * sizeof(T) / 4;
  uint32_t w0[kWords], w1[kWords];
  load_run<N>(x_row + e0, w0);
  load_run<N>(x_row + e1, w1);
  bool bad = false;
  int32_t cosine[N], sine[N];                                // of the lane's N pairs
  if (rotates) {
    int32_t pos = ptx::ld_dep(a.positions + t);
    if (pos < 0 || pos >= a.max_pos) { bad = true; pos = 0; }
    const uint4* w = reinterpret_cast<const uint4*>(a.rope + (int64_t)pos * a.rot + 2 * N * j);
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      const uint4 v = ptx::ld_dep(w + i);
      const uint32_t cs[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        cosine[4 * i + u] = sext_half(cs[u], 0);
        sine[4 * i + u] = sext_half(cs[u], 1);
      }
    }
  }
  int8_t* cache_row = nullptr;                               // first byte of the token's row of head h0 in its cache
  if (a.k_cache && part > 0 && live) {
    const int32_t slot = ptx::ld_dep(a.slots + t);
    if (slot >= 0 && slot < a.n_slots) {
      const int64_t page = slot >> a.log_page, row = slot & ((1 << a.log_page) - 1);
      cache_row = (part == 1 ? a.k_cache : a.v_cache) + ((((page * a.kv_heads + h0) << a.log_page) + row) * kHeadDim);
    } else if (slot != -1) bad = true;
  }
  int8_t* out_row = live && (a.with_kv || part == 0) ? a.out + (t * (a.with_kv ? heads_all : a.heads) + head_base + h0) * kHeadDim : nullptr;
  int32_t gam[2 * N];
  if (NORM && part < 2) {
    uint32_t w0[N / 2], w1[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      w0[i] = reinterpret_cast<const uint32_t*>(a.gamma[part] + e0)[i];
      w1[i] = reinterpret_cast<const uint32_t*>(a.gamma[part] + e1)[i];
    }
    unpack_run<N, int16_t>(w0, gam);
    unpack_run<N, int16_t>(w1, gam + N);
  }

  for (int h = h0; h < h1; ++h) {
    int32_t x[2 * N];
    unpack_run<N, T>(w0, x);
    unpack_run<N, T>(w1, x + N);
    if (h + 1 < h1) {
      x_row += kHeadDim;
      load_run<N>(x_row + e0, w0);
      load_run<N>(x_row + e1, w1);
    }
    if (part == 2) {
      requant_16<2 * N>(x, a.b[2], a.c[2], 127);
    } else {
      if constexpr (NORM) {
        int64_t ss = 0;
#pragma unroll
        for (int i = 0; i < 2 * N; ++i) ss += (int64_t)x[i] * x[i];
#pragma unroll
        for (int d = 1; d < kLanes; d <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, d);
        constexpr int s0 = sizeof(T) == 1 ? 16 : 10;
        // ISqrt(ss 2^s0) = floor(sqrt(floor(ss 2^(s0+2) / 4)))
        const uint32_t r = max(ln_root<3>((uint64_t)ss << (s0 + 2), 4u, 0x80000000u), 1u);
        const int l = bit_length(r), sh = l + 26 - s0 / 2 + a.g[part];
        const uint32_t y = r << (32 - l);                    // floor(2^(l+29) / r) = floor(2^61 / y)
        uint32_t rho = reciprocal_q31(y) >> 2;
        rho += (uint64_t(1) << 61) - (uint64_t)rho * y >= y ? 1u : 0u;
        if (__all_sync(0xffffffffu, sh >= 33)) {
          const int32_t add = 1 << (sh - 33);
#pragma unroll
          for (int i = 0; i < 2 * N; ++i) x[i] = clamp_sym(requant_high(x[i] * gam[i], (int32_t)rho, add, sh - 32), 32767);
        } else {
          const int64_t add = int64_t(1) << (sh - 1);
#pragma unroll
          for (int i = 0; i < 2 * N; ++i) x[i] = requant_add(x[i] * gam[i], (int32_t)rho, add, sh, 32767);
        }
      } else {
        requant_16<2 * N>(x, a.b[part], a.c[part], 32767);
      }
      if (rotates) {
        if (a.interleaved) {
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const int32_t c = cosine[i], s = sine[i], ua = x[2 * i], ub = x[2 * i + 1];
            x[2 * i] = (ua * c - ub * s + (1 << 20)) >> 21;
            x[2 * i + 1] = (ua * s + ub * c + (1 << 20)) >> 21;
          }
        } else {
#pragma unroll
          for (int i = 0; i < N; ++i) {
            const int32_t c = cosine[i], s = sine[i], ua = x[i], ub = x[i + N];
            x[i] = (ua * c - ub * s + (1 << 20)) >> 21;
            x[i + N] = (ua * s + ub * c + (1 << 20)) >> 21;
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < 2 * N; ++i) x[i] = (x[i] + 64) >> 7;
      }
#pragma unroll
      for (int i = 0; i < 2 * N; ++i) x[i] = max(x[i], -127);          // (the upper end saturates below)
    }
    uint32_t w[N / 2];
#pragma unroll
    for (int i = 0; i < N / 2; ++i) w[i] = pack4_sat_s8(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
    if (out_row) {
      store_run<N>(out_row + e0, w);
      store_run<N>(out_row + e1, w + N / 4);
      out_row += kHeadDim;
    }
    if (cache_row) {
      store_run<N>(cache_row + e0, w);
      store_run<N>(cache_row + e1, w + N / 4);
      cache_row += (int64_t)kHeadDim << a.log_page;
    }
  }
  if (bad) atomicCAS(a.status, 0, IBERT_ERR_VALUE_RANGE);
}

template <typename T, bool NORM>
int launch_typed(ibert_ctx* ctx, const RopeArgs& a) {
  const bool wide = a.rot % 16 == 0;
  const int tokens = wide ? 8 : 4;                 // of a warp
  const int64_t per_block = (int64_t)tokens * (kRopeThreads / 32), blocks = (a.T + per_block - 1) / per_block * a.chunks;
  if (blocks > INT32_MAX) return IBERT_ERR_SHAPE;
  return launch_pdl(wide ? qkv_rope_kernel<T, NORM, 8> : qkv_rope_kernel<T, NORM, 4>, dim3((unsigned)blocks), dim3(kRopeThreads), 0,
                    ctx->stream, 1, a);
}

}  // namespace

int launch_qkv_rope(ibert_ctx* ctx, RopeArgs a, bool x_is_i16, bool norm) {
  // heads per group of lanes: up to eight (what is loaded once per token and part costs half a head), fewer while the groups
  // would not fill the GPU
  const bool kv = a.with_kv || a.k_cache;
  const int64_t vectors = a.T * (a.heads + (kv ? 2 * a.kv_heads : 0));
  const int per = (int)std::min<int64_t>(8, std::max<int64_t>(1, vectors / ((int64_t)ctx->num_sms * 128)));
  a.chunks_q = (a.heads + per - 1) / per;
  a.per_q = (a.heads + a.chunks_q - 1) / a.chunks_q;
  a.chunks_kv = kv ? (a.kv_heads + per - 1) / per : 0;
  a.per_kv = kv ? (a.kv_heads + a.chunks_kv - 1) / a.chunks_kv : 1;
  a.chunks = a.chunks_q + 2 * a.chunks_kv;
  a.status = ctx->d_status;
  if (x_is_i16) return norm ? launch_typed<int16_t, true>(ctx, a) : launch_typed<int16_t, false>(ctx, a);
  return norm ? launch_typed<int8_t, true>(ctx, a) : launch_typed<int8_t, false>(ctx, a);
}

}  // namespace ibert
