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

// clamp(round(x b / 2^c), +-qmax) of a 16-bit x.  k = 32 - c <= 16: x 2^k fits 32 bits and the result is one upper word.
__device__ __forceinline__ int32_t requant_16(int32_t x, int32_t b, int c, int k, int64_t half, int32_t qmax) {
  if (k <= 16) return clamp_sym(requant_upper((int32_t)((uint32_t)x << k), b), qmax);
  return requant_add(x, b, half, c, qmax);
}

// 32 / N lanes own one head vector, a lane two runs of N elements such that both elements of every rotated pair are its
// own: with rotated halves runs N j and rot/2 + N j in lane j, and the dimensions that stay in the lanes behind; interleaved
// (and without rotation) the 2 N elements from 2 N j.  N = 8 (16-byte loads of Q16, and the root and the reciprocal of a head
// on four lanes instead of eight) wherever rot is a multiple of 16.  The lanes take `per` heads of one token one after the
// other, so that position, slot, cos, sin and the gammas are loaded once for them, with the next head's elements in flight.
// The N groups of a warp take N tokens and the same heads: Q and K on one side, V on the other do different work, and mixed
// in a warp they cost half as much again.
template <typename T, bool NORM, int N>
__global__ void __launch_bounds__(kRopeThreads, 3)
qkv_rope_kernel(const __grid_constant__ RopeArgs a) {
  constexpr int kLanes = 32 / N;
  const int j = threadIdx.x & (kLanes - 1);
  const int heads_all = a.heads + 2 * a.kv_heads;
  const int64_t item = (int64_t)blockIdx.x * (kRopeThreads / 32) + (threadIdx.x >> 5);
  const uint32_t group = ((1u << kLanes) - 1u) << (threadIdx.x & (32 - kLanes));
  ptx::grid_dep_wait();
  const int64_t t_group = item / a.chunks, t = t_group * N + (threadIdx.x & 31) / kLanes;
  if (t >= a.T) return;                                      // (whole groups of lanes; shuffles stay within one)
  int chunk = (int)(item - t_group * a.chunks);
  // chunks of `per` heads of Q, then of K, then of V
  const int part = chunk < a.chunks_q ? 0 : (chunk < a.chunks_q + a.chunks_kv ? 1 : 2);
  chunk -= part == 0 ? 0 : (part == 1 ? a.chunks_q : a.chunks_q + a.chunks_kv);
  const int n_heads = part == 0 ? a.heads : a.kv_heads;
  const int h0 = chunk * a.per, h1 = min(h0 + a.per, n_heads);         // within the part
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
  if (a.k_cache && part > 0) {
    const int32_t slot = ptx::ld_dep(a.slots + t);
    if (slot >= 0 && slot < a.n_slots) {
      const int64_t page = slot >> a.log_page, row = slot & ((1 << a.log_page) - 1);
      cache_row = (part == 1 ? a.k_cache : a.v_cache) + ((((page * a.kv_heads + h0) << a.log_page) + row) * kHeadDim);
    } else if (slot != -1) bad = true;
  }
  int8_t* out_row = a.with_kv || part == 0 ? a.out + (t * (a.with_kv ? heads_all : a.heads) + head_base + h0) * kHeadDim : nullptr;
  const int64_t half_c = rounding_half(a.c[part]);
  int32_t gam[2 * N];
  if (NORM && part < 2) {
#pragma unroll
    for (int i = 0; i < 2 * N; ++i) gam[i] = a.gamma[part][i < N ? e0 + i : e1 + i - N];
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
#pragma unroll
      for (int i = 0; i < 2 * N; ++i) x[i] = requant_16(x[i], a.b[2], a.c[2], a.k[2], half_c, 127);
    } else {
      if constexpr (NORM) {
        int64_t ss = 0;
#pragma unroll
        for (int i = 0; i < 2 * N; ++i) ss += (int64_t)x[i] * x[i];
#pragma unroll
        for (int d = 1; d < kLanes; d <<= 1) ss += __shfl_xor_sync(group, ss, d);
        constexpr int s0 = sizeof(T) == 1 ? 16 : 10;
        // ISqrt(ss 2^s0) = floor(sqrt(floor(ss 2^(s0+2) / 4)))
        const uint32_t r = max(ln_root<3>((uint64_t)ss << (s0 + 2), 4u, 0x80000000u), 1u);
        const int l = bit_length(r), sh = l + 26 - s0 / 2 + a.g[part];
        const uint32_t y = r << (32 - l);                    // floor(2^(l+29) / r) = floor(2^61 / y)
        uint32_t rho = reciprocal_q31(y) >> 2;
        rho += (uint64_t(1) << 61) - (uint64_t)rho * y >= y ? 1u : 0u;
        const int64_t add = int64_t(1) << (sh - 1);
        if (sh >= 32) {                                      // the upper word, shifted on
#pragma unroll
          for (int i = 0; i < 2 * N; ++i)
            x[i] = clamp_sym(requant_upper_add(x[i] * gam[i], (int32_t)rho, add) >> (sh - 32), 32767);
        } else {
#pragma unroll
          for (int i = 0; i < 2 * N; ++i) x[i] = requant_add(x[i] * gam[i], (int32_t)rho, add, sh, 32767);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 2 * N; ++i) x[i] = requant_16(x[i], a.b[part], a.c[part], a.k[part], half_c, 32767);
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
  const int64_t warps = (a.T + tokens - 1) / tokens * a.chunks, blocks = (warps + kRopeThreads / 32 - 1) / (kRopeThreads / 32);
  if (blocks > INT32_MAX) return IBERT_ERR_SHAPE;
  return launch_pdl(wide ? qkv_rope_kernel<T, NORM, 8> : qkv_rope_kernel<T, NORM, 4>, dim3((unsigned)blocks), dim3(kRopeThreads), 0,
                    ctx->stream, 1, a);
}

}  // namespace

int launch_qkv_rope(ibert_ctx* ctx, RopeArgs a, bool x_is_i16, bool norm) {
  // heads per group of lanes: one while there are fewer heads than lanes on the GPU, up to four beyond
  const bool kv = a.with_kv || a.k_cache;
  const int64_t vectors = a.T * (a.heads + (kv ? 2 * a.kv_heads : 0));
  a.per = (int)std::min<int64_t>(4, std::max<int64_t>(1, vectors / ((int64_t)ctx->num_sms * 512)));
  a.chunks_q = (a.heads + a.per - 1) / a.per;
  a.chunks_kv = kv ? (a.kv_heads + a.per - 1) / a.per : 0;
  a.chunks = a.chunks_q + 2 * a.chunks_kv;
  for (int i = 0; i < 3; ++i) a.k[i] = 32 - a.c[i];
  a.status = ctx->d_status;
  if (x_is_i16) return norm ? launch_typed<int16_t, true>(ctx, a) : launch_typed<int16_t, false>(ctx, a);
  return norm ? launch_typed<int8_t, true>(ctx, a) : launch_typed<int8_t, false>(ctx, a);
}

}  // namespace ibert
