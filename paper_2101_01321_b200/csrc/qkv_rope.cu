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
#include "device_utils.cuh"
#include "sm100_ptx.cuh"

namespace ibert {
namespace {

constexpr int kRopeThreads = 256;

__device__ __forceinline__ int bit_length(uint32_t v) { return 32 - __clz(v); }

// four consecutive elements of a head
__device__ __forceinline__ void load4(const int16_t* p, int32_t* x) {
  const uint2 w = __ldcs(reinterpret_cast<const uint2*>(p));
  x[0] = sext_half(w.x, 0); x[1] = sext_half(w.x, 1); x[2] = sext_half(w.y, 0); x[3] = sext_half(w.y, 1);
}
__device__ __forceinline__ void load4(const int8_t* p, int32_t* x) {
  const uint32_t w = __ldcs(reinterpret_cast<const uint32_t*>(p));
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = sext_byte(w, i);
}

// Eight lanes own one head vector, a lane two groups of four elements such that both elements of every rotated pair are
// its own: with rotated halves the pairs (4j + i, rot/2 + 4j + i) in lane j and the part that stays in the lanes behind,
// interleaved (and without rotation) elements 8j .. 8j + 7.  A group of eight lanes takes `per` heads of one token one
// after the other, so cos, sin and the gammas are loaded once for them.
template <typename T, bool NORM>
__global__ void __launch_bounds__(kRopeThreads)
qkv_rope_kernel(const __grid_constant__ RopeArgs a) {
  const int lane8 = threadIdx.x & 7;
  const int heads_all = a.heads + 2 * a.kv_heads;
  const int heads_read = a.with_kv || a.k_cache ? heads_all : a.heads;
  const int chunks = (heads_read + a.per - 1) / a.per;
  const int64_t item = (int64_t)blockIdx.x * (kRopeThreads / 8) + (threadIdx.x >> 3);
  const bool live = item < a.T * chunks;                     // (whole groups of eight lanes; shuffles stay within one)
  const uint32_t group = 0xffu << (threadIdx.x & 24);
  ptx::grid_dep_launch();
  ptx::grid_dep_wait();
  if (!live) return;
  const int64_t t = item / chunks;
  const int h0 = (int)(item - t * chunks) * a.per, h1 = min(h0 + a.per, heads_read);

  const int half = a.rot >> 1;
  const bool rotates = 8 * lane8 < a.rot;                    // rot is a multiple of 8: all of a lane's elements or none
  const int e0 = !a.interleaved && rotates ? 4 * lane8 : 8 * lane8;
  const int e1 = !a.interleaved && rotates ? half + 4 * lane8 : 8 * lane8 + 4;
  bool bad = false;
  int32_t cs[4];                                             // (cos, sin) of the lane's four pairs
  if (rotates) {
    int32_t pos = ptx::ld_dep(a.positions + t);
    if (pos < 0 || pos >= a.max_pos) { bad = true; pos = 0; }
    const int4 w = ptx::ld_dep(reinterpret_cast<const int4*>(a.rope + (int64_t)pos * a.rot) + lane8);
    cs[0] = w.x; cs[1] = w.y; cs[2] = w.z; cs[3] = w.w;
  }
  int8_t* cache_row = nullptr;                               // first byte of head 0's row in the K cache
  int64_t v_minus_k = 0;
  if (a.k_cache) {
    const int32_t slot = ptx::ld_dep(a.slots + t);
    if (slot >= 0 && slot < a.n_slots) {
      const int64_t page = slot >> a.log_page, row = slot & ((1 << a.log_page) - 1);
      cache_row = a.k_cache + (((page * a.kv_heads) << a.log_page) + row) * kHeadDim;
      v_minus_k = a.v_cache - a.k_cache;
    } else if (slot != -1) bad = true;
  }
  const T* x_row = static_cast<const T*>(a.x) + t * (int64_t)heads_all * kHeadDim;
  int8_t* out_row = a.out + t * (int64_t)(a.with_kv ? heads_all : a.heads) * kHeadDim;

  for (int h = h0; h < h1; ++h) {
    const int part = h < a.heads ? 0 : (h < a.heads + a.kv_heads ? 1 : 2);     // Q, K or V
    int32_t x[8];
    load4(x_row + h * kHeadDim + e0, x);
    load4(x_row + h * kHeadDim + e1, x + 4);
    uint32_t w0, w1;
    if (part == 2) {
      int32_t y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = requant_add(x[i], a.b[2], rounding_half(a.c[2]), a.c[2], 127);
      w0 = pack4_sat_s8(y[0], y[1], y[2], y[3]);
      w1 = pack4_sat_s8(y[4], y[5], y[6], y[7]);
    } else {
      int32_t u[8];
      if constexpr (NORM) {
        int64_t ss = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) ss += (int64_t)x[i] * x[i];
        ss += __shfl_xor_sync(group, ss, 1);
        ss += __shfl_xor_sync(group, ss, 2);
        ss += __shfl_xor_sync(group, ss, 4);
        constexpr int s0 = sizeof(T) == 1 ? 16 : 10;
        // ISqrt(ss 2^s0) = floor(sqrt(floor(ss 2^(s0+2) / 4)))
        const uint32_t r = max(ln_root<3>((uint64_t)ss << (s0 + 2), 4u, 0x80000000u), 1u);
        const int l = bit_length(r), sh = l + 26 - s0 / 2 + a.g[part];
        const uint32_t y = r << (32 - l);                    // floor(2^(l+29) / r) = floor(2^61 / y)
        uint32_t rho = reciprocal_q31(y) >> 2;
        rho += (uint64_t(1) << 61) - (uint64_t)rho * y >= y ? 1u : 0u;
        const int64_t add = int64_t(1) << (sh - 1);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int e = i < 4 ? e0 + i : e1 + i - 4;
          u[i] = requant_add(x[i] * a.gamma[part][e], (int32_t)rho, add, sh, 32767);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = requant_add(x[i], a.b[part], rounding_half(a.c[part]), a.c[part], 32767);
      }
      int32_t y[8];
      if (rotates) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int32_t c = sext_half(cs[i], 0), s = sext_half(cs[i], 1);
          const int32_t ua = a.interleaved ? u[2 * i] : u[i], ub = a.interleaved ? u[2 * i + 1] : u[i + 4];
          const int32_t ya = ua * c - ub * s, yb = ua * s + ub * c;
          if (a.interleaved) { y[2 * i] = ya; y[2 * i + 1] = yb; } else { y[i] = ya; y[i + 4] = yb; }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = (y[i] + (1 << 20)) >> 21;
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = (u[i] + 64) >> 7;
      }
      w0 = pack4_sat_s8(max(y[0], -127), max(y[1], -127), max(y[2], -127), max(y[3], -127));
      w1 = pack4_sat_s8(max(y[4], -127), max(y[5], -127), max(y[6], -127), max(y[7], -127));
    }
    if (a.with_kv || part == 0) {
      *reinterpret_cast<uint32_t*>(out_row + h * kHeadDim + e0) = w0;
      *reinterpret_cast<uint32_t*>(out_row + h * kHeadDim + e1) = w1;
    }
    if (part != 0 && cache_row) {
      int8_t* row = cache_row + (part == 2 ? v_minus_k : 0) +
                    ((int64_t)(h - a.heads - (part == 2 ? a.kv_heads : 0)) << a.log_page) * kHeadDim;
      *reinterpret_cast<uint32_t*>(row + e0) = w0;
      *reinterpret_cast<uint32_t*>(row + e1) = w1;
    }
  }
  if (bad) atomicCAS(a.status, 0, IBERT_ERR_VALUE_RANGE);
}

}  // namespace

int launch_qkv_rope(ibert_ctx* ctx, RopeArgs a, bool x_is_i16, bool norm) {
  const int heads_read = a.with_kv || a.k_cache ? a.heads + 2 * a.kv_heads : a.heads;
  a.per = 1;
  a.status = ctx->d_status;
  const int64_t items = a.T * ((heads_read + a.per - 1) / a.per);
  const int64_t blocks = (items + kRopeThreads / 8 - 1) / (kRopeThreads / 8);
  if (blocks > INT32_MAX) return IBERT_ERR_SHAPE;
  const dim3 grid((unsigned)blocks), block(kRopeThreads);
  if (x_is_i16)
    return norm ? launch_pdl(qkv_rope_kernel<int16_t, true>, grid, block, 0, ctx->stream, 1, a)
                : launch_pdl(qkv_rope_kernel<int16_t, false>, grid, block, 0, ctx->stream, 1, a);
  return norm ? launch_pdl(qkv_rope_kernel<int8_t, true>, grid, block, 0, ctx->stream, 1, a)
              : launch_pdl(qkv_rope_kernel<int8_t, false>, grid, block, 0, ctx->stream, 1, a);
}

}  // namespace ibert
