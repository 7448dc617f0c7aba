// Bookkeeping of a paged key-value cache on the GPU: from the lengths of the requests and what each of them gets in
// this step, the pages that are taken from and given back to the pool, the block tables, and for every new token its
// position and its place ("slot") in the cache.  No counterpart in the paper.
//
// Everything is a prefix sum over the requests followed by independent look-ups: the k-th page taken in the step is
// entry n - 1 - k of the stack of free pages, the i-th token belongs to the request whose range of the running token
// count holds i.  A token's page is therefore known without waiting for whoever writes it into the block table, and one
// launch does it all.  Bound by latency (a few hundred requests, some 10 KB): three dependent rounds of loads and the
// scans.
#include <algorithm>

#include "device_utils.cuh"
#include "sm100_ptx.cuh"

namespace ibert {
namespace {

constexpr int kSlotThreads = 1024;

struct SlotArgs {
  const int32_t *lens, *fresh;      // [B] tokens held, tokens to come (negative: the request has ended)
  int32_t* tables;                  // [B][max_pages]
  int32_t* stack;                   // free pages, `*n_free` of them
  const int32_t* n_free;
  int32_t B, log_page, max_pages, in_place;
  int64_t capacity, max_tokens;
  int32_t *lens_out, *n_free_out, *cu, *slots, *positions;
  int32_t* status;
};

// inclusive scan of one 64-bit value per thread over the block; `s_warp` holds 32 words
template <typename Op>
__device__ __forceinline__ int64_t block_scan(int64_t v, int64_t* s_warp, Op op) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t u = __shfl_up_sync(0xffffffffu, v, d);
    if (lane >= d) v = op(v, u);
  }
  __syncthreads();                  // the words of an earlier scan have been read
  if (lane == 31) s_warp[warp] = v;
  __syncthreads();
  if (warp == 0) {
    int64_t w = lane < kSlotThreads / 32 ? s_warp[lane] : 0;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const int64_t u = __shfl_up_sync(0xffffffffu, w, d);
      if (lane >= d) w = op(w, u);
    }
    s_warp[lane] = w;
  }
  __syncthreads();
  return warp ? op(v, s_warp[warp - 1]) : v;
}

// the request whose range [p[b], p[b + 1]) holds i, for 0 <= i < p[B]
__device__ __forceinline__ int owner(const int32_t* p, int B, int32_t i) {
  int lo = 0, hi = B;               // p[lo] <= i < p[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (p[mid] <= i) lo = mid; else hi = mid;
  }
  return lo;
}

__global__ void __launch_bounds__(kSlotThreads, 1)
kv_slots_kernel(const SlotArgs a) {
  extern __shared__ int32_t s_req[];
  __shared__ int64_t s_warp[32];
  const int B = a.B, tid = threadIdx.x;
  int32_t* s_tok = s_req;                  // [B + 1] first new token of a request
  int32_t* s_need = s_tok + B + 1;         // [B + 1] pages taken by the requests in front
  int32_t* s_give = s_need + B + 1;        // [B + 1] pages given back by the requests in front
  int32_t* s_len = s_give + B + 1;         // [B] tokens held, -1 - tokens: the request has ended
  const int32_t P = 1 << a.log_page;
  const int64_t most = (int64_t)a.max_pages << a.log_page;
  bool bad = false;
  // (no early start of the next kernel: the packed attention reads row offsets ahead of its dependency wait, and those may
  // be this kernel's)
  ptx::grid_dep_wait();

  const int64_t n_in = *a.n_free;
  const int64_t n0 = n_in < 0 ? 0 : (n_in > a.capacity ? a.capacity : n_in);
  bad |= n_in != n0;
  const int per = (B + kSlotThreads - 1) / kSlotThreads, b0 = min(tid * per, B), b1 = min(b0 + per, B);
  auto pages = [&](int64_t n) { return (int32_t)((n + P - 1) >> a.log_page); };
  // ---- new tokens: running count, cut off at max_tokens
  const int64_t cap = a.max_tokens;
  auto add_capped = [cap](int64_t x, int64_t y) { return x + y < cap ? x + y : cap; };
  int64_t sum = 0;
  for (int b = b0; b < b1; ++b) {
    int32_t len = a.lens[b];              // (plain loads: what the call writes may lie in the same arrays)
    const int32_t f = ptx::ld_dep(a.fresh + b);
    if (len < 0 || len > most) { bad = true; len = len < 0 ? 0 : (int32_t)most; }
    s_len[b] = f < 0 ? -1 - len : len;
    sum += max(f, 0);
  }
  const int64_t mine = sum < cap ? sum : cap;
  int64_t tokens = block_scan(mine, s_warp, add_capped);
  const int64_t total_tokens = s_warp[31];
  int64_t before = __shfl_up_sync(0xffffffffu, tokens, 1);
  if ((tid & 31) == 0) before = tid ? s_warp[(tid >> 5) - 1] : 0;
  bad |= before + sum > cap;
  // ---- pages: taken and given back, both running counts in one word
  sum = 0;
  for (int b = b0; b < b1; ++b) {
    s_tok[b] = (int32_t)before;
    const int32_t f = max(ptx::ld_dep(a.fresh + b), 0);
    const int64_t next = add_capped(before, f);
    const int32_t held = s_len[b];
    if (held < 0) sum += (int64_t)pages(-1 - held) << 32;
    else {
      const int64_t after = held + (next - before);
      bad |= after > most;
      sum += pages(after < most ? after : most) - pages(held);
    }
    before = next;
  }
  const int64_t run = block_scan(sum, s_warp, [](int64_t x, int64_t y) { return x + y; });
  const int32_t total_need = (int32_t)s_warp[31], total_give = (int32_t)(s_warp[31] >> 32);
  int64_t at = run - sum;
  for (int b = b0; b < b1; ++b) {
    s_need[b] = (int32_t)at;
    s_give[b] = (int32_t)(at >> 32);
    const int32_t held = s_len[b];
    if (held < 0) at += (int64_t)pages(-1 - held) << 32;
    else {
      const int64_t next = b + 1 < b1 ? s_tok[b + 1] : before;
      const int64_t after = held + (next - s_tok[b]);
      at += pages(after < most ? after : most) - pages(held);
    }
  }
  if (tid == 0) {
    s_tok[B] = (int32_t)total_tokens;
    s_need[B] = total_need;
    s_give[B] = total_give;
  }
  // every CTA has read the lengths and the count: they may be written in place from here on
  if (a.in_place) ptx::cluster_sync(); else __syncthreads();

  const int64_t n1 = n0 + total_give < a.capacity ? n0 + total_give : a.capacity;
  bad |= n0 + total_give > a.capacity;
  // the i-th page given back, and the k-th page taken (-1: there is none)
  auto given = [&](int32_t i) {
    const int b = owner(s_give, B, i);
    return a.tables[(int64_t)b * a.max_pages + (i - s_give[b])];
  };
  auto taken = [&](int32_t k) {
    const int64_t p = n1 - 1 - k;
    return p < 0 ? -1 : (p < n0 ? a.stack[p] : given((int32_t)(p - n0)));
  };
  // ---- everything that is written, one list of work items over all CTAs: tokens, pages given back, pages taken, requests
  const int64_t first_give = a.max_tokens, first_need = first_give + total_give, first_req = first_need + total_need;
  for (int64_t w = (int64_t)blockIdx.x * kSlotThreads + tid; w < first_req + B; w += (int64_t)gridDim.x * kSlotThreads) {
    if (w < a.max_tokens) {
      int32_t slot = -1, pos = 0;
      if (w < total_tokens) {
        const int b = owner(s_tok, B, (int32_t)w);
        const int32_t held = s_len[b], had = pages(held);
        const int64_t p = held + (w - s_tok[b]);
        const int32_t j = (int32_t)(p >> a.log_page);
        const int32_t page = p >= most ? -1
                             : j < had ? a.tables[(int64_t)b * a.max_pages + j] : taken(s_need[b] + j - had);
        const int64_t s = ((int64_t)page << a.log_page) + (p & (P - 1));
        if (page >= 0 && s <= INT32_MAX) slot = (int32_t)s; else bad = true;
        pos = p < most ? (int32_t)p : 0;
      }
      a.slots[w] = slot;
      a.positions[w] = pos;
    } else if (w < first_need) {
      const int32_t i = (int32_t)(w - first_give);
      if (n0 + i < n1) a.stack[n0 + i] = given(i);
    } else if (w < first_req) {
      const int32_t k = (int32_t)(w - first_need);
      const int b = owner(s_need, B, k);
      a.tables[(int64_t)b * a.max_pages + pages(s_len[b]) + (k - s_need[b])] = taken(k);
    } else {
      const int b = (int)(w - first_req);
      const int32_t held = s_len[b];
      int64_t after = held < 0 ? 0 : held + (int64_t)(s_tok[b + 1] - s_tok[b]);
      if (held >= 0) {               // as many tokens as have found a page
        const int64_t got = n1 - s_need[b], need = s_need[b + 1] - s_need[b];
        const int64_t room = ((int64_t)pages(held) + (got < 0 ? 0 : (got < need ? got : need))) << a.log_page;
        if (after > room) { bad = true; after = room > held ? room : held; }
      }
      a.lens_out[b] = (int32_t)after;
      a.cu[b] = s_tok[b];
    }
  }
  if (blockIdx.x == 0 && tid == 0) {
    a.cu[B] = (int32_t)total_tokens;
    a.n_free_out[0] = (int32_t)(n1 > total_need ? n1 - total_need : 0);
  }
  if (bad) atomicCAS(a.status, 0, IBERT_ERR_VALUE_RANGE);
}

}  // namespace

int launch_kv_slots(ibert_ctx* ctx, const int32_t* lens, const int32_t* new_lens, int32_t* tables, int32_t* stack,
                    const int32_t* n_free, int B, int log_page, int max_pages, int64_t capacity, int64_t max_tokens,
                    int32_t* lens_out, int32_t* n_free_out, int32_t* cu, int32_t* slots, int32_t* positions) {
  // Written in place, the lengths must have been read by all CTAs before: one cluster, eight CTAs (256 requests and a token for each, some
  // pages given back 5.4 us, 131,000 tokens 25).  Else as many as there are tokens for, four at least (5.1, by one CTA 7.2; 131,000 tokens 6.8).
  const bool in_place = lens_out == lens || n_free_out == n_free;
  const int ctas = in_place ? 8 : (int)std::min<int64_t>(ctx->num_sms, std::max<int64_t>(4, (max_tokens + B) / kSlotThreads + 1));
  SlotArgs a{lens, new_lens, tables, stack, n_free, B, log_page, max_pages, in_place, capacity, max_tokens,
             lens_out, n_free_out, cu, slots, positions, ctx->d_status};
  const size_t smem = (4 * (size_t)B + 3) * sizeof(int32_t);
  static bool set[kMaxDevices] = {false};
  bool& done = set[ctx->device % kMaxDevices];
  if (!done) {                             // (for the largest batch, not this one: other threads' launches have the same limit)
    if (cudaFuncSetAttribute(kv_slots_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             (4 * kMaxRequests + 3) * (int)sizeof(int32_t)) != cudaSuccess) {
      cudaGetLastError();
      return IBERT_ERR_CUDA;
    }
    done = true;
  }
  return launch_pdl(kv_slots_kernel, dim3(ctas), dim3(kSlotThreads), smem, ctx->stream, in_place ? ctas : 1, a);
}

}  // namespace ibert
