// Eviction from the paged cache by accumulated attention weight, for sm_100a: two kernels, neither with any arithmetic on the tokens.
//
// evict_select_kernel, one CTA per (request, kv head).  Of n > keep tokens the first `sinks` and the last `recent` stay; of the others
// the need = keep - sinks - recent with the largest 64-bit keys: the weight as the 32-bit integer that compares like it (-0 as +0, NaN
// below everything), then the slot's complement.  No two keys are equal, so what is kept is what is not below the need-th largest.
// It is found by digits of 12 bits from the top: a histogram of the candidates that agree with the digits so far, and the bin in which the
// count from above reaches what is still needed.  As soon as that bin holds few enough they are listed and ranked against one another;
// with weights that differ that is after the first digit, which is counted as the weights arrive.  Histograms are integer counts and the
// list's order decides nothing, so the order of the atomics does not show.  One read of the weights from memory: what comes after finds them
// in shared memory, or in L2 where there are more than fit.
// Bound by instructions and by barriers of 32 warps, not by memory: 8 heads of 4608 weights 8 us, 256 of 4200..9000 18 us (two CTAs to an
// SM, 74 % of issue slots).  Not kept: three digits to the end and two scans of the block (25 us; 512 or 256 threads 16 us for the 8 heads),
// copies of the histogram by lane (no gain: 60 bins hold most counts, but the conflicts are not what it waits for).
//
// evict_move_kernel, one CTA per (new page, kv head, request): the 64 tokens of the page from their slots.  A token's K codes, scales,
// V and Delta_S entries are whole 16-, 8- and 2-byte pieces in every slot, whose places depend on the slot (include/mpfa.h), so the new
// page is written once, in full, with the rest of it zeros.  Bound by memory: 32 requests x 8 heads x 4001 tokens, 0.21 GB read (0.26 from
// DRAM: 2 bytes of Delta_S and 8 of scales out of 32-byte sectors) and as much written, 75 us alone, 5.8 TB/s; a thread to each piece with the
// slots in shared memory, each kind of piece read and written in turn, 89.
// Both, back to back: one request cut from 4608 to 4096 tokens 10.7 us, 32 cut from 4200..9000 to 4001 93.
#include <cuda_bf16.h>

#include "common.cuh"
#include "sm100_ptx.cuh"

namespace mpfa {
namespace {

struct EvictParams {
  uint8_t *k_codes, *k_sf, *v_fp8;
  uint16_t *delta;            // may be null
  const int32_t *page_table, *seq_lens, *new_table;
  const float *weights;
  int32_t *kept, *new_lens;
  float *new_weights;
  int32_t *status;
  size_t weights_stride, new_stride;
  int B, H_q, H_kv, num_pages, max_pages, new_pages, keep, sinks, recent;
  __device__ __forceinline__ int length(int b) const { return min(max(seq_lens[b], 0), max_pages * PAGE); }
};

constexpr int SEL_THREADS = 1024, SEL_WARPS = SEL_THREADS / 32;
constexpr int DIGIT = 12, BINS = 1 << DIGIT;
constexpr int LIST = SEL_THREADS / 4;   // ranked against one another by four threads each
constexpr int SEL_CACHE = 49152;   // weights held in shared memory between the passes: 192 KB
constexpr int SEL_AHEAD = 4;       // loads of a thread on the way

__device__ __forceinline__ uint32_t order_of(float w) {
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// What the warps before this one have, of a count for each warp in tmp.
__device__ __forceinline__ uint32_t before_warp(const uint32_t *tmp) {
  static_assert(SEL_WARPS == 32, "a lane for each warp");
  const int lane = threadIdx.x & 31;
  return __reduce_add_sync(0xffffffffu, lane < (int)(threadIdx.x >> 5) ? tmp[lane] : 0u);
}

struct SelectShared {
  union {   // the list is made when the last histogram has been read
    __align__(16) uint32_t hist[BINS];
    uint64_t list[LIST];
  };
  uint32_t tmp[2][SEL_WARPS], bin, need, inside, listed;
  uint64_t border;
};

// The slots kept of n > keep, to kept[] in ascending order.  HELD: `held` has the orders of all weights, and sh.hist the counts of the
// candidates' first digits; otherwise both are made from the weights w in global memory.
template <bool HELD>
__device__ __forceinline__ void select_tokens(const EvictParams &p, const uint32_t *held, const float *w, int n, int32_t *kept, SelectShared &sh) {
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  const int first = p.sinks, last = n - p.recent;   // the candidates: [first, last)
  auto order = [&](int i) { return HELD ? held[i] : order_of(w[i]); };
  uint32_t need = (uint32_t)(p.keep - p.sinks - p.recent);
  uint32_t least = 0xffffffffu;   // no weight has this order
  int slot = -1;                  // of those of the least order, the last that stays
  if (need > 0) {
    // the digits so far, of the orders and then of the slots' complements
    uint32_t value = 0, mask = 0, s_value = 0, s_mask = 0;
    int shift = 32;
    bool by_slot = false, counted = HELD;
#pragma unroll 1
    for (uint32_t inside = (uint32_t)(last - first); inside > LIST; counted = false) {
      if (shift == 0) shift = 32, by_slot = true;
      const int bits = min(DIGIT, shift);
      shift -= bits;
      const uint32_t digit = (1u << bits) - 1u;
      if (!counted) {
        __syncthreads();   // of the pass before: bin, need, inside and the histogram have been read
        reinterpret_cast<uint4 *>(sh.hist)[t] = make_uint4(0u, 0u, 0u, 0u);
        __syncthreads();
#pragma unroll 2
        for (int i = first + t; i < last; i += SEL_THREADS) {
          const uint32_t u = order(i), s = ~(uint32_t)i;
          if ((u & mask) == value && (s & s_mask) == s_value) atomicAdd(&sh.hist[((by_slot ? s : u) >> shift) & digit], 1u);
        }
      }
      __syncthreads();
      // four bins to a lane, the highest first: the warp, then the lane and the bin in which the count from above reaches `need`
      static_assert(BINS == 4 * SEL_THREADS, "four bins to a thread");
      const uint4 c4 = reinterpret_cast<const uint4 *>(sh.hist)[SEL_THREADS - 1 - t];
      const uint32_t c[4] = {c4.w, c4.z, c4.y, c4.x}, sum = (c[0] + c[1]) + (c[2] + c[3]), total = __reduce_add_sync(0xffffffffu, sum);
      if (lane == 0) sh.tmp[0][warp] = total;
      __syncthreads();
      uint32_t above = before_warp(sh.tmp[0]);
      if (above < need && need <= above + total) {
        uint32_t incl = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const uint32_t v = __shfl_up_sync(0xffffffffu, incl, o);
          if (lane >= o) incl += v;
        }
        above += incl - sum;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          if (above < need && need <= above + c[u]) sh.bin = (uint32_t)(BINS - 1 - 4 * t - u), sh.need = need - above, sh.inside = c[u];
          above += c[u];
        }
      }
      if (t == 0) sh.listed = 0;
      __syncthreads();
      (by_slot ? s_value : value) |= sh.bin << shift;
      (by_slot ? s_mask : mask) |= digit << shift;
      need = sh.need, inside = sh.inside;
    }
    // the candidates of that bin, in any order; the one with need - 1 larger ones is the last that stays
    __syncthreads();
    if (mask == 0) {   // no digit was needed
      if (t == 0) sh.listed = 0;
      __syncthreads();
    }
#pragma unroll 4
    for (int i = first + t; i < last; i += SEL_THREADS) {
      const uint32_t u = order(i), s = ~(uint32_t)i;
      if ((u & mask) == value && (s & s_mask) == s_value) sh.list[atomicAdd(&sh.listed, 1u)] = (uint64_t)u << 32 | s;
    }
    __syncthreads();
    // four threads to a candidate
    const int m = (int)sh.listed;
    if (warp * 8 < m) {
      const uint64_t mine = (t >> 2) < m ? sh.list[t >> 2] : ~0ull;
      uint32_t larger = 0;
#pragma unroll 4
      for (int i = t & 3; i < m; i += 4) larger += sh.list[i] > mine ? 1u : 0u;
      larger += __shfl_xor_sync(0xffffffffu, larger, 1);
      larger += __shfl_xor_sync(0xffffffffu, larger, 2);
      if ((t >> 2) < m && larger == need - 1) sh.border = mine;
    }
    __syncthreads();
    least = (uint32_t)(sh.border >> 32), slot = (int)~(uint32_t)sh.border;
  }
  // In the order of the slots: each warp takes a run of them, counts, and writes when it knows what the warps before it have.
  const int run = ((n + SEL_WARPS - 1) / SEL_WARPS + 31) / 32 * 32, begin = min(warp * run, n), end = min(begin + run, n);
  auto stays = [&](int i) {
    if (i >= end) return false;
    const uint32_t u = order(i);
    return i < first || i >= last || u > least || (u == least && i <= slot);
  };
  uint32_t count = 0, answers = 0;   // of the first 32 groups of 32 slots lane k keeps the k-th answer
#pragma unroll 2
  for (int i0 = begin, k = 0; i0 < end; i0 += 32, ++k) {
    const uint32_t bits = __ballot_sync(0xffffffffu, stays(i0 + lane));
    count += __popc(bits);
    if (k == lane) answers = bits;
  }
  if (lane == 0) sh.tmp[1][warp] = count;
  __syncthreads();
  uint32_t to = before_warp(sh.tmp[1]);
#pragma unroll 2
  for (int i0 = begin, k = 0; i0 < end; i0 += 32, ++k) {
    const uint32_t bits = k < 32 ? __shfl_sync(0xffffffffu, answers, k) : __ballot_sync(0xffffffffu, stays(i0 + lane));
    if (bits >> lane & 1u) kept[to + __popc(bits & ((1u << lane) - 1u))] = i0 + lane;
    to += __popc(bits);
  }
}

__global__ void __launch_bounds__(SEL_THREADS) evict_select_kernel(const __grid_constant__ EvictParams p) {
  extern __shared__ uint32_t held[];          // the orders of the weights, where they fit
  __shared__ SelectShared sh;
  grid_dependency_wait();
  launch_dependents();
  const int hk = blockIdx.x, b = blockIdx.y, t = threadIdx.x;
  const size_t head = (size_t)b * p.H_kv + hk;
  const float *const w = p.weights + head * p.weights_stride;
  int32_t *const kept = p.kept + head * p.keep;
  float *const out = p.new_weights + head * p.new_stride;
  // the first weights are requested before the length is known: their slots exist whatever it is
  const int most = p.max_pages * PAGE;
  float x[SEL_AHEAD];
#pragma unroll
  for (int u = 0; u < SEL_AHEAD; ++u) x[u] = t + u * SEL_THREADS < most ? w[t + u * SEL_THREADS] : 0.0f;
  const int n = p.length(b), count = min(n, p.keep);
  reinterpret_cast<uint4 *>(sh.hist)[t] = make_uint4(0u, 0u, 0u, 0u);
  if (hk == 0 && t == 0) p.new_lens[b] = count;
  for (size_t i = (size_t)count + t; i < p.new_stride; i += SEL_THREADS) out[i] = 0.0f;
  for (int i = count + t; i < p.keep; i += SEL_THREADS) kept[i] = -1;
  if (n <= p.keep) {
    for (int i = t; i < n; i += SEL_THREADS) kept[i] = i;
  } else if (n <= SEL_CACHE) {
    __syncthreads();
#pragma unroll 1
    for (int i0 = t;;) {
#pragma unroll
      for (int u = 0; u < SEL_AHEAD; ++u) {
        const int i = i0 + u * SEL_THREADS;
        if (i < n) {
          const uint32_t o = order_of(x[u]);
          held[i] = o;
          if (i >= p.sinks && i < n - p.recent) atomicAdd(&sh.hist[o >> (32 - DIGIT)], 1u);
        }
      }
      i0 += SEL_AHEAD * SEL_THREADS;
      if (i0 >= n) break;
#pragma unroll
      for (int u = 0; u < SEL_AHEAD; ++u) x[u] = i0 + u * SEL_THREADS < n ? w[i0 + u * SEL_THREADS] : 0.0f;
    }
    __syncthreads();
    select_tokens<true>(p, held, w, n, kept, sh);
  } else {
    select_tokens<false>(p, held, w, n, kept, sh);
  }
}

// A warp takes eight tokens of a new page: their V is 64 pieces of 16 bytes, their K codes 32, and their Delta_S 16 bytes of each head's
// row there.  Everything is read before anything is written.
constexpr int MOVE_THREADS = 256;
__global__ void __launch_bounds__(MOVE_THREADS, 8) evict_move_kernel(const __grid_constant__ EvictParams p) {
  const int page = blockIdx.x, hk = blockIdx.y, b = blockIdx.z, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  grid_dependency_wait();
  const int at = page * PAGE + warp * 8 + (lane & 7);   // lane l: token l mod 8
  const int to = p.new_table[(size_t)b * p.new_pages + page];
  const int from = at < p.keep ? p.kept[((size_t)b * p.H_kv + hk) * p.keep + at] : -1;   // -1 past the last token
  const int count = min(p.length(b), p.keep);
  if (page * PAGE >= count) return;
  if (from >= 0 && lane < 8) {
    const size_t head = (size_t)b * p.H_kv + hk;
    p.new_weights[head * p.new_stride + at] = p.weights[head * p.weights_stride + from];
  }
  if (to < 0 || to >= p.num_pages) {
    if (threadIdx.x == 0) atomicOr(p.status, MPFA_DEV_BAD_PAGE);
    return;
  }
  int id = -1;
  if (from >= 0) {
    id = p.page_table[(size_t)b * p.max_pages + from / PAGE];
    if (id < 0 || id >= p.num_pages) {
      id = -1;
      atomicOr(p.status, MPFA_DEV_BAD_PAGE);
    }
  }
  const int slot = from & (PAGE - 1);
  const int G = p.H_q / p.H_kv;
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
  uint4 v[2] = {zero, zero}, k = zero;
  uint2 sf = make_uint2(0u, 0u);
  uint16_t d[2] = {0, 0};
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int i = (lane >> 3) + 4 * u, c = lane & 7;
    const int id_i = __shfl_sync(0xffffffffu, id, i), s = __shfl_sync(0xffffffffu, slot, i);
    if (id_i >= 0) v[u] = *reinterpret_cast<const uint4 *>(p.v_fp8 + ((size_t)id_i * p.H_kv + hk) * 8192 + s * 128 + ((c ^ (s & 7)) << 4));
  }
  {
    const int i = lane >> 2, c = lane & 3;
    const int id_i = __shfl_sync(0xffffffffu, id, i), s = __shfl_sync(0xffffffffu, slot, i);
    if (id_i >= 0) k = *reinterpret_cast<const uint4 *>(p.k_codes + ((size_t)id_i * p.H_kv + hk) * 4096 + s * 64 + ((c ^ ((s & 7) >> 1)) << 4));
  }
  if (id >= 0) {
    const size_t slab = (size_t)id * p.H_kv + hk;
    if (lane < 8) sf = *reinterpret_cast<const uint2 *>(p.k_sf + slab * 512 + slot * 8);
    if (p.delta) {
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int g = (lane >> 3) + 4 * u;
        if (g < G) d[u] = p.delta[(slab * G + g) * PAGE + (((slot >> 3) ^ g) << 3) + (slot & 7)];
      }
    }
  }
  const size_t dst = (size_t)to * p.H_kv + hk;
  const int row = warp * 8;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int i = (lane >> 3) + 4 * u, c = lane & 7;
    *reinterpret_cast<uint4 *>(p.v_fp8 + dst * 8192 + (row + i) * 128 + ((c ^ i) << 4)) = v[u];
  }
  {
    const int i = lane >> 2, c = lane & 3;
    *reinterpret_cast<uint4 *>(p.k_codes + dst * 4096 + (row + i) * 64 + ((c ^ (i >> 1)) << 4)) = k;
  }
  if (lane < 8) *reinterpret_cast<uint2 *>(p.k_sf + dst * 512 + (row + lane) * 8) = sf;
  if (p.delta) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int g = (lane >> 3) + 4 * u;
      if (g < G) p.delta[(dst * G + g) * PAGE + ((warp ^ g) << 3) + (lane & 7)] = d[u];
    }
  }
}

bool overlap(const void *a, size_t na, const void *b, size_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + nb && y < x + na;
}

}  // namespace
}  // namespace mpfa

using namespace mpfa;

extern "C" mpfa_status mpfa_evict_paged(const mpfa_paged_kv *kv, const int32_t *page_table, int B, int max_pages_per_req,
                                        const int32_t *seq_lens, const float *weights, int weights_stride, int keep, int sinks, int recent,
                                        const int32_t *new_table, int new_max_pages, int32_t *kept, int32_t *new_lens, float *new_weights,
                                        int new_weights_stride, int32_t *device_status, void *stream) {
  if (!kv || !page_table || !seq_lens || !weights || !new_table || !kept || !new_lens || !new_weights || !device_status)
    return MPFA_ERR_INVALID_ARG;
  if (!kv->k_codes || !kv->k_sf || !kv->v_fp8 || kv->num_pages <= 0 || kv->H_q <= 0 || kv->H_kv <= 0) return MPFA_ERR_INVALID_ARG;
  if (B <= 0 || max_pages_per_req <= 0 || new_max_pages <= 0 || keep <= 0 || sinks < 0 || recent < 0) return MPFA_ERR_INVALID_ARG;
  if ((int64_t)sinks + recent > keep || (int64_t)new_max_pages * PAGE < keep) return MPFA_ERR_INVALID_ARG;
  if (kv->page_size != PAGE || kv->H_q % kv->H_kv != 0 || kv->H_q / kv->H_kv > 8) return MPFA_ERR_UNSUPPORTED;
  if (max_pages_per_req > (1 << 24) || new_max_pages > (1 << 24) || B > 65535 || kv->H_kv > 65535) return MPFA_ERR_UNSUPPORTED;
  if (weights_stride < max_pages_per_req * PAGE || new_weights_stride < keep) return MPFA_ERR_INVALID_ARG;
  const size_t heads = (size_t)B * kv->H_kv;
  if (overlap(weights, heads * weights_stride * sizeof(float), new_weights, heads * new_weights_stride * sizeof(float)) ||
      overlap(seq_lens, (size_t)B * sizeof(int32_t), new_lens, (size_t)B * sizeof(int32_t)))
    return MPFA_ERR_INVALID_ARG;
  if (!aligned(kv->k_codes, 256) || !aligned(kv->k_sf, 256) || !aligned(kv->v_fp8, 256) || !aligned(kv->delta_s_bf16, 256) ||
      !aligned(weights, 4) || !aligned(new_weights, 4))
    return MPFA_ERR_ALIGNMENT;
  int dev = 0, n_sm = 0;
  mpfa_status rc = device_info(&dev, &n_sm);
  if (rc != MPFA_OK) return rc;
  EvictParams p;
  p.k_codes = kv->k_codes;
  p.k_sf = kv->k_sf;
  p.v_fp8 = kv->v_fp8;
  p.delta = static_cast<uint16_t *>(kv->delta_s_bf16);
  p.page_table = page_table;
  p.seq_lens = seq_lens;
  p.new_table = new_table;
  p.weights = weights;
  p.kept = kept;
  p.new_lens = new_lens;
  p.new_weights = new_weights;
  p.status = device_status;
  p.weights_stride = (size_t)weights_stride;
  p.new_stride = (size_t)new_weights_stride;
  p.B = B;
  p.H_q = kv->H_q;
  p.H_kv = kv->H_kv;
  p.num_pages = kv->num_pages;
  p.max_pages = max_pages_per_req;
  p.new_pages = new_max_pages;
  p.keep = keep;
  p.sinks = sinks;
  p.recent = recent;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const int most = max_pages_per_req * PAGE;   // no request is longer
  const size_t smem = (size_t)(most <= SEL_CACHE ? most : SEL_CACHE) * sizeof(uint32_t);
  if ((rc = allow_smem<evict_select_kernel>(smem)) != MPFA_OK) return rc;
  MPFA_CUDA_OK(launch(evict_select_kernel, dim3((unsigned)p.H_kv, (unsigned)B), dim3(SEL_THREADS), smem, s, p));
  const int pages = (keep + PAGE - 1) / PAGE;
  MPFA_CUDA_OK(launch(evict_move_kernel, dim3((unsigned)(pages < max_pages_per_req ? pages : max_pages_per_req), (unsigned)p.H_kv, (unsigned)B),
                      dim3(MOVE_THREADS), 0, s, p));
  return MPFA_OK;
}
