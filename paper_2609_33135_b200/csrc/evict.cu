// Eviction from the paged cache by accumulated attention weight, for sm_100a: two kernels, neither with any arithmetic on the tokens.
//
// evict_select_kernel, one CTA per (request, kv head).  Of n > keep tokens the first `sinks` and the last `recent` stay; of the others
// the need = keep - sinks - recent of largest weight, equal ones by slot.  Weights are ordered as the 32-bit integers that compare like
// them (-0 as +0, NaN below everything).  The need-th largest is found digit by digit (11, 11, 10 bits): a histogram of the candidates
// that agree with the digits so far, and the bin in which the count from above reaches what is still needed.  Then one ordered pass
// over the slots writes those above the value found, and the lowest slots of those equal to it.  Histograms are integer counts, so the
// order of the atomics does not show.  One read of the weights from memory: the passes after the first find them in shared memory, or
// in L2 where there are more than fit.
//
// evict_move_kernel, one CTA per (new page, kv head, request): the 64 tokens of the page from their slots.  A token's K codes, scales,
// V and Delta_S entries are whole 16-, 8- and 2-byte pieces in every slot, whose places depend on the slot (include/mpfa.h), so the new
// page is written once, in full, with the rest of it zeros.
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
constexpr int DIGIT = 11, BINS = 1 << DIGIT;
constexpr int SEL_CACHE = 49152;   // weights held in shared memory between the passes: 192 KB

__device__ __forceinline__ uint32_t order_of(float w) {
  if (w != w) return 0u;
  const uint32_t u = __float_as_uint(w + 0.0f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Exclusive sum over the block in thread order, and the total.  tmp: SEL_WARPS + 1 words.
__device__ __forceinline__ uint32_t block_scan(uint32_t x, uint32_t *tmp, uint32_t &total) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint32_t incl = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t v = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += v;
  }
  __syncthreads();   // tmp of the scan before has been read
  if (lane == 31) tmp[warp] = incl;
  __syncthreads();
  if (warp == 0) {
    const uint32_t mine = tmp[lane];
    uint32_t s = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t v = __shfl_up_sync(0xffffffffu, s, o);
      if (lane >= o) s += v;
    }
    tmp[lane] = s - mine;
    if (lane == 31) tmp[SEL_WARPS] = s;
  }
  __syncthreads();
  total = tmp[SEL_WARPS];
  return tmp[warp] + incl - x;
}

__global__ void __launch_bounds__(SEL_THREADS) evict_select_kernel(const __grid_constant__ EvictParams p) {
  extern __shared__ uint32_t held[];          // the order of each slot's weight, where they fit
  __shared__ uint32_t hist[BINS], tmp[SEL_WARPS + 1], found[2];
  grid_dependency_wait();
  launch_dependents();
  const int hk = blockIdx.x, b = blockIdx.y, t = threadIdx.x;
  const size_t head = (size_t)b * p.H_kv + hk;
  const float *const w = p.weights + head * p.weights_stride;
  int32_t *const kept = p.kept + head * p.keep;
  float *const out = p.new_weights + head * p.new_stride;
  const int n = p.length(b), count = min(n, p.keep);
  if (hk == 0 && t == 0) p.new_lens[b] = count;
  for (size_t i = (size_t)count + t; i < p.new_stride; i += SEL_THREADS) out[i] = 0.0f;
  for (int i = count + t; i < p.keep; i += SEL_THREADS) kept[i] = -1;
  if (n <= p.keep) {
    for (int i = t; i < n; i += SEL_THREADS) kept[i] = i, out[i] = w[i];
    return;
  }
  const int first = p.sinks, last = n - p.recent;   // the candidates: [first, last)
  const bool fits = n <= SEL_CACHE;
  if (fits)
    for (int i = t; i < n; i += SEL_THREADS) held[i] = order_of(w[i]);
  uint32_t need = (uint32_t)(p.keep - p.sinks - p.recent), value = 0, mask = 0;
  if (need > 0) {
    int shift = 32;
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
      const int bits = pass < 2 ? DIGIT : 32 - 2 * DIGIT;
      shift -= bits;
      __syncthreads();
      for (int i = t; i < BINS; i += SEL_THREADS) hist[i] = 0;
      __syncthreads();
      for (int i = first + t; i < last; i += SEL_THREADS) {
        const uint32_t u = fits ? held[i] : order_of(w[i]);
        if ((u & mask) == value) atomicAdd(&hist[(u >> shift) & ((1u << bits) - 1u)], 1u);
      }
      __syncthreads();
      // two bins to a thread, the highest first: the bin in which the count from above reaches `need`
      const int hi = BINS - 1 - 2 * t;
      const uint32_t a = hist[hi], c = hist[hi - 1];
      uint32_t total;
      const uint32_t above = block_scan(a + c, tmp, total);
      if (above < need && need <= above + a + c) {
        const bool second = need > above + a;
        found[0] = (uint32_t)(second ? hi - 1 : hi);
        found[1] = need - above - (second ? a : 0u);   // how many of that bin
      }
      __syncthreads();
      value |= found[0] << shift;
      mask |= ((1u << bits) - 1u) << shift;
      need = found[1];
    }
  } else {
    value = 0xffffffffu;
  }
  // All candidates above `value` and the first `need` of those equal to it, in the order of the slots.
  __syncthreads();
  uint32_t at = 0, equal = 0;   // written, and equal ones met, so far
#pragma unroll 1
  for (int i0 = 0; i0 < n; i0 += SEL_THREADS) {
    const int i = i0 + t;
    const bool in = i < n, candidate = in && i >= first && i < last;
    float x = 0.0f;
    uint32_t u = 0;
    if (in) x = w[i], u = candidate ? (fits ? held[i] : order_of(x)) : 0u;
    const bool eq = candidate && u == value && p.keep > p.sinks + p.recent;
    const bool sure = in && (!candidate || u > value);
    // both counts in one scan: at most 1024 each
    uint32_t total;
    const uint32_t before = block_scan((sure ? 1u : 0u) | (eq ? 0x10000u : 0u), tmp, total);
    const uint32_t eq_before = equal + (before >> 16);
    const bool take = sure || (eq && eq_before < need);
    // of the equal ones before this slot, those that were taken count
    const uint32_t eq_taken = min(eq_before, need) - min(equal, need);
    if (take) {
      const uint32_t to = at + (before & 0xffffu) + eq_taken;
      kept[to] = i;
      out[to] = x;
    }
    const uint32_t eq_total = total >> 16;
    at += (total & 0xffffu) + min(equal + eq_total, need) - min(equal, need);
    equal += eq_total;
  }
}

constexpr int MOVE_THREADS = 256;
__global__ void __launch_bounds__(MOVE_THREADS) evict_move_kernel(const __grid_constant__ EvictParams p) {
  __shared__ int64_t slab[PAGE];   // (page, kv head) slab that a token comes from, -1: none
  __shared__ int slot[PAGE];
  const int page = blockIdx.x, hk = blockIdx.y, b = blockIdx.z, t = threadIdx.x;
  grid_dependency_wait();
  const int count = min(p.length(b), p.keep);
  if (page * PAGE >= count) return;
  const int to = p.new_table[(size_t)b * p.new_pages + page];
  if (to < 0 || to >= p.num_pages) {
    if (t == 0) atomicOr(p.status, MPFA_DEV_BAD_PAGE);
    return;
  }
  if (t < PAGE) {
    int64_t s = -1;
    int at = 0;
    if (page * PAGE + t < count) {
      at = p.kept[((size_t)b * p.H_kv + hk) * p.keep + page * PAGE + t];
      const int from = p.page_table[(size_t)b * p.max_pages + at / PAGE];
      if (from >= 0 && from < p.num_pages)
        s = (int64_t)from * p.H_kv + hk;
      else
        atomicOr(p.status, MPFA_DEV_BAD_PAGE);
    }
    slab[t] = s;
    slot[t] = at % PAGE;
  }
  __syncthreads();
  const size_t dst = (size_t)to * p.H_kv + hk;
  const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
  {   // K codes: four 16-byte pieces a token
    const int i = t >> 2, c = t & 3, s = slot[i];
    uint4 x = zero;
    if (slab[i] >= 0) x = *reinterpret_cast<const uint4 *>(p.k_codes + slab[i] * 4096 + s * 64 + ((c ^ ((s & 7) >> 1)) << 4));
    *reinterpret_cast<uint4 *>(p.k_codes + dst * 4096 + i * 64 + ((c ^ ((i & 7) >> 1)) << 4)) = x;
  }
#pragma unroll
  for (int u = 0; u < 2; ++u) {   // V: eight
    const int i = (t >> 3) + 32 * u, c = t & 7, s = slot[i];
    uint4 x = zero;
    if (slab[i] >= 0) x = *reinterpret_cast<const uint4 *>(p.v_fp8 + slab[i] * 8192 + s * 128 + ((c ^ (s & 7)) << 4));
    *reinterpret_cast<uint4 *>(p.v_fp8 + dst * 8192 + i * 128 + ((c ^ (i & 7)) << 4)) = x;
  }
  if (t < PAGE) {
    uint2 x = make_uint2(0u, 0u);
    if (slab[t] >= 0) x = *reinterpret_cast<const uint2 *>(p.k_sf + slab[t] * 512 + slot[t] * 8);
    *reinterpret_cast<uint2 *>(p.k_sf + dst * 512 + t * 8) = x;
  }
  if (p.delta) {
    const int G = p.H_q / p.H_kv;
    for (int k = t; k < G * PAGE; k += MOVE_THREADS) {
      const int g = k / PAGE, i = k % PAGE, s = slot[i];
      uint16_t x = 0;
      if (slab[i] >= 0) x = p.delta[(slab[i] * G + g) * PAGE + (((s >> 3) ^ (g & 7)) << 3) + (s & 7)];
      p.delta[(dst * G + g) * PAGE + (((i >> 3) ^ (g & 7)) << 3) + (i & 7)] = x;
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
  if (max_pages_per_req > (1 << 24) || B > 65535 || kv->H_kv > 65535) return MPFA_ERR_UNSUPPORTED;
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
