// Eviction from the paged cache by accumulated attention weight, for sm_100a: two kernels, neither with any arithmetic on the tokens.
//
// evict_select_kernel, one CTA per row of weights (request, kv head), or where rows are long and few a cluster: each CTA takes a part of the
// slots, its histogram's counts are added up by all of them, a part of the bins each, and the first ranks the list.  Of n > keep tokens the first `sinks` and the last `recent` stay; of the others
// the need = keep - sinks - recent with the largest 64-bit keys: the weight as the 32-bit integer that compares like it (-0 as +0, NaN
// below everything), then the slot's complement.  No two keys are equal, so what is kept is what is not below the need-th largest.
// It is found by digits of 12 bits from the top: a histogram of the candidates that agree with the digits so far, and the bin in which the
// count from above reaches what is still needed.  As soon as that bin holds few enough they are listed and ranked against one another;
// with weights that differ that is after the first digit, which is counted as the weights arrive.  Histograms are integer counts and the
// list's order decides nothing, so the order of the atomics does not show.  One read of the weights from memory: what comes after finds them
// in shared memory, or in L2 where there are more than fit.
// Bound by instructions and by barriers of 32 warps, not by memory: 8 heads of 4608 weights 8 us, 256 of 4200..9000 18 us (two CTAs to an
// SM, 74 to 77 % of issue slots).  Not kept: three digits to the end and two scans of the block (25 us; 512 or 256 threads 16 us for the 8 heads),
// copies of the histogram by lane (no gain: 60 bins hold most counts, but the conflicts are not what it waits for).  One CTA to a row of 131072
// weights: the whole call 164 us, by eight 30.5 (the rule and more figures stand at the launch; a row that is short in a wide table pays 3 us
// for the cluster).
//
// evict_move_kernel, one CTA per (new page, kv head, request): the 64 tokens of the page from their slots.  A token's K codes, scales,
// V and Delta_S entries are whole 16-, 8- and 2-byte pieces in every slot, whose places depend on the slot (include/mpfa.h), so the new
// page is written once, in full, with the rest of it zeros.  Bound by memory: 32 requests x 8 heads x 4001 tokens, 0.21 GB read (0.26 from
// DRAM: 2 bytes of Delta_S and 8 of scales out of 32-byte sectors) and as much written, 75 us alone, 5.8 TB/s; a thread to each piece with the
// slots in shared memory, each kind of piece read and written in turn, 89.
// Both, back to back: one request cut from 4608 to 4096 tokens 10.7 us (9.8 to 12.1), 32 cut from 4200..9000 to 4001 93 to 95.
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
constexpr int SEL_ALONE = 16384, SEL_PART = 4096;   // slots that the longest row can have: for one CTA; for each of several, at least

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

constexpr int SEL_CLUSTER = 8;
struct SelectShared {
  union {   // the list is made when the last histogram has been read
    __align__(16) uint32_t hist[BINS];
    uint64_t list[LIST];        // the first CTA's
  };
  uint32_t tmp[2][SEL_WARPS], bin, need, inside, listed;
  uint32_t total[SEL_CLUSTER], stay[SEL_CLUSTER];   // each CTA's candidates in its part of the bins; its slots that stay
  uint64_t border;
};

// The CTAs that share a row: C of them, this one the r-th.  One: shared memory and barriers of its own.
template <bool CLUSTER>
struct Team {
  int C, r;
  __device__ __forceinline__ void sync() const {   // writes to shared memory, the others' included, are seen after it
    if (CLUSTER) {
      __syncwarp();
      cluster_arrive();
      cluster_wait();
    } else {
      __syncthreads();
    }
  }
  template <class T>
  __device__ __forceinline__ void tell(T &x, T value) const {   // one thread: the variable in every CTA
    if (CLUSTER) {
      for (int q = 0; q < C; ++q) cluster_store(cluster_address(smem_u32(&x), q), value);
    } else {
      x = value;
    }
  }
};

// This CTA's part [begin, end) of a row of n > keep slots: those that stay, to kept[] in ascending order.  HELD: `held` has the orders of the
// part's weights (from held[0] on), and sh.hist the counts of its candidates' first digits; otherwise both are made from the weights w in
// global memory.  Those are read in each pass, and a program that goes on adding to them meanwhile makes the passes disagree: then a bin may not
// be found, more be listed than were counted, and more stay than the row has room for, so each of the three has its own bound there.
template <bool CLUSTER, bool HELD>
__device__ __forceinline__ void select_tokens(const EvictParams &p, const Team<CLUSTER> &team, const uint32_t *held, const float *w, int n, int begin,
                                              int end, int32_t *kept, SelectShared &sh) {
  const int t = threadIdx.x, warp = t >> 5, lane = t & 31;
  const int first = max(p.sinks, begin), last = min(n - p.recent, end);   // the part's candidates: [first, last)
  auto order = [&](int i) { return HELD ? held[i - begin] : order_of(w[i]); };
  uint32_t need = (uint32_t)(p.keep - p.sinks - p.recent);
  uint32_t least = 0xffffffffu;   // no weight has this order
  int slot = -1;                  // of those of the least order, the last that stays
  if (need > 0) {
    // the digits so far, of the orders and then of the slots' complements
    uint32_t value = 0, mask = 0, s_value = 0, s_mask = 0;
    int shift = 32;
    bool by_slot = false, counted = HELD;
#pragma unroll 1
    for (uint32_t inside = (uint32_t)(n - p.recent - p.sinks); inside > LIST; counted = false) {
      if (shift == 0) {
        if (!HELD && by_slot) break;
        shift = 32, by_slot = true;
      }
      const int bits = min(DIGIT, shift);
      shift -= bits;
      const uint32_t digit = (1u << bits) - 1u;
      if (!counted) {
        __syncthreads();   // of the pass before: bin, need and inside have been read, and the histogram before that
        reinterpret_cast<uint4 *>(sh.hist)[t] = make_uint4(0u, 0u, 0u, 0u);
        __syncthreads();
#pragma unroll 2
        for (int i = first + t; i < last; i += SEL_THREADS) {
          const uint32_t u = order(i), s = ~(uint32_t)i;
          if ((u & mask) == value && (s & s_mask) == s_value) atomicAdd(&sh.hist[((by_slot ? s : u) >> shift) & digit], 1u);
        }
      }
      team.sync();
      // Each CTA takes its part of the bins, the highest first, four to a lane or fewer, adds up what all CTAs have there and tells the others
      // the sum; the part, the warp, the lane and the bin are found in which the count from above reaches `need`.
      static_assert(BINS == 4 * SEL_THREADS, "at most four bins to a thread");
      uint32_t c[4] = {0u, 0u, 0u, 0u};
      int top;   // the thread's highest bin
      if (CLUSTER) {
        const int part = BINS / team.C, per = max(part / SEL_THREADS, 1);
        top = BINS - 1 - team.r * part - t * per;
#pragma unroll
        for (int u = 0; u < 2; ++u)
          if (u < per && t * per < part) {
            const uint32_t at = smem_u32(&sh.hist[top - u]);
            for (int q = 0; q < team.C; ++q) c[u] += cluster_load(cluster_address(at, q));
          }
      } else {
        top = BINS - 1 - 4 * t;
        const uint4 c4 = reinterpret_cast<const uint4 *>(sh.hist)[SEL_THREADS - 1 - t];
        c[0] = c4.w, c[1] = c4.z, c[2] = c4.y, c[3] = c4.x;
      }
      const uint32_t sum = (c[0] + c[1]) + (c[2] + c[3]), total = __reduce_add_sync(0xffffffffu, sum);
      if (lane == 0) sh.tmp[0][warp] = total;
      __syncthreads();
      uint32_t above = before_warp(sh.tmp[0]);
      if (CLUSTER) {
        if (warp == 0) {
          const uint32_t all = __reduce_add_sync(0xffffffffu, sh.tmp[0][lane]);
          if (lane < team.C) cluster_store(cluster_address(smem_u32(&sh.total[team.r]), lane), all);
        }
        team.sync();
        for (int q = 0; q < team.r; ++q) above += sh.total[q];
      }
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
          if (above < need && need <= above + c[u]) team.tell(sh.bin, (uint32_t)(top - u)), team.tell(sh.need, need - above), team.tell(sh.inside, c[u]);
          above += c[u];
        }
      }
      team.sync();
      (by_slot ? s_value : value) |= sh.bin << shift;
      (by_slot ? s_mask : mask) |= digit << shift;
      need = sh.need, inside = sh.inside;
    }
    // The candidates of that bin, in any order, on the first CTA; the one with need - 1 larger ones is the last that stays.
    if (t == 0) sh.listed = 0;
    team.sync();
#pragma unroll 4
    for (int i = first + t; i < last; i += SEL_THREADS) {
      const uint32_t u = order(i), s = ~(uint32_t)i;
      if ((u & mask) == value && (s & s_mask) == s_value) {
        const uint64_t key = (uint64_t)u << 32 | s;
        if (CLUSTER) {
          const uint32_t at = cluster_add(cluster_address(smem_u32(&sh.listed), 0), 1u);
          if (HELD || at < LIST) cluster_store(cluster_address(smem_u32(&sh.list[0]), 0) + 8 * at, key);
        } else {
          const uint32_t at = atomicAdd(&sh.listed, 1u);
          if (HELD || at < LIST) sh.list[at] = key;
        }
      }
    }
    team.sync();
    // four threads to a candidate
    if (!CLUSTER || team.r == 0) {
      const int m = HELD ? (int)sh.listed : min((int)sh.listed, LIST);
      if (warp * 8 < m) {
        const uint64_t mine = (t >> 2) < m ? sh.list[t >> 2] : ~0ull;
        uint32_t larger = 0;
#pragma unroll 4
        for (int i = t & 3; i < m; i += 4) larger += sh.list[i] > mine ? 1u : 0u;
        larger += __shfl_xor_sync(0xffffffffu, larger, 1);
        larger += __shfl_xor_sync(0xffffffffu, larger, 2);
        if ((t & 3) == 0 && (t >> 2) < m && larger == need - 1) team.tell(sh.border, mine);
      }
    }
    team.sync();
    least = (uint32_t)(sh.border >> 32), slot = (int)~(uint32_t)sh.border;
  }
  // In the order of the slots: each warp takes a run of them, counts, and writes when it knows what is before it.
  const int run = ((end - begin + SEL_WARPS - 1) / SEL_WARPS + 31) / 32 * 32, from = min(begin + warp * run, end), until = min(from + run, end);
  auto stays = [&](int i) {
    if (i >= until) return false;
    const uint32_t u = order(i);
    return i < p.sinks || i >= n - p.recent || u > least || (u == least && i <= slot);
  };
  uint32_t count = 0, answers = 0;   // of the first 32 groups of 32 slots lane k keeps the k-th answer
#pragma unroll 2
  for (int i0 = from, k = 0; i0 < until; i0 += 32, ++k) {
    const uint32_t bits = __ballot_sync(0xffffffffu, stays(i0 + lane));
    count += __popc(bits);
    if (k == lane) answers = bits;
  }
  if (lane == 0) sh.tmp[1][warp] = count;
  __syncthreads();
  uint32_t to = before_warp(sh.tmp[1]);
  if (CLUSTER) {
    if (p.keep == p.sinks + p.recent) team.sync();   // no other barrier has told that all CTAs are there
    if (warp == 0) {
      const uint32_t all = __reduce_add_sync(0xffffffffu, sh.tmp[1][lane]);
      if (lane < team.C) cluster_store(cluster_address(smem_u32(&sh.stay[team.r]), lane), all);
    }
    team.sync();   // the last access to another CTA's memory is behind it
    for (int q = 0; q < team.r; ++q) to += sh.stay[q];
  }
#pragma unroll 2
  for (int i0 = from, k = 0; i0 < until; i0 += 32, ++k) {
    const uint32_t bits = k < 32 ? __shfl_sync(0xffffffffu, answers, k) : __ballot_sync(0xffffffffu, stays(i0 + lane));
    const uint32_t at = to + __popc(bits & ((1u << lane) - 1u));
    if ((bits >> lane & 1u) && (HELD || at < (uint32_t)p.keep)) kept[at] = i0 + lane;
    to += __popc(bits);
  }
}

// grid (C x kv heads, requests); the C CTAs of a row are a cluster.
template <bool CLUSTER>
__global__ void __launch_bounds__(SEL_THREADS) evict_select_kernel(const __grid_constant__ EvictParams p, int C) {
  extern __shared__ uint32_t held[];          // the orders of the part's weights, where they fit
  __shared__ SelectShared sh;
  grid_dependency_wait();
  launch_dependents();
  const Team<CLUSTER> team{CLUSTER ? C : 1, CLUSTER ? (int)blockIdx.x % C : 0};
  const int hk = (int)blockIdx.x / team.C, b = blockIdx.y, t = threadIdx.x;
  const size_t head = (size_t)b * p.H_kv + hk;
  const float *const w = p.weights + head * p.weights_stride;
  int32_t *const kept = p.kept + head * p.keep;
  float *const out = p.new_weights + head * p.new_stride;
  // where the part begins at slot 0 whatever the length, its first weights are requested before that is known: their slots exist
  const int most = p.max_pages * PAGE;
  float x[SEL_AHEAD];
  if (!CLUSTER) {
#pragma unroll
    for (int u = 0; u < SEL_AHEAD; ++u) x[u] = t + u * SEL_THREADS < most ? w[t + u * SEL_THREADS] : 0.0f;
  }
  const int n = p.length(b), count = min(n, p.keep);
  const int part = (n + team.C - 1) / team.C, begin = min(team.r * part, n), end = min(begin + part, n);
  reinterpret_cast<uint4 *>(sh.hist)[t] = make_uint4(0u, 0u, 0u, 0u);
  if (hk == 0 && team.r == 0 && t == 0) p.new_lens[b] = count;
  for (size_t i = (size_t)count + team.r * SEL_THREADS + t; i < p.new_stride; i += (size_t)team.C * SEL_THREADS) out[i] = 0.0f;
  for (int i = count + team.r * SEL_THREADS + t; i < p.keep; i += team.C * SEL_THREADS) kept[i] = -1;
  if (n <= p.keep) {
    for (int i = begin + t; i < end; i += SEL_THREADS) kept[i] = i;
  } else if (part <= SEL_CACHE) {
    __syncthreads();
#pragma unroll 1
    for (int i0 = begin + t;;) {
      if (CLUSTER) {
#pragma unroll
        for (int u = 0; u < SEL_AHEAD; ++u) x[u] = i0 + u * SEL_THREADS < end ? w[i0 + u * SEL_THREADS] : 0.0f;
      }
#pragma unroll
      for (int u = 0; u < SEL_AHEAD; ++u) {
        const int i = i0 + u * SEL_THREADS;
        if (i < end) {
          const uint32_t o = order_of(x[u]);
          held[i - begin] = o;
          if (i >= p.sinks && i < n - p.recent) atomicAdd(&sh.hist[o >> (32 - DIGIT)], 1u);
        }
      }
      i0 += SEL_AHEAD * SEL_THREADS;
      if (i0 >= end) break;
      if (!CLUSTER) {
#pragma unroll
        for (int u = 0; u < SEL_AHEAD; ++u) x[u] = i0 + u * SEL_THREADS < n ? w[i0 + u * SEL_THREADS] : 0.0f;
      }
    }
    __syncthreads();
    select_tokens<CLUSTER, true>(p, team, held, w, n, begin, end, kept, sh);
  } else {
    select_tokens<CLUSTER, false>(p, team, held, w, n, begin, end, kept, sh);
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
  int from = at < p.keep ? p.kept[((size_t)b * p.H_kv + hk) * p.keep + at] : -1;   // -1 past the last token
  const int n = p.length(b), count = min(n, p.keep);
  if (page * PAGE >= count) return;
  if (from >= n) from = -1;   // not written by a selection whose weights changed (select_tokens): what was there before
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
      !aligned(weights, 4) || !aligned(new_weights, 4) || !aligned(page_table, 4) || !aligned(seq_lens, 4) || !aligned(new_table, 4) ||
      !aligned(kept, 4) || !aligned(new_lens, 4))
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
  // CTAs to a row.  One up to SEL_ALONE slots, more where an SM is free for each of them (two to an SM lose more than they gain, and clusters of
  // eight leave SMs of a GPC over) and they have SEL_PART slots each; of a part of the device the driver says what fits.  One request, 32:8 heads,
  // one CTA / as many as the rule says (us): 9000 slots 14.3 / 16.7 with two, 16384 18.8 / 18.8 with four, 32768 29.4 / 20.1, 65536 81.8 / 23.2,
  // 131072 164 / 30.5; two of 20000 23.1 / 20.4 with four, 29.4 with eight; four of 32768 67.4 / 59.2 with four, 83.2 with eight; eight of
  // 65536 115 / 65.3 with two, 75.9 with four; sixteen of 16384 62.9 / 78.1 with two.
  const int most = max_pages_per_req * PAGE;   // no request is longer
  int C = SEL_CLUSTER;
  while (C > 1 && (most <= SEL_ALONE || most < C * SEL_PART || (C < 8 ? (int64_t)heads * C > n_sm : (int64_t)heads * C * 3 > 2 * n_sm))) C /= 2;
  const auto bytes = [&](int c) {
    const int part = (most + c - 1) / c;
    return (size_t)(part <= SEL_CACHE ? part : SEL_CACHE) * sizeof(uint32_t);
  };
  // What the kernel is allowed is the most that any call needs, since it holds for all of them: set to this call's own size, it would lower what
  // another host thread has just set for a longer row, whose launch would be refused.
  const auto grid = [&](int c) { return Grid(dim3((unsigned)(c * p.H_kv), (unsigned)B), (unsigned)c); };
  if (C > 1) {
    if ((rc = allow_smem<evict_select_kernel<true>>(SEL_CACHE * sizeof(uint32_t))) != MPFA_OK) return rc;
    while (C > 1 && max_active_clusters(evict_select_kernel<true>, grid(C), dim3(SEL_THREADS), bytes(C), s) < 1) C /= 2;
  }
  if (C > 1) {
    MPFA_CUDA_OK(launch(evict_select_kernel<true>, grid(C), dim3(SEL_THREADS), bytes(C), s, p, C));
  } else {
    if ((rc = allow_smem<evict_select_kernel<false>>(SEL_CACHE * sizeof(uint32_t))) != MPFA_OK) return rc;
    MPFA_CUDA_OK(launch(evict_select_kernel<false>, grid(1), dim3(SEL_THREADS), bytes(1), s, p, 1));
  }
  const int pages = (keep + PAGE - 1) / PAGE;
  MPFA_CUDA_OK(launch(evict_move_kernel, dim3((unsigned)(pages < max_pages_per_req ? pages : max_pages_per_req), (unsigned)p.H_kv, (unsigned)B),
                      dim3(MOVE_THREADS), 0, s, p));
  return MPFA_OK;
}
