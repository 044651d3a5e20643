// Eviction from a paged cache: the rows to keep by accumulated weight (a radix selection per
// request), and the moves that close the gaps.
#include "budget.h"
#include "common.cuh"

namespace seer {
namespace {

// ------------------------------------------------------------------ the choice
// The K first rows in the order (recent, sink, mass, lower row) stay.  A row's place in it is a
// 32-bit key: the mass as an ordered integer below the three values that NaN, sinks and recent
// rows take.  The K-th largest key is found 11, 11 and 10 bits at a time by histograms, the
// rows equal to it that stay are the lowest, and two counts over the rows number the moves.
// A CTA takes a request, or a cluster of CTAs a long one, each a stretch of its rows, whose keys stay
// in shared memory across the passes (from the matrices again where they do not fit).  In a cluster
// the CTAs add their histograms' filled bins to the first one's, which finds the bin and tells the
// others (all reading all: 5 us a pass of 16 CTAs).  Sums of integers: the order of the atomics
// leaves no trace.  Bound by latency: two loads, three passes of a barrier or two each, the two
// counts, and 20 KB of instructions.  64 requests of 200 to 8000 rows 7.7 to 8.8 us, one of 120000
// 12.4 to 13.5.
constexpr int kSelThreads = 1024;
constexpr int kSelWarps = kSelThreads / 32;
constexpr int kSelKeys = 16384;             // keys of a CTA in shared memory
constexpr int kBins = 2048;
constexpr long kRankRows = 8192;            // of a request per CTA, while the GPU has room for more CTAs
constexpr int kMostRanks = 16;
constexpr int kAhead = 8;                   // rows of a thread whose loads are under way
constexpr uint32_t kKeyRecent = 0xffffffffu, kKeySink = 0xfffffffeu, kKeyNan = 0xfffffffdu;

struct SelShared {
  unsigned hist[3][kBins];                  // of this CTA; the first one's become the cluster's
  uint4 totals[kMostRanks];                 // per CTA: rows above / at the key before K, above / at it behind
  uint4 counts[kSelWarps];                  // the same per warp of this CTA
  unsigned warp_sum[kSelWarps];
  unsigned found_bin, found_above, found_all;   // found_all: every row of the bin stays
  uint32_t keys[kSelKeys];
};

__device__ __forceinline__ void add_cluster(uint32_t addr, unsigned v) {
  asm volatile("red.relaxed.cluster.shared::cluster.add.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
__device__ __forceinline__ void st_cluster(uint32_t addr, unsigned v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
__device__ __forceinline__ void st_cluster4(uint32_t addr, uint4 v) {
  asm volatile("st.shared::cluster.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
template <int RANKS>
__device__ __forceinline__ void sync_ranks() {
  if constexpr (RANKS > 1) cluster_sync();
  else __syncthreads();
}

__device__ __forceinline__ uint32_t mass_key(float m) {
  if (m != m) return kKeyNan;
  const uint32_t u = __float_as_uint(m + 0.f);            // -0 and 0 are one value
  return u ^ ((u >> 31) != 0 ? 0xffffffffu : 0x80000000u);
}

template <int RANKS>
__global__ void __launch_bounds__(kSelThreads) evict_select_kernel(const SelectArgs a) {
  extern __shared__ __align__(16) uint8_t smem[];
  SelShared& sh = *reinterpret_cast<SelShared*>(smem);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  for (int i = tid; i < 3 * kBins; i += kSelThreads) (&sh.hist[0][0])[i] = 0;
  pdl_enter();
  const int b = blockIdx.x / RANKS, rank = blockIdx.x % RANKS;
  const int L0 = a.kv_len[b], budget = a.budget[b], gone = a.gone ? a.gone[b] : 0;
  sync_ranks<RANKS>();                      // every CTA's histograms are zero, and the lengths read before one writes
  const bool sound = L0 >= 0 && L0 <= a.ld_mass && budget >= 0;
  const int L = sound ? L0 : 0, K = sound ? min(budget, L) : 0;
  const bool good = sound && min(K, L - K) <= a.ld_move;
  if (!good || K == L || K == 0) {          // nothing to choose
    if (rank == 0 && tid == 0) {
      if (!good) record_error(a.err, sound ? kErrCapacity : kErrLayout);
      a.len_out[b] = good ? K : L0;
      a.gone_out[b] = gone + (good ? L - K : 0);
      a.n_moves[b] = 0;
    }
    return;
  }
  const long long young = static_cast<long long>(L) + gone - min(a.recent, K);
  // rank's rows [r0, r1), a warp's [w0, w1) of them: both multiples of 32 from their starts
  const int share = ((L + RANKS - 1) / RANKS + 31) / 32 * 32;
  const int r0 = static_cast<int>(min(static_cast<long long>(L), static_cast<long long>(share) * rank));
  const int r1 = static_cast<int>(min(static_cast<long long>(L), static_cast<long long>(r0) + share));
  const bool held = r1 - r0 <= kSelKeys;
  const float* mass = a.mass + static_cast<size_t>(b) * a.ld_mass;
  const int* birth = a.birth + static_cast<size_t>(b) * a.ld_mass;
  const auto row_key = [&](int born, float m) { return born >= young ? kKeyRecent : (born < a.sinks ? kKeySink : mass_key(m)); };
  const auto key_of = [&](int t) { return held ? sh.keys[t - r0] : row_key(birth[t], mass[t]); };

  // ---- the K-th largest key
  uint32_t prefix = 0;
  unsigned need = K;                        // rows with the prefix that stay
#pragma unroll 1
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0), bins = pass == 2 ? kBins / 2 : kBins;
    unsigned* hist = sh.hist[pass];
    if (pass == 0) {
#pragma unroll 1
      for (unsigned t0 = r0 + tid; t0 < static_cast<unsigned>(r1); t0 += kAhead * kSelThreads) {   // (may pass 2^31)
        int born[kAhead];
        float m[kAhead];
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {  // all loads first
          const unsigned t = min(t0 + e * kSelThreads, r1 - 1u);
          born[e] = birth[t];
          m[e] = mass[t];
        }
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
          const unsigned t = t0 + e * kSelThreads;
          const uint32_t k = row_key(born[e], m[e]);
          if (t < static_cast<unsigned>(r1)) {
            if (held) sh.keys[t - r0] = k;
            atomicAdd(&hist[k >> 21], 1u);
          }
        }
      }
    } else {
      const int above = pass == 1 ? 21 : 10;
#pragma unroll 2
      for (int t = r0 + tid; t < r1; t += kSelThreads) {
        const uint32_t k = key_of(t);
        if ((k >> above) == (prefix >> above)) atomicAdd(&hist[(k >> shift) & (bins - 1)], 1u);
      }
    }
    if (RANKS > 1) {
      __syncthreads();
      if (rank != 0)
        for (int i = tid; i < bins; i += kSelThreads) {
          const unsigned v = hist[i];
          if (v != 0) add_cluster(cluster_addr(hist + i, 0), v);
        }
    }
    sync_ranks<RANKS>();
    if (rank == 0) {
      // thread i owns the bins 2 i and 2 i + 1 counted from the top
      const int low = bins - 2 - 2 * tid;
      uint2 own = make_uint2(0, 0);
      if (low >= 0) own = *reinterpret_cast<const uint2*>(hist + low);
      const unsigned sum = own.x + own.y;
      unsigned inc = sum;
#pragma unroll
      for (int off = 1; off < 32; off <<= 1) {
        const unsigned v = __shfl_up_sync(0xffffffffu, inc, off);
        if (lane >= off) inc += v;
      }
      if (lane == 31) sh.warp_sum[warp] = inc;
      __syncthreads();
      unsigned before = inc - sum + __reduce_add_sync(0xffffffffu, lane < warp ? sh.warp_sum[lane] : 0u);
      if (before < need && need <= before + sum) {         // one thread's bins
        const bool upper = need <= before + own.y;
        const unsigned bin = low + upper, over = upper ? before : before + own.y;
        const unsigned whole = need - over == (upper ? own.y : own.x);
        if (RANKS == 1) {
          sh.found_bin = bin;
          sh.found_above = over;
          sh.found_all = whole;
        } else {
          for (int r = 0; r < RANKS; ++r) {
            st_cluster(cluster_addr(&sh.found_bin, r), bin);
            st_cluster(cluster_addr(&sh.found_above, r), over);
            st_cluster(cluster_addr(&sh.found_all, r), whole);
          }
        }
      }
    }
    sync_ranks<RANKS>();
    prefix |= sh.found_bin << shift;
    need -= sh.found_above;
    if (sh.found_all != 0) {                // often after two passes: the keys from the bin's first on stay
      prefix -= 1;                          // (not 0, or all rows would)
      need = 0;
      break;
    }
    // (the next found is written behind a barrier that every thread reaches after this)
  }

  // ---- counts per warp: rows above the key and at it, before row K and behind
  const int wshare = (share / 32 + kSelWarps - 1) / kSelWarps * 32;
  const int w0 = static_cast<int>(min(static_cast<long long>(r1), r0 + static_cast<long long>(warp) * wshare));
  const int w1 = static_cast<int>(min(static_cast<long long>(r1), static_cast<long long>(w0) + wshare));
  uint4 n = make_uint4(0, 0, 0, 0);
#pragma unroll 2
  for (int t = w0 + lane; t - lane < w1; t += 32) {
    const uint32_t k = t < w1 ? key_of(t) : 0;
    const bool over = t < w1 && k > prefix, at = t < w1 && k == prefix;
    const unsigned first = __ballot_sync(0xffffffffu, t < K);
    const unsigned m = __ballot_sync(0xffffffffu, over), e = __ballot_sync(0xffffffffu, at);
    n.x += __popc(m & first);
    n.y += __popc(e & first);
    n.z += __popc(m & ~first);
    n.w += __popc(e & ~first);
  }
  if (lane == 0) sh.counts[warp] = n;
  __syncthreads();
  // of all warps before this one, and of the whole CTA
  uint4 c = sh.counts[lane], all;
  all.x = __reduce_add_sync(0xffffffffu, c.x);
  all.y = __reduce_add_sync(0xffffffffu, c.y);
  all.z = __reduce_add_sync(0xffffffffu, c.z);
  all.w = __reduce_add_sync(0xffffffffu, c.w);
  unsigned above = __reduce_add_sync(0xffffffffu, lane < warp ? c.x + c.z : 0u);
  unsigned equal = __reduce_add_sync(0xffffffffu, lane < warp ? c.y + c.w : 0u);
  unsigned above_k = all.x, equal_k = all.y;
  if (RANKS > 1) {
    if (tid < RANKS) st_cluster4(cluster_addr(&sh.totals[rank], tid), all);
    cluster_sync();                         // nobody touches another CTA's memory from here on
    c = lane < RANKS ? sh.totals[lane & (kMostRanks - 1)] : make_uint4(0, 0, 0, 0);
    above_k = __reduce_add_sync(0xffffffffu, c.x);
    equal_k = __reduce_add_sync(0xffffffffu, c.y);
    above += __reduce_add_sync(0xffffffffu, lane < rank ? c.x + c.z : 0u);
    equal += __reduce_add_sync(0xffffffffu, lane < rank ? c.y + c.w : 0u);
  }
  const unsigned kept_k = above_k + min(need, equal_k);    // rows before K that stay
  if (rank == 0 && tid == 0) {
    a.len_out[b] = K;
    a.gone_out[b] = gone + (L - K);
    a.n_moves[b] = K - static_cast<int>(kept_k);
  }

  // ---- the moves: place i of the holes before K, row i of the kept behind
  int* from = a.move_from + static_cast<size_t>(b) * a.ld_move;
  int* to = a.move_to + static_cast<size_t>(b) * a.ld_move;
#pragma unroll 2
  for (int t = w0 + lane; t - lane < w1; t += 32) {
    const uint32_t k = t < w1 ? key_of(t) : 0;
    const bool over = t < w1 && k > prefix, at = t < w1 && k == prefix;
    const unsigned m = __ballot_sync(0xffffffffu, over), e = __ballot_sync(0xffffffffu, at);
    const unsigned less = (1u << lane) - 1;
    const unsigned ties = equal + __popc(e & less);
    const unsigned kept = above + __popc(m & less) + min(ties, need);   // rows before t that stay
    const bool keep = over || (at && ties < need);
    if (t < w1) {
      if (t < K && !keep) to[t - kept] = t;
      if (t >= K && keep) from[kept - kept_k] = t;
    }
    above += __popc(m);
    equal += __popc(e);
  }
}

// ------------------------------------------------------------------ the moves
// Row move_from of a request becomes its row move_to; sources and places are apart, so all
// moves go at once.  Bound by HBM behind a chain of loads (counts, lists, pages, rows): each moved
// row is read once and written once.  All requests' moves form one line; a warp takes 2 KB of a row
// at a time, its loads ahead of its stores.  6.7k rows of 4 KB, 55 MB, 13 us; 64 rows 3.6.  (1 or 4 KB
// a warp and 32 registers: the same; two pieces a warp at once 18 us, the next piece's places
// looked up meanwhile 15: both cost warps.)
constexpr int kEvictThreads = 256;
constexpr int kSeg = 2048;

__global__ void __launch_bounds__(kEvictThreads) kv_evict_kernel(const EvictArgs a) {
  extern __shared__ int first[];            // [B + 1] a request's first move on the line, cut at 2^31 - 1
  __shared__ long long warp_sum[kEvictThreads / 32];
  pdl_enter();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const auto moves_of = [&](int b, bool report) {
    const int n = a.n_moves[b];
    if (n >= 0 && n <= a.ld_move) return n;
    if (report) record_error(a.err, kErrLayout);
    return 0;
  };
  long long sum = 0;
  for (int b0 = 0; b0 < a.B; b0 += kEvictThreads) {
    const int b = b0 + tid;
    const long long v = b < a.B ? moves_of(b, blockIdx.x == 0) : 0;
    long long inc = v;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const long long x = __shfl_up_sync(0xffffffffu, inc, off);
      if (lane >= off) inc += x;
    }
    if (lane == 31) warp_sum[warp] = inc;
    __syncthreads();
    long long before = sum, all = 0;
    for (int w = 0; w < kEvictThreads / 32; ++w) {
      if (w < warp) before += warp_sum[w];
      all += warp_sum[w];
    }
    if (b < a.B) first[b] = static_cast<int>(min(before + inc - v, 0x7fffffffll));
    sum += all;
    __syncthreads();
  }
  if (tid == 0) first[a.B] = static_cast<int>(min(sum, 0x7fffffffll));
  __syncthreads();

  const int segs = (a.row_bytes + kSeg - 1) / kSeg;
  const long long total = static_cast<long long>(first[a.B]) * segs, step = static_cast<long long>(gridDim.x) * (kEvictThreads / 32);
  for (long long x = static_cast<long long>(blockIdx.x) * (kEvictThreads / 32) + warp; x < total; x += step) {
    const int move = static_cast<int>(x / segs), seg = static_cast<int>(x - static_cast<long long>(move) * segs);
    int lo = 0, hi = a.B;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (first[mid] <= move) lo = mid; else hi = mid;
    }
    const size_t at = static_cast<size_t>(lo) * a.ld_move + (move - first[lo]);
    const int t[2] = {a.move_from[at], a.move_to[at]};
    const long long room = min(static_cast<long long>(a.pages.max_pages) << a.pages.page_shift,
                               a.kv_len ? static_cast<long long>(a.kv_len[lo]) : 0x7fffffffll);
    size_t row[2];
    bool good = true;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      int page = -1;
      if (t[e] >= 0 && t[e] < room && (t[e] < a.ld_mass || (!a.mass && !a.birth)))
        page = a.pages.table[static_cast<size_t>(lo) * a.pages.max_pages + (t[e] >> a.pages.page_shift)];
      if (page < 0 || page >= a.pages.n_pages) good = false;
      row[e] = (static_cast<size_t>(page) << a.pages.page_shift) + (t[e] & ((1 << a.pages.page_shift) - 1));
    }
    if (!good) {
      if (lane == 0) record_error(a.err, kErrLayout);
      continue;
    }
    uint8_t* kv = static_cast<uint8_t*>(a.pages.kv);
    const int begin = seg * kSeg + lane * 16;
    uint4 w[kSeg / 512];
#pragma unroll
    for (int e = 0; e < kSeg / 512; ++e)
      if (begin + e * 512 < a.row_bytes) w[e] = *reinterpret_cast<const uint4*>(kv + row[0] * a.row_bytes + begin + e * 512);
#pragma unroll
    for (int e = 0; e < kSeg / 512; ++e)
      if (begin + e * 512 < a.row_bytes) *reinterpret_cast<uint4*>(kv + row[1] * a.row_bytes + begin + e * 512) = w[e];
    if (seg == 0 && lane == 0) {
      const size_t base = static_cast<size_t>(lo) * a.ld_mass;
      if (a.mass) a.mass[base + t[1]] = a.mass[base + t[0]];
      if (a.birth) a.birth[base + t[1]] = a.birth[base + t[0]];
    }
  }
}

template <int RANKS>
cudaError_t launch_ranks(const SelectArgs& a, cudaStream_t st) {
  static bool attr_set[64] = {};
  if (RANKS > 8) {
    const cudaError_t e = cudaFuncSetAttribute(evict_select_kernel<RANKS>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
  }
  const cudaError_t e = set_smem_limit_once(evict_select_kernel<RANKS>, static_cast<int>(sizeof(SelShared)), attr_set);
  if (e != cudaSuccess) return e;
  return launch_kernel_overlap(launch_overlap_enabled(), RANKS, evict_select_kernel<RANKS>, dim3(a.B * RANKS), dim3(kSelThreads),
                               sizeof(SelShared), st, a);
}

}  // namespace

cudaError_t launch_evict_select(const SelectArgs& a, int num_sms, cudaStream_t st) {
  // CTAs of a request: as many as its longest row count gives work, and the GPU has room for
  int ranks = 1;
  while (ranks < kMostRanks && a.ld_mass > kRankRows * ranks && a.B * ranks < 2 * num_sms) ranks *= 2;
  switch (ranks) {
    case 1: return launch_ranks<1>(a, st);
    case 2: return launch_ranks<2>(a, st);
    case 4: return launch_ranks<4>(a, st);
    case 8: return launch_ranks<8>(a, st);
    default: return launch_ranks<16>(a, st);
  }
}

cudaError_t launch_kv_evict(const EvictArgs& a, int num_sms, cudaStream_t st) {
  if (a.B > kPageTableMaxB) return cudaErrorInvalidValue;
  const int smem = (a.B + 1) * static_cast<int>(sizeof(int));
  if (smem > 46 * 1024) {
    static bool attr_set[64] = {};
    const cudaError_t e = set_smem_limit_once(kv_evict_kernel, (kPageTableMaxB + 1) * static_cast<int>(sizeof(int)), attr_set);
    if (e != cudaSuccess) return e;
  }
  const long long segs = (a.row_bytes + kSeg - 1) / kSeg;
  const long long work = (static_cast<long long>(a.B) * a.ld_move * segs + kEvictThreads / 32 - 1) / (kEvictThreads / 32);
  const long long most = 8ll * num_sms;
  return launch_kernel(kv_evict_kernel, dim3(static_cast<unsigned>(work < 1 ? 1 : (work < most ? work : most))), dim3(kEvictThreads), smem, st, a);
}

}  // namespace seer
