// Kernels of the paged K/V cache: page tables and slots from request lengths,
// storing rotated rows at their slots, keeping the accepted rows of a draft.
#include "common.cuh"
#include "paged.h"

namespace seer {
namespace {

// ------------------------------------------------------------------ page tables
// Integer prefix sums over the requests and one division by the page size a row.
// Bound by latency (launch, two dependent loads, the scan): 8 B + 4 bytes a page + 8 to
// 20 bytes a row is little.  Every block repeats the scan of the whole batch, so that
// rows need no second launch; rows then spread over the grid and find their request by
// bisection in shared memory.  8 requests of one row 2.6 us, 256 prompts (93k rows) 4.9.
constexpr int kTableThreads = 256;

// Exclusive prefix of v over the block's threads, and the block's total; two values at once.
struct Pair64 {
  long long a, b;
};
__device__ __forceinline__ Pair64 block_scan(Pair64 v, Pair64* warp_sums, Pair64& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  Pair64 inc = v;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const long long a = __shfl_up_sync(0xffffffffu, inc.a, off), b = __shfl_up_sync(0xffffffffu, inc.b, off);
    if (lane >= off) {
      inc.a += a;
      inc.b += b;
    }
  }
  if (lane == 31) warp_sums[warp] = inc;
  __syncthreads();
  Pair64 before{0, 0};
  total = Pair64{0, 0};
#pragma unroll
  for (int w = 0; w < kTableThreads / 32; ++w) {
    const Pair64 s = warp_sums[w];
    if (w < warp) {
      before.a += s.a;
      before.b += s.b;
    }
    total.a += s.a;
    total.b += s.b;
  }
  __syncthreads();
  return Pair64{before.a + inc.a - v.a, before.b + inc.b - v.b};
}

// A request's counts after the checks that keep every later index in range.
struct Request {
  int cached, fresh, old_pages, pages, kv_len;
};
__device__ __forceinline__ Request read_request(const PageTableArgs& a, int b, bool report) {
  Request r;
  int c = a.cached[b], n = a.fresh[b];
  if (c < 0 || n < 0) {
    if (report) record_error(a.err, kErrLayout);
    c = max(c, 0);
    n = max(n, 0);
  }
  const long long room = min(static_cast<long long>(a.max_pages) << a.page_shift, static_cast<long long>(kMaxKeys));
  const long long total = static_cast<long long>(c) + n;
  if (total > room && report) record_error(a.err, kErrCapacity);
  if (n > kMaxDraft && (a.parent || a.mask) && report) record_error(a.err, kErrLayout);
  const int up = (1 << a.page_shift) - 1;
  r.cached = c;
  r.fresh = n;
  r.kv_len = static_cast<int>(total < room ? total : room);
  r.pages = (static_cast<long long>(r.kv_len) + up) >> a.page_shift;
  r.old_pages = min(static_cast<int>((static_cast<long long>(c) + up) >> a.page_shift), r.pages);
  return r;
}

__device__ __forceinline__ int checked_page(const PageTableArgs& a, int page, int code, bool report) {
  if (page >= 0 && page < a.n_pages) return page;
  if (report) record_error(a.err, code);
  return -1;
}
// The i-th page taken from the free list, or -1 when the list ends before it.
__device__ __forceinline__ int free_page(const PageTableArgs& a, long long i, bool report) {
  if (i < 0 || i >= a.n_free) {
    if (report) record_error(a.err, kErrCapacity);
    return -1;
  }
  return checked_page(a, a.free_pages[i], kErrLayout, report);
}

__global__ void __launch_bounds__(kTableThreads) page_tables_kernel(const PageTableArgs a) {
  pdl_enter();
  extern __shared__ int sh[];
  int* cu = sh;                    // [B + 1] first new row of each request, cut at 2^31 - 1
  int* first = sh + a.B + 1;       // [B] index of its first taken page in the free list, cut likewise
  __shared__ Pair64 warp_sums[kTableThreads / 32];
  const bool lead = blockIdx.x == 0;
  const long long limit = 0x7fffffff;
  Pair64 sum{0, *a.head};
  for (int b0 = 0; b0 < a.B; b0 += kTableThreads) {
    const int b = b0 + threadIdx.x;
    Request r{};
    if (b < a.B) r = read_request(a, b, lead);
    Pair64 total;
    const Pair64 at = block_scan(Pair64{r.fresh, r.pages - r.old_pages}, warp_sums, total);
    if (b < a.B) {
      cu[b] = static_cast<int>(min(sum.a + at.a, limit));
      first[b] = static_cast<int>(min(sum.b + at.b, limit));
      if (lead) {
        a.cu[b] = cu[b];
        a.kv_len[b] = r.kv_len;
      }
    }
    sum.a += total.a;
    sum.b += total.b;
  }
  if (threadIdx.x == 0) {
    cu[a.B] = static_cast<int>(min(sum.a, limit));
    if (lead) {
      a.cu[a.B] = cu[a.B];
      *a.head_out = static_cast<int>(min(sum.b, limit));
      if (sum.a > a.T_cap) record_error(a.err, kErrRows);
    }
  }
  __syncthreads();

  // table entries: a warp per request
  const int lane = threadIdx.x & 31;
  for (int b = (blockIdx.x * kTableThreads + threadIdx.x) >> 5; b < a.B; b += gridDim.x * (kTableThreads / 32)) {
    const Request r = read_request(a, b, false);
    int* row = a.table + static_cast<size_t>(b) * a.max_pages;
    for (int i = r.old_pages + lane; i < r.pages; i += 32)
      row[i] = free_page(a, static_cast<long long>(first[b]) + (i - r.old_pages), true);
  }

  // rows: a thread each
  const int rows = min(cu[a.B], a.T_cap), page_rows = 1 << a.page_shift;
  for (int row = blockIdx.x * kTableThreads + threadIdx.x; row < rows; row += gridDim.x * kTableThreads) {
    int lo = 0, hi = a.B;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (cu[mid] <= row) lo = mid; else hi = mid;
    }
    const Request r = read_request(a, lo, false);
    const int i = row - cu[lo];
    const long long at = static_cast<long long>(r.cached) + i;
    const long long page_index = at >> a.page_shift;
    int page = -1;                 // a row past the request's room has no slot
    // entries that were there are read from the table, new ones from the free list: other
    // blocks may not have written them yet
    if (at < r.kv_len) {
      if (page_index < r.old_pages)
        page = checked_page(a, a.table[static_cast<size_t>(lo) * a.max_pages + page_index], kErrLayout, true);
      else
        page = free_page(a, first[lo] + page_index - r.old_pages, false);
    }
    a.slot[row] = page < 0 ? -1 : page * page_rows + static_cast<int>(at & (page_rows - 1));
    int depth = i;
    uint64_t bits = 0;
    if (r.fresh <= kMaxDraft) {
      if (a.parent) {
        int node = i;
        depth = -1;
        while (node >= 0) {        // a parent is an earlier row, so the walk ends
          bits |= 1ull << node;
          ++depth;
          const int up = a.parent[cu[lo] + node];
          if (up < -1 || up >= node) {
            record_error(a.err, kErrLayout);
            break;
          }
          node = up;
        }
      } else {
        bits = i == 63 ? ~0ull : (2ull << i) - 1;
      }
    }
    a.position[row] = static_cast<int>(min(r.cached + static_cast<long long>(depth), limit));
    if (a.mask) a.mask[row] = bits;
  }
}

// ------------------------------------------------------------------ rotated rows into the cache
template <int T>
struct Vec16;                      // 16 bytes of a storage type as floats
template <>
struct Vec16<kF32> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void unpack(uint4 w, float (&f)[4]) {
    f[0] = __uint_as_float(w.x);
    f[1] = __uint_as_float(w.y);
    f[2] = __uint_as_float(w.z);
    f[3] = __uint_as_float(w.w);
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[4]) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
};
template <bool F16>
struct Vec16Half {
  static constexpr int N = 8;
  static __device__ __forceinline__ void unpack(uint4 w, float (&f)[8]) {
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = lo16(v[i], F16);
      f[2 * i + 1] = hi16(v[i], F16);
    }
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[8]) {
    return make_uint4(pack2(f[0], f[1], F16), pack2(f[2], f[3], F16), pack2(f[4], f[5], F16), pack2(f[6], f[7], F16));
  }
};
template <>
struct Vec16<kBF16> : Vec16Half<false> {};
template <>
struct Vec16<kF16> : Vec16Half<true> {};

constexpr int kAppendThreads = 256;
constexpr int kAppendRows = 4;

// (x_i, x_{i + dh/2}) turns by position * theta^(-2i/dh).  The angle is taken in turns as
// position * rate modulo 1 in 64-bit integers (rate = theta^(-2i/dh) / 2 pi, from the host in
// fp64: off by at most 3.4 2^-53 of itself, which the position multiplies); the product is
// exact, and its fraction goes to sincospif.
// One pass: q, k and v are read once, q | k written to `rotated`, k | v to the cache row.
// Bound by HBM.  A block takes up to four rows, so that their sines are one a thread, and a
// thread UNROLL of their items (16 bytes of a head's lower half and the 16 of its upper half),
// loads ahead of the stores.  Sines and cosines lie in groups of four, the groups of
// neighbouring lanes side by side (pair by pair they met 8 times in a bank).  17.9k rows of
// 32 + 8 + 8 heads of 128, 479 MB, 73 us (6.5 TB/s; one item a thread at a time 88); 64 rows 2.9.
template <int T, bool ROTATE>
__global__ void __launch_bounds__(kAppendThreads) kv_append_kernel(const KvAppendArgs a, const __grid_constant__ TurnRates rates) {
  pdl_enter();
  using V = Vec16<T>;
  constexpr int QUADS = V::N / 4, UNROLL = 3, es = 16 / V::N;
  __shared__ float4 cosines[kAppendRows][QUADS][64 / V::N], sines[kAppendRows][QUADS][64 / V::N];
  __shared__ int slots[kAppendRows];
  const int dh = a.pages.head_dim, half = dh / 2, n_kv = a.pages.n_kv;
  int M = a.M_dev ? *a.M_dev : a.T_cap;
  if (M < 0 || M > a.T_cap) {
    if (blockIdx.x == 0 && threadIdx.x == 0) record_error(a.err, kErrRows);
    M = M < 0 ? 0 : a.T_cap;
  }
  const int pool_rows = a.pages.n_pages << a.pages.page_shift;
  const int per_head = half / V::N;               // items of a head
  const int items = (a.n_heads + 2 * n_kv) * per_head;
  const long kv_row = 2l * n_kv * dh * es, high = static_cast<long>(half) * es;
  const int G = a.rows_per_block;
  for (int row0 = blockIdx.x * G; row0 < M; row0 += gridDim.x * G) {
    const int rows = min(G, M - row0);
    __syncthreads();                              // the rows before are done with the tables
    if (ROTATE)
      for (int j = threadIdx.x; j < rows * half; j += kAppendThreads) {
        const int r = j / half, i = j - r * half, c = i / V::N, e = i % V::N;
        const uint64_t part = static_cast<uint64_t>(static_cast<int64_t>(a.position[row0 + r])) * rates.rate[i];
        float sn, cs;
        sincospif(static_cast<float>(static_cast<int64_t>(part)) * 0x1p-63f, &sn, &cs);
        reinterpret_cast<float*>(&cosines[r][e / 4][c])[e % 4] = cs;
        reinterpret_cast<float*>(&sines[r][e / 4][c])[e % 4] = sn;
      }
    if (threadIdx.x < rows) {
      int s = a.slot[row0 + threadIdx.x];
      if (s < -1 || s >= pool_rows) {
        record_error(a.err, kErrLayout);
        s = -1;
      }
      slots[threadIdx.x] = s;
    }
    __syncthreads();
    for (int j0 = threadIdx.x; j0 < rows * items; j0 += UNROLL * kAppendThreads) {
      uint4 lo[UNROLL], hi[UNROLL];
      int row[UNROLL], head[UNROLL], chunk[UNROLL];
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) {
        const int j = j0 + u * kAppendThreads;
        row[u] = j / items;
        const int it = j - row[u] * items;
        head[u] = it / per_head;
        chunk[u] = it - head[u] * per_head;
        const bool wanted = row[u] < rows && ((a.rotated && head[u] < a.n_heads + n_kv) || (head[u] >= a.n_heads && slots[row[u]] >= 0));
        if (!wanted) {
          row[u] = -1;
          continue;
        }
        const uint8_t* src = a.qkv + static_cast<size_t>(row0 + row[u]) * a.ld + static_cast<long>(head[u]) * dh * es + chunk[u] * 16;
        lo[u] = *reinterpret_cast<const uint4*>(src);
        hi[u] = *reinterpret_cast<const uint4*>(src + high);
      }
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) {
        if (row[u] < 0) continue;
        const bool turned = head[u] < a.n_heads + n_kv;
        if (ROTATE && turned) {
          float x[V::N], y[V::N];
          V::unpack(lo[u], x);
          V::unpack(hi[u], y);
#pragma unroll
          for (int g = 0; g < QUADS; ++g) {
            const float4 c4 = cosines[row[u]][g][chunk[u]], s4 = sines[row[u]][g][chunk[u]];
            const float cs[4] = {c4.x, c4.y, c4.z, c4.w}, sn[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float p = x[4 * g + e], w = y[4 * g + e];
              x[4 * g + e] = fmaf(p, cs[e], -w * sn[e]);
              y[4 * g + e] = fmaf(w, cs[e], p * sn[e]);
            }
          }
          lo[u] = V::pack(x);
          hi[u] = V::pack(y);
        }
        const long at = static_cast<long>(head[u]) * dh * es + chunk[u] * 16;
        if (turned && a.rotated) {
          uint8_t* rot = a.rotated + static_cast<size_t>(row0 + row[u]) * a.ld_rot + at;
          *reinterpret_cast<uint4*>(rot) = lo[u];
          *reinterpret_cast<uint4*>(rot + high) = hi[u];
        }
        if (head[u] >= a.n_heads && slots[row[u]] >= 0) {   // k | v follow q as they do in the cache row
          uint8_t* dst = static_cast<uint8_t*>(a.pages.kv) + static_cast<size_t>(slots[row[u]]) * kv_row + at -
                         static_cast<long>(a.n_heads) * dh * es;
          *reinterpret_cast<uint4*>(dst) = lo[u];
          *reinterpret_cast<uint4*>(dst + high) = hi[u];
        }
      }
    }
  }
}

// ------------------------------------------------------------------ accepted drafts
// Cache row cached + k of a request becomes its row cached + accepted[k], in ascending k.
// accepted ascends strictly, so accepted[k] >= k and a row is read before a later k could
// overwrite it; a thread moves the same 16 bytes of every row in that order, eight rows'
// loads ahead of their stores.  Latency: a few rows a request (128 requests 2.3 us).
constexpr int kAcceptThreads = 128;

__global__ void __launch_bounds__(kAcceptThreads) kv_accept_kernel(const KvAcceptArgs a) {
  pdl_enter();
  __shared__ int src[kMaxDraft], dst[kMaxDraft];
  const int b = blockIdx.y;
  const int c = a.cached[b];
  int n = a.n_accepted[b];
  bool good = c >= 0 && n >= 0 && n <= a.max_draft && c <= kMaxKeys - n;
  if (!good) n = 0;
  for (int k = threadIdx.x; k < n; k += kAcceptThreads) {
    const int* list = a.accepted + static_cast<size_t>(b) * a.max_draft;
    const int from = list[k], before = k > 0 ? list[k - 1] : -1;
    bool fine = from > before && from < a.max_draft;
    int rows[2] = {-1, -1};
    if (fine)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const long long at = static_cast<long long>(c) + (e == 0 ? from : k);
        const long long page_index = at >> a.pages.page_shift;
        const int page = page_index < a.pages.max_pages ? a.pages.table[static_cast<size_t>(b) * a.pages.max_pages + page_index] : -1;
        if (page < 0 || page >= a.pages.n_pages) fine = false;
        else rows[e] = (page << a.pages.page_shift) + static_cast<int>(at & ((1 << a.pages.page_shift) - 1));
      }
    src[k] = rows[0];
    dst[k] = rows[1];
    good = good && fine;
  }
  // a request with a bad list keeps none of its draft
  if (!__syncthreads_and(good)) {
    if (threadIdx.x == 0 && blockIdx.x == 0) {
      record_error(a.err, kErrLayout);
      a.len_out[b] = c;
    }
    return;
  }
  if (threadIdx.x == 0 && blockIdx.x == 0) a.len_out[b] = c + n;
  const long at = (static_cast<long>(blockIdx.x) * kAcceptThreads + threadIdx.x) * 16;
  if (at >= a.row_bytes) return;
  uint8_t* kv = static_cast<uint8_t*>(a.pages.kv) + at;
  for (int k0 = 0; k0 < n; k0 += 8) {
    uint4 w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (k0 + e < n) w[e] = *reinterpret_cast<const uint4*>(kv + static_cast<size_t>(src[k0 + e]) * a.row_bytes);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (k0 + e < n) *reinterpret_cast<uint4*>(kv + static_cast<size_t>(dst[k0 + e]) * a.row_bytes) = w[e];
  }
}

}  // namespace

cudaError_t launch_page_tables(const PageTableArgs& a, int num_sms, cudaStream_t st) {
  if (a.B > kPageTableMaxB) return cudaErrorInvalidValue;
  const int smem = (2 * a.B + 1) * static_cast<int>(sizeof(int));
  if (smem > 46 * 1024) {
    static bool attr_set[64] = {};
    cudaError_t e = set_smem_limit_once(page_tables_kernel, (2 * kPageTableMaxB + 1) * static_cast<int>(sizeof(int)), attr_set);
    if (e != cudaSuccess) return e;
  }
  const long work = a.T_cap / kTableThreads + a.B / (kTableThreads / 32) + 1l;
  const unsigned blocks = static_cast<unsigned>(work < num_sms ? work : num_sms);
  return launch_kernel(page_tables_kernel, dim3(blocks), dim3(kTableThreads), smem, st, a);
}

cudaError_t launch_kv_append(int type, const KvAppendArgs& args, const TurnRates& rates, bool rotate, int num_sms,
                             cudaStream_t st) {
  if (args.T_cap <= 0) return cudaSuccess;
  KvAppendArgs a = args;
  a.rows_per_block = a.T_cap >= 2 * kAppendRows * num_sms ? kAppendRows : 1;
  const int groups = (a.T_cap + a.rows_per_block - 1) / a.rows_per_block;
  const dim3 grid(groups < 8 * num_sms ? groups : 8 * num_sms);
#define SEER_APPEND(T)                                                                                             \
  if (type == T)                                                                                                   \
    return rotate ? launch_kernel(kv_append_kernel<T, true>, grid, dim3(kAppendThreads), 0, st, a, rates)          \
                  : launch_kernel(kv_append_kernel<T, false>, grid, dim3(kAppendThreads), 0, st, a, rates);
  SEER_APPEND(kF32)
  SEER_APPEND(kBF16)
  SEER_APPEND(kF16)
#undef SEER_APPEND
  return cudaErrorInvalidValue;
}

cudaError_t launch_kv_accept(const KvAcceptArgs& a, cudaStream_t st) {
  if (a.B > 65535) return cudaErrorInvalidValue;
  const int chunks = (a.row_bytes / 16 + kAcceptThreads - 1) / kAcceptThreads;
  return launch_kernel(kv_accept_kernel, dim3(chunks, a.B), dim3(kAcceptThreads), 0, st, a);
}

}  // namespace seer
