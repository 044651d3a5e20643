// Attention weight that cached rows receive: per key the softmax weights of a request's last
// rows, summed over them and over all query heads.
//   mass[t] = keep mass[t] + sum_h sum_i 2^(s_hi(t) - m_hi) / l_hi,  s = q k log2(e) / sqrt(dh),
//   m_hi = max_t s_hi(t),  l_hi = sum_t 2^(s_hi(t) - m_hi).
// A column is one query row of one head.  A softmax's weight needs its whole row first, so the
// keys are gone through twice: for every column's maximum and sum, then for the weights.
#include <math.h>

#include "attn_math.cuh"
#include "budget.h"
#include "common.cuh"

namespace seer {
namespace {

constexpr int kThreads = 256;
constexpr int KEYS = kMassKeys;

// ------------------------------------------------------------------ requests and their key tiles
struct Request {
  int q0, rows;           // its first row of q, and how many the batch gives it
  int n, look, kv;        // new rows, those that look, keys
  bool good;
};
__device__ __forceinline__ Request read_request(const MassArgs& a, int b) {
  Request r{};
  const int q0 = a.cu[b], end = a.cu[b + 1], kv = a.kv_len[b];
  r.good = q0 >= 0 && end >= q0 && end <= a.T_cap;
  const int rows = r.good ? end - q0 : 0;
  const int n = a.accepted ? a.n_accepted[b] : rows;
  r.good = r.good && n >= 0 && n <= rows && (!a.accepted || n <= a.max_draft) && kv >= n && kv <= a.ld_mass && kv <= kMaxKeys &&
           kv <= (static_cast<long long>(a.pages.max_pages) << a.pages.page_shift);
  if (!r.good) return r;
  r.q0 = q0;
  r.rows = rows;
  r.n = n;
  r.look = min(n, a.window);
  r.kv = kv;
  return r;
}
__device__ __forceinline__ int tiles_of(const Request& r) { return (r.kv + KEYS - 1) / KEYS; }

// first[b] = key tiles of the requests before b, first[B] all; by the whole block.  Requests
// past the call's key capacity have no tiles, nor has any behind them.
__device__ __forceinline__ void tile_line(const MassArgs& a, int* first, long long* warp_sum, bool report) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
  long long sum = 0;
  for (int b0 = 0; b0 < a.B; b0 += blockDim.x) {
    const int b = b0 + tid;
    Request r{};
    if (b < a.B) {
      r = read_request(a, b);
      if (!r.good && report) record_error(a.err, kErrLayout);
    }
    const long long v = tiles_of(r);
    long long inc = v;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const long long x = __shfl_up_sync(0xffffffffu, inc, off);
      if (lane >= off) inc += x;
    }
    if (lane == 31) warp_sum[warp] = inc;
    __syncthreads();
    long long before = sum;
    for (int w = 0; w < warps; ++w) {
      if (w < warp) before += warp_sum[w];
      sum += warp_sum[w];
    }
    if (b < a.B) {
      if (before + inc > a.cap_tiles && v > 0 && report) record_error(a.err, kErrCapacity);
      first[b + 1] = static_cast<int>(before + inc > a.cap_tiles ? -1 : before + inc);
    }
    __syncthreads();
  }
  if (tid == 0) first[0] = 0;
  __syncthreads();
  // -1 marks the capacity's end: later requests start and end where the last good one did
  if (first[a.B] < 0) {
    int lo = 0, hi = a.B;                       // first[lo] >= 0, first[hi] < 0
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (first[mid] >= 0) lo = mid; else hi = mid;
    }
    const int end = first[lo];
    __syncthreads();
    for (int b = lo + 1 + tid; b <= a.B; b += blockDim.x) first[b] = end;
    __syncthreads();
  }
}
// The request of place x on the line.
__device__ __forceinline__ int request_at(const int* first, int B, int x) {
  int lo = 0, hi = B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}
// Run c of n over `total` places: [cut(c), cut(c + 1)), and the run that holds x.
__device__ __forceinline__ int cut(long long total, int c, int n) { return static_cast<int>(total * c / n); }
__device__ __forceinline__ int run_of(long long total, long long x, int n) { return static_cast<int>(((x + 1) * n - 1) / total); }

// Row of q of a request's i-th looking row, or -1 (an accepted entry outside the draft).
__device__ __forceinline__ int query_row(const MassArgs& a, const Request& r, int b, int i, bool report) {
  const int k = r.n - r.look + i;
  if (!a.accepted) return r.q0 + k;
  const int e = a.accepted[static_cast<size_t>(b) * a.max_draft + k];
  if (e >= 0 && e < r.rows) return r.q0 + e;
  if (report) record_error(a.err, kErrLayout);
  return -1;
}
// Pool row of key t of request b, or -1.
__device__ __forceinline__ long key_row(const MassArgs& a, int b, int t, bool report) {
  const int page = a.pages.table[static_cast<size_t>(b) * a.pages.max_pages + (t >> a.pages.page_shift)];
  if (page < 0 || page >= a.pages.n_pages) {
    if (report) record_error(a.err, kErrLayout);
    return -1;
  }
  return (static_cast<long>(page) << a.pages.page_shift) + (t & ((1 << a.pages.page_shift) - 1));
}

// (m, l) of two sets of keys; m = -inf: nothing but hidden or -inf scores.
__device__ __forceinline__ float2 join(float2 x, float2 y) {
  const float m = fmaxf(x.x, y.x);
  const float base = m == -INFINITY ? 0.f : m;
  return make_float2(m, x.y * ex2(x.x - base) + y.y * ex2(y.x - base));
}
// (m, 1 / l) as the weights take it: 2^(s - m) / l.
__device__ __forceinline__ float2 finish(float2 x) { return make_float2(x.x == -INFINITY ? 0.f : x.x, 1.f / x.y); }

// Workspace of the general path: per piece of a request's tiles and column (m, l), then per
// request and column (m, 1 / l).
__host__ __device__ inline long columns(const MassArgs& a) { return static_cast<long>(a.n_heads) * a.window; }
__device__ __forceinline__ float2* final_stats(const MassArgs& a) { return static_cast<float2*>(a.ws); }
__device__ __forceinline__ float2* piece_stats(const MassArgs& a) { return final_stats(a) + a.B * columns(a); }

// ------------------------------------------------------------------ the general path
// Scores of one 64-key tile and 16 columns on the CUDA cores: keys and queries of a head in
// shared memory as fp32, a thread 4 columns of one key.
constexpr int COLS = 16;
template <int T>
__device__ __forceinline__ float load1(const void* p, long i) {
  if constexpr (T == kF32) return static_cast<const float*>(p)[i];
  else if constexpr (T == kBF16) return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
  else return __half2float(static_cast<const __half*>(p)[i]);
}
struct TileShared {
  float k[KEYS][132];
  float q[COLS][128];
  int col_row[COLS];                          // new row of a column counted from the first that looks, -1: none
};
template <int T>
__device__ __forceinline__ void load_queries(const MassArgs& a, const Request& r, int b, int kvh, int col0, TileShared& sh) {
  const int dh = a.pages.head_dim, g = a.n_heads / a.pages.n_kv;
  for (int x = threadIdx.x; x < COLS * dh; x += kThreads) {
    const int j = x / dh, d = x - j * dh, col = col0 + j, i = col / g;
    int row = -1;
    if (i < r.look) row = query_row(a, r, b, i, false);
    sh.q[j][d] = row < 0 ? 0.f : load1<T>(a.q, row * a.ld_q + static_cast<long>(kvh * g + col % g) * dh + d);
    if (d == 0) sh.col_row[j] = row < 0 ? -1 : i;
  }
}
template <int T>
__device__ __forceinline__ void load_keys(const MassArgs& a, const Request& r, int b, int kvh, int t0, TileShared& sh, bool report) {
  const int dh = a.pages.head_dim;
  for (int x = threadIdx.x; x < KEYS * dh; x += kThreads) {
    const int j = x / dh, d = x - j * dh;
    const long row = t0 + j < r.kv ? key_row(a, b, t0 + j, report && d == 0) : -1;
    sh.k[j][d] = row < 0 ? 0.f : load1<T>(a.pages.kv, (row * 2 * a.pages.n_kv + kvh) * dh + d);
  }
}
// Scores of this thread's key (threadIdx.x % 64) and columns 4 (threadIdx.x / 64) .. + 3.
__device__ __forceinline__ void tile_scores(int dh, float scale, const TileShared& sh, float (&s)[4]) {
  const int key = threadIdx.x % KEYS, c0 = threadIdx.x / KEYS * 4;
#pragma unroll
  for (int e = 0; e < 4; ++e) s[e] = 0.f;
  for (int d = 0; d < dh; d += 4) {
    const float4 k = *reinterpret_cast<const float4*>(&sh.k[key][d]);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float4 q = *reinterpret_cast<const float4*>(&sh.q[c0 + e][d]);
      s[e] = fmaf(k.w, q.w, fmaf(k.z, q.z, fmaf(k.y, q.y, fmaf(k.x, q.x, s[e]))));
    }
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) s[e] = __fmul_rn(s[e], scale);   // rounded: both passes then see one value
}

// Maxima and sums: the tiles of all requests and key/value heads on one line, a run a block.
template <int T>
__global__ void __launch_bounds__(kThreads) mass_stats_kernel(const MassArgs a, const float scale) {
  pdl_enter();
  extern __shared__ __align__(16) uint8_t smem[];
  TileShared& sh = *reinterpret_cast<TileShared*>(smem);
  int* first = reinterpret_cast<int*>(smem + sizeof(TileShared));
  __shared__ long long warp_sum[kThreads / 32];
  __shared__ float2 halves[kThreads / 32][4];
  tile_line(a, first, warp_sum, blockIdx.x == 0);
  const int hk = a.pages.n_kv, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = a.n_heads / hk;
  const long long total = static_cast<long long>(first[a.B]) * hk;
  const int runs = static_cast<int>(min(static_cast<long long>(a.runs), total)), run = blockIdx.x;
  if (run >= runs) return;
  long long at = total * run / runs;
  const long long end = total * (run + 1) / runs;
  while (at < end) {
    // unit (b, kvh): tiles first[b] * hk + kvh * tiles ..
    const int b = request_at(first, a.B, static_cast<int>(at / hk));
    const Request r = read_request(a, b);
    const int tiles = tiles_of(r);
    const long long inside = at - static_cast<long long>(first[b]) * hk;
    const int kvh = static_cast<int>(inside / tiles), tile0 = static_cast<int>(inside - static_cast<long long>(kvh) * tiles);
    const int tile1 = static_cast<int>(min(static_cast<long long>(tiles), tile0 + (end - at)));
    at += tile1 - tile0;
    float2* out = piece_stats(a) + (run + static_cast<long>(b) * hk + kvh) * (static_cast<long>(g) * a.window);
    for (int col0 = 0; col0 < r.look * g; col0 += COLS) {
      __syncthreads();
      load_queries<T>(a, r, b, kvh, col0, sh);
      float2 stat[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) stat[e] = make_float2(-INFINITY, 0.f);
      for (int tile = tile0; tile < tile1; ++tile) {
        __syncthreads();
        load_keys<T>(a, r, b, kvh, tile * KEYS, sh, true);
        __syncthreads();
        float s[4];
        tile_scores(a.pages.head_dim, scale, sh, s);
        const int t = tile * KEYS + tid % KEYS;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = sh.col_row[tid / KEYS * 4 + e];
          if (i >= 0 && t <= r.kv - r.look + i && t < r.kv) stat[e] = join(stat[e], make_float2(s[e] == s[e] ? s[e] : -INFINITY, s[e] == s[e] ? 1.f : s[e]));
        }
      }
#pragma unroll
      for (int off = 16; off > 0; off >>= 1)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 other = make_float2(__shfl_xor_sync(0xffffffffu, stat[e].x, off), __shfl_xor_sync(0xffffffffu, stat[e].y, off));
          stat[e] = join(stat[e], other);
        }
      if (lane == 0)
#pragma unroll
        for (int e = 0; e < 4; ++e) halves[warp][e] = stat[e];
      __syncthreads();
      if (tid < COLS && col0 + tid < r.look * g) out[col0 + tid] = join(halves[tid / 4 * 2][tid % 4], halves[tid / 4 * 2 + 1][tid % 4]);
    }
  }
}

// A column's pieces in order of their keys: a block per (request, key/value head).
__global__ void __launch_bounds__(kThreads) mass_join_kernel(const MassArgs a) {
  pdl_enter();
  extern __shared__ int first[];
  __shared__ long long warp_sum[kThreads / 32];
  tile_line(a, first, warp_sum, false);
  const int hk = a.pages.n_kv, g = a.n_heads / hk;
  const long long total = static_cast<long long>(first[a.B]) * hk;
  const int runs = static_cast<int>(min(static_cast<long long>(a.runs), total));
  for (long long unit = blockIdx.x; unit < static_cast<long long>(a.B) * hk; unit += gridDim.x) {
    const int b = static_cast<int>(unit / hk), kvh = static_cast<int>(unit % hk);
    const int tiles = first[b + 1] - first[b];
    if (tiles == 0) continue;
    const Request r = read_request(a, b);
    const long long at = static_cast<long long>(first[b]) * hk + static_cast<long long>(kvh) * tiles;
    const int c0 = run_of(total, at, runs), c1 = run_of(total, at + tiles - 1, runs);
    for (int col = threadIdx.x; col < r.look * g; col += kThreads) {
      float2 s = make_float2(-INFINITY, 0.f);
      for (int c = c0; c <= c1; ++c) s = join(s, piece_stats(a)[(c + unit) * (static_cast<long>(g) * a.window) + col]);
      // an entry outside the draft has no weights
      final_stats(a)[b * columns(a) + static_cast<long>(kvh) * g * a.window + col] =
          query_row(a, r, b, col / g, kvh == 0) < 0 ? make_float2(0.f, 0.f) : finish(s);
    }
  }
}

// The weights: a block a tile of keys, all heads' columns in order.
template <int T>
__global__ void __launch_bounds__(kThreads) mass_weights_kernel(const MassArgs a, const float scale) {
  pdl_enter();
  extern __shared__ __align__(16) uint8_t smem[];
  TileShared& sh = *reinterpret_cast<TileShared*>(smem);
  int* first = reinterpret_cast<int*>(smem + sizeof(TileShared));
  __shared__ long long warp_sum[kThreads / 32];
  __shared__ float sums[kThreads];
  __shared__ float2 stat[COLS];
  tile_line(a, first, warp_sum, false);
  const int hk = a.pages.n_kv, tid = threadIdx.x, g = a.n_heads / hk;
  for (int x = blockIdx.x; x < first[a.B]; x += gridDim.x) {
    const int b = request_at(first, a.B, x);
    const Request r = read_request(a, b);
    const int t0 = (x - first[b]) * KEYS, t = t0 + tid % KEYS;
    float sum = 0.f;
    if (r.look > 0)
      for (int kvh = 0; kvh < hk; ++kvh) {
        __syncthreads();
        load_keys<T>(a, r, b, kvh, t0, sh, false);
        for (int col0 = 0; col0 < r.look * g; col0 += COLS) {
          __syncthreads();
          load_queries<T>(a, r, b, kvh, col0, sh);
          if (tid < COLS && col0 + tid < r.look * g)
            stat[tid] = final_stats(a)[b * columns(a) + static_cast<long>(kvh) * g * a.window + col0 + tid];
          __syncthreads();
          float s[4];
          tile_scores(a.pages.head_dim, scale, sh, s);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int j = tid / KEYS * 4 + e, i = sh.col_row[j];
            if (i >= 0 && t <= r.kv - r.look + i) sum += ex2(s[e] - stat[j].x) * stat[j].y;
          }
        }
      }
    __syncthreads();
    sums[tid] = sum;
    __syncthreads();
    if (tid < KEYS && t < r.kv) {
      float w = 0.f;
#pragma unroll
      for (int e = 0; e < kThreads / KEYS; ++e) w += sums[e * KEYS + tid];
      const size_t at = static_cast<size_t>(b) * a.ld_mass + t;
      const int c = r.kv - r.n;
      if (t < c && a.keep != 0.f) w = fmaf(a.keep, a.mass_in[at], w);
      a.mass_out[at] = w;
      if (a.birth && t >= c) a.birth[at] = t + (a.gone ? a.gone[b] : 0);
    }
  }
}

int general_runs(int num_sms) { return 2 * num_sms; }

}  // namespace

size_t mass_workspace(int type, int B, int T_kv_cap, int n_heads, int n_kv, int head_dim, int window, int num_sms) {
  const size_t cols = static_cast<size_t>(n_heads) * window, unit = static_cast<size_t>(n_heads / n_kv) * window;
  return 8 * (B * cols + (general_runs(num_sms) + static_cast<size_t>(B) * n_kv) * unit);
}

cudaError_t launch_mass(int type, const MassArgs& args, int num_sms, cudaStream_t st) {
  MassArgs a = args;
  const float scale = 1.4426950408889634f / sqrtf(static_cast<float>(a.pages.head_dim));
  a.runs = general_runs(num_sms);
  const int line = (a.B + 1) * static_cast<int>(sizeof(int)), smem = static_cast<int>(sizeof(TileShared)) + line;
  const int most = static_cast<int>(sizeof(TileShared)) + (kPageTableMaxB + 1) * static_cast<int>(sizeof(int));
  const long units = static_cast<long>(a.B) * a.pages.n_kv;
  const int joins = static_cast<int>(units < 4l * num_sms ? units : 4l * num_sms);
  const int tiles = a.cap_tiles < 4 * num_sms ? a.cap_tiles : 4 * num_sms;
  {
    static bool set[64] = {};
    const cudaError_t e = set_smem_limit_once(mass_join_kernel, (kPageTableMaxB + 1) * static_cast<int>(sizeof(int)), set);
    if (e != cudaSuccess) return e;
  }
#define SEER_MASS(T)                                                                                          \
  if (type == T) {                                                                                            \
    static bool set0[64] = {}, set1[64] = {};                                                                 \
    cudaError_t e = set_smem_limit_once(mass_stats_kernel<T>, most, set0);                                    \
    if (e == cudaSuccess) e = set_smem_limit_once(mass_weights_kernel<T>, most, set1);                        \
    if (e == cudaSuccess) e = launch_kernel(mass_stats_kernel<T>, dim3(a.runs), dim3(kThreads), smem, st, a, scale); \
    if (e == cudaSuccess) e = launch_kernel(mass_join_kernel, dim3(joins), dim3(kThreads), line, st, a);      \
    if (e == cudaSuccess) e = launch_kernel(mass_weights_kernel<T>, dim3(tiles), dim3(kThreads), smem, st, a, scale); \
    return e;                                                                                                 \
  }
  SEER_MASS(kF32)
  SEER_MASS(kBF16)
  SEER_MASS(kF16)
#undef SEER_MASS
  return cudaErrorInvalidValue;
}

}  // namespace seer
