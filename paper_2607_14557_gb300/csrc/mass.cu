// Attention weight that cached rows receive: per key the softmax weights of a request's last
// rows, summed over them and over all query heads.
//   mass[t] = keep mass[t] + sum_h sum_i 2^(s_hi(t) - m_hi) / l_hi,  s = q k log2(e) / sqrt(dh),
//   m_hi = max_t s_hi(t),  l_hi = sum_t 2^(s_hi(t) - m_hi).
// A column is one query row of one head.  A softmax's weight needs its whole row first.  Here the
// scores of one pass over the keys are kept, with each run's maxima and sums per column, and a
// second kernel joins these and adds up the weights: for fp32, and for 16-bit calls of few columns.
// (tc_mass.cu: many columns, whose scores would be more than the keys, are multiplied twice.)
#include "mass_common.cuh"

namespace seer {
namespace {

constexpr int kThreads = 256;
constexpr int KEYS = 64;                     // keys of a tile

__device__ __forceinline__ int tiles_of(const MassRequest& r) { return (r.kv + KEYS - 1) / KEYS; }
// Key tiles that the call's key capacity allows.
__host__ __device__ inline int tile_capacity(const MassArgs& a) { return a.T_kv_cap / KEYS + a.B; }

// first[b] = key tiles of the requests before b, first[B] all; by the whole block.  Requests
// past the call's key capacity, counted in keys, have no tiles, nor has any behind them.
__device__ __forceinline__ void tile_line(const MassArgs& a, int* first, long long* warp_sum, bool report) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
  long long sum = 0;
#pragma unroll 1
  for (int b0 = 0; b0 < a.B; b0 += blockDim.x) {
    const int b = b0 + tid;
    long long v = 0;
    if (b < a.B) {
      const MassRequest r = read_request(a, b);
      if (!r.good && report) record_error(a.err, kErrLayout);
      v = pack_keys<KEYS>(r.kv);
    }
    long long inc = v;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const long long x = __shfl_up_sync(0xffffffffu, inc, off);
      if (lane >= off) inc += x;
    }
    if (lane == 31) warp_sum[warp] = inc;
    __syncthreads();
    long long before = sum + inc;
#pragma unroll 1
    for (int w = 0; w < warps; ++w) {
      if (w < warp) before += warp_sum[w];
      sum += warp_sum[w];
    }
    if (b < a.B) {
      const bool fits = within(before, a.T_kv_cap);
      if (!fits && v > 0 && report) record_error(a.err, kErrCapacity);
      first[b + 1] = fits ? static_cast<int>(tiles_in<KEYS>(before)) : -1;
    }
    sum = cut_sum(sum, a.T_kv_cap);
    __syncthreads();
  }
  if (tid == 0) first[0] = 0;
  __syncthreads();
  // -1 marks the capacity's end: later requests start and end where the last good one did
  if (first[a.B] < 0) {
    int lo = 0, hi = a.B;                       // first[lo] >= 0, first[hi] < 0
#pragma unroll 1
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (first[mid] >= 0) lo = mid; else hi = mid;
    }
    const int end = first[lo];
    __syncthreads();
#pragma unroll 1
    for (int b = lo + 1 + tid; b <= a.B; b += blockDim.x) first[b] = end;
    __syncthreads();
  }
}

// Workspace: the prefix sums of the tiles, per piece and column (m, l), the scores as
// [tile][column][64].
struct ScoreWork {
  int* first;             // [B + 1]
  float2* stats;
  float* scores;
};
__host__ __device__ inline int columns(const MassArgs& a) { return a.n_heads * a.window; }
__host__ __device__ inline size_t first_bytes(int B) { return (4 * (static_cast<size_t>(B) + 1) + 15) / 16 * 16; }
// fp32: a unit is 16 columns of a key/value head; a piece's statistics are a unit's.  16-bit: a piece
// holds all columns.
constexpr int COLS = 16;
__host__ __device__ inline int unit_blocks(int n_heads, int n_kv, int window) { return (n_heads / n_kv * window + COLS - 1) / COLS; }
__host__ __device__ inline size_t stat_count(bool f32, int B, int runs, int n_heads, int n_kv, int window) {
  if (f32) {
    const size_t units = static_cast<size_t>(n_kv) * unit_blocks(n_heads, n_kv, window);
    return (runs + B * units) * COLS;
  }
  return ((runs + static_cast<size_t>(B)) * n_heads * window + 1) / 2 * 2;
}
__device__ __forceinline__ ScoreWork score_work(const MassArgs& a, bool f32) {
  float2* st = reinterpret_cast<float2*>(static_cast<uint8_t*>(a.ws) + first_bytes(a.B));
  return ScoreWork{static_cast<int*>(a.ws), st, reinterpret_cast<float*>(st + stat_count(f32, a.B, a.runs, a.n_heads, a.pages.n_kv, a.window))};
}

// ------------------------------------------------------------------ fp32
// Scores of a 64-key tile and 16 columns at a time on the CUDA cores: keys and queries of a head in
// shared memory, a thread 4 columns of one key.  Units (request, key/value head, 16 columns) times
// tiles form the line, so that a small call spreads over the GPU; a run's tiles of a unit leave one
// (m, l) per column.  Bound by the latency of a step for small calls, by shared memory for large: 16
// columns are multiplied where a head has four, and no key is on its way meanwhile.  2 to 24 accepted
// rows of 5 requests over 1 to 900 rows, 4 / 2 heads of 64: 14 to 15 us with the sums; one token for
// each of 64 requests over 200 to 8000 rows (32 / 8 heads of 128) 250 us for 497 MB.
struct TileShared {
  float k[KEYS][132];
  float q[COLS][128];
  long row[2][KEYS];                          // pool rows of this tile's keys and the next one's, -1: zeros
  int place[COLS];                            // a column's row among those that look, -1: none
};

__global__ void __launch_bounds__(kThreads) mass_scores_f32_kernel(const MassArgs a, const float scale) {
  pdl_enter();
  extern __shared__ __align__(16) uint8_t smem[];
  TileShared& sh = *reinterpret_cast<TileShared*>(smem);
  int* first = reinterpret_cast<int*>(smem + sizeof(TileShared));
  __shared__ long long warp_sum[kThreads / 32];
  __shared__ float2 halves[kThreads / 32][4];
  tile_line(a, first, warp_sum, blockIdx.x == 0);
  const ScoreWork w = score_work(a, true);
  const int hk = a.pages.n_kv, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = a.n_heads / hk, cc = g * a.window;
  const int blocks = unit_blocks(a.n_heads, hk, a.window), units = hk * blocks, dh = a.pages.head_dim, chunks = dh / 4;
  if (blockIdx.x == 0)
    for (int b = tid; b <= a.B; b += kThreads) w.first[b] = first[b];
  const int total = first[a.B] * units, length = run_length(total, a.runs), run = blockIdx.x;
  int at = min(static_cast<long long>(run) * length, static_cast<long long>(total));
  const int end = min(static_cast<long long>(at) + length, static_cast<long long>(total));
#pragma unroll 1
  while (at < end) {
    const int b = request_at(first, a.B, at / units);
    const MassRequest r = read_request(a, b);
    const int tiles = tiles_of(r), inside = at - first[b] * units, unit = inside / tiles, tile0 = inside - unit * tiles;
    const int tile1 = min(tiles, tile0 + (end - at)), kvh = unit / blocks, col0 = (unit - kvh * blocks) * COLS;
    at += tile1 - tile0;
    if (col0 >= r.look * g) continue;
    const auto look_up = [&](int tile, long (&rows)[KEYS]) {
      if (tid < KEYS) rows[tid] = tile < tile1 && tile * KEYS + tid < r.kv ? key_row(a, b, tile * KEYS + tid, true) : -1;
    };
    __syncthreads();                            // the unit before is done with the queries
    look_up(tile0, sh.row[0]);
#pragma unroll 2
    for (int x = tid; x < COLS * chunks; x += kThreads) {
      const int j = x / chunks, c = x - j * chunks, col = col0 + j, i = col / g;
      const int row = i < r.look && col < cc ? query_row(a, r, b, i, false) : -1;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      if (row >= 0) v = reinterpret_cast<const float4*>(static_cast<const float*>(a.q) + row * a.ld_q + static_cast<long>(kvh * g + col % g) * dh)[c];
      *reinterpret_cast<float4*>(&sh.q[j][4 * c]) = v;
      if (c == 0) sh.place[j] = row < 0 ? -1 : i;
    }
    float2 stat[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) stat[e] = make_float2(-INFINITY, 0.f);
    const int key = tid % KEYS, c0 = tid / KEYS * 4;
#pragma unroll 1
    for (int tile = tile0; tile < tile1; ++tile) {
      const int now = (tile - tile0) & 1;
      __syncthreads();                          // rows are there, the tile before is done with the keys
#pragma unroll 1
      for (int x0 = tid; x0 < KEYS * chunks; x0 += 4 * kThreads) {
        float4 v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int x = min(x0 + e * kThreads, KEYS * chunks - 1), j = x / chunks;
          const long row = sh.row[now][j];
          v[e] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (row >= 0) v[e] = reinterpret_cast<const float4*>(static_cast<const float*>(a.pages.kv) + (row * 2 * hk + kvh) * dh)[x - j * chunks];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int x = min(x0 + e * kThreads, KEYS * chunks - 1), j = x / chunks;
          *reinterpret_cast<float4*>(&sh.k[j][4 * (x - j * chunks)]) = v[e];
        }
      }
      look_up(tile + 1, sh.row[now ^ 1]);
      __syncthreads();
      float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 2
      for (int d = 0; d < dh; d += 4) {
        const float4 k = *reinterpret_cast<const float4*>(&sh.k[key][d]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float4 q = *reinterpret_cast<const float4*>(&sh.q[c0 + e][d]);
          s[e] = fmaf(k.w, q.w, fmaf(k.z, q.z, fmaf(k.y, q.y, fmaf(k.x, q.x, s[e]))));
        }
      }
      const int t = tile * KEYS + key;
      float* out = w.scores + (static_cast<size_t>(first[b] + tile) * hk + kvh) * cc * KEYS + key;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float v = __fmul_rn(s[e], scale);  // as it is kept
        if (col0 + c0 + e < cc) out[(col0 + c0 + e) * KEYS] = v;
        const int i = sh.place[c0 + e];
        if (i >= 0 && t <= r.kv - r.look + i) stat[e] = join(stat[e], make_float2(v == v ? v : -INFINITY, v == v ? 1.f : v));
      }
    }
#pragma unroll 1
    for (int off = 16; off > 0; off >>= 1)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        stat[e] = join(stat[e], make_float2(__shfl_xor_sync(0xffffffffu, stat[e].x, off), __shfl_xor_sync(0xffffffffu, stat[e].y, off)));
    if (lane == 0)
#pragma unroll
      for (int e = 0; e < 4; ++e) halves[warp][e] = stat[e];
    __syncthreads();
    if (tid < COLS)
      w.stats[(run + static_cast<size_t>(b) * units + unit) * COLS + tid] = join(halves[tid / 4 * 2][tid % 4], halves[tid / 4 * 2 + 1][tid % 4]);
  }
}

// ------------------------------------------------------------------ few columns, 16-bit
// Where a key/value head has at most 16 columns (a decoded token of up to 16 heads) the scores
// are kept: 4 bytes a column and key beside the key's 2 head_dim bytes, so the cache is read
// once and the second kernel reads the scores, mostly from L2.  Bound by HBM.  One token for each
// of 64 requests over 200 to 8000 rows (32 / 8 heads of 128), 249 MB, 57 us of which the sums' kernel
// takes 8 behind this one (4.4 TB/s; 5.6 while the keys stream); two requests over 700 and 433
// 11.4 us.  Against the tensor cores' path (tc_mass.cu), four and 16 columns a head: 64 requests 69
// and 105 us against 140, eight 25 and 39.5 against 39.5, two 17 and 29 against 26.  (With caches cold;
// 16 columns a head of 64 requests 95 us in a row of calls: at head_dim 128 two column blocks' queries beside
// the keys spill 68 bytes at the 96 registers of two CTAs an SM.)
// A warp multiplies 16 keys of a head at a time by m16n8k16: the order of a product's terms is
// free, so a lane's 16 bytes of a row serve as the k-indices that the fragment wants from it, and Q
// is cut alike.  A lane keeps the maxima and sums of its two columns over its keys.
constexpr int kFewCols = 16;                // columns of a key/value head at most
constexpr int kFewAll = 1024;               // of all heads
constexpr int GROUP = 16;                   // keys of a step

template <bool F16>
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if (F16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// A CTA: eight warps that multiply and two that load.  A stage is what the eight take at once, 16
// keys of eight heads, or of fewer heads more keys; a key's heads lie side by side in the pool and
// come as one bulk copy, rows of a stage 64 bytes further apart than they are long, so that the
// fragments' 16-byte reads meet in no bank.  Two CTAs per SM, three stages each.  One key/value
// head of 128 takes 120 KB of them, which leaves one CTA per SM (as many thousands of requests do, whose
// sums lie beside the stages), and the runs come in two waves: 64 requests, 16 / 1 heads, 32 MB, 41 us.
constexpr int kStages = 3, kLoaders = 2, kScoreThreads = kThreads + 32 * kLoaders, kWarps = kThreads / 32;
__host__ __device__ constexpr int stage_bytes(int heads, int dh) { return kWarps / heads * GROUP * (heads * dh * 2 + 64); }
__host__ __device__ constexpr int ring_bytes(int n_kv, int dh) { return kStages * stage_bytes(n_kv < kWarps ? n_kv : kWarps, dh); }

// A barrier of the multiplying warps; whether any of their threads says so.
__device__ __forceinline__ bool any_of_multipliers(bool mine) {
  uint32_t any;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 p, %1, 0;\n\t"
      "bar.red.or.pred q, 1, %2, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(any)
      : "r"(static_cast<uint32_t>(mine)), "n"(kThreads)
      : "memory");
  return any != 0;
}

__device__ __forceinline__ void mbar_expect_tx(uint64_t* bar, uint32_t bytes) {
  asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bulk_load(void* smem_dst, const void* src, int bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(smem_u32(smem_dst)), "l"(src), "r"(bytes), "r"(smem_u32(bar))
               : "memory");
}

template <bool F16, int DH, int NT>
__global__ void __launch_bounds__(kScoreThreads, 2) mass_scores_kernel(const MassArgs a, const float scale) {
  extern __shared__ __align__(128) uint8_t ring[];
  int* first = reinterpret_cast<int*>(ring + ring_bytes(a.pages.n_kv, DH));
  __shared__ long long warp_sum[kScoreThreads / 32];
  __shared__ float2 shares[kWarps][NT * 8];
  __shared__ uint64_t full[kStages], empty[kStages];
  __shared__ int pages[kWarps * GROUP];         // of the next keys to load
  __shared__ int abort_word;
  volatile int* abort_flag = &abort_word;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) {
    for (int i = 0; i < kStages; ++i) {
      mbar_init(&full[i], kLoaders);
      mbar_init(&empty[i], kWarps);
    }
    abort_word = 0;
    fence_barrier_init();
  }
  pdl_enter();
  tile_line(a, first, warp_sum, blockIdx.x == 0);
  const int total = first[a.B], length = run_length(total, a.runs), run = blockIdx.x;
  if (run == 0)
    for (int b = tid; b <= a.B; b += kScoreThreads) score_work(a, false).first[b] = first[b];
  int at = run * length;
  const int end = min(at + length, total);
  if (at >= end) return;
  const int hk = a.pages.n_kv, g = a.n_heads / hk, cc = g * a.window;
  const ScoreWork w = score_work(a, false);
  // warps of a head: its keys are dealt to them 16 at a time
  const int heads = min(hk, kWarps), per_head = kWarps / heads;
  const int pitch = heads * DH * 2 + 64, stage = stage_bytes(heads, DH);
  const int page_mask = (1 << a.pages.page_shift) - 1;
  unsigned step = 0;                            // stages used
  bool ok = true;
#pragma unroll 1
  for (int b = request_at(first, a.B, at); ok && at < end; ++b) {
    if (first[b + 1] <= at) continue;
    const MassRequest r = read_request(a, b);
    const int tile0 = at - first[b], tile1 = min(first[b + 1], end) - first[b];
    at += tile1 - tile0;
    const int cols = r.look * g;
    if (cols == 0) continue;
    const int groups = min(tile1 * KEYS, r.kv + GROUP - 1) / GROUP;      // key groups [4 tile0, groups)
    const int group0 = tile0 * (KEYS / GROUP), steps = (groups - group0 + per_head - 1) / per_head;
#pragma unroll 1
    for (int head0 = 0; ok && head0 < hk; head0 += heads) {
      const int here = min(heads, hk - head0);
      if (warp >= kWarps) {
        // ---- loads: a lane a key, the loading warps in turn (a warp's copies go out 50 ns apart); the
        // pages of 128 keys are looked up together
        const int loader = warp - kWarps;
        const int keys = per_head * GROUP, bytes = here * DH * 2, batch = kWarps * GROUP / keys;
        const long row_bytes = 4l * hk * DH;
        const uint8_t* pool = static_cast<const uint8_t*>(a.pages.kv) + head0 * DH * 2;
        const int* table = a.pages.table + static_cast<size_t>(b) * a.pages.max_pages;
#pragma unroll 1
        for (int i = 0; i < steps; ++i, ++step) {
          const int s = step % kStages;
          if (i % batch == 0) {
            __syncwarp();
#pragma unroll
            for (int e = 0; e < kWarps * GROUP / kLoaders / 32; ++e) {
              const int k = (lane + 32 * e) * kLoaders + loader, t = (group0 + i * per_head) * GROUP + k;
              pages[k] = t < r.kv ? table[t >> a.pages.page_shift] : -1;
            }
            __syncwarp();
          }
          if (step >= kStages && !warp_wait(&empty[s], (step / kStages - 1) & 1, abort_flag, a.err)) {
            ok = false;
            break;
          }
#pragma unroll 1
          for (int k = lane * kLoaders + loader; k - lane * kLoaders < keys; k += 32 * kLoaders) {
            const int t = (group0 + i * per_head) * GROUP + k, page = k < keys ? pages[i % batch * keys + k] : -1;
            const bool wanted = k < keys && t < r.kv, there = wanted && page >= 0 && page < a.pages.n_pages;
            uint8_t* dst = ring + s * stage + k * pitch;
            const int rows = __popc(__ballot_sync(0xffffffffu, there));
            if (lane == 0) mbar_expect_tx(&full[s], rows * bytes);
            __syncwarp();
            if (there) {
              bulk_load(dst, pool + ((static_cast<long>(page) << a.pages.page_shift) + (t & page_mask)) * row_bytes, bytes, &full[s]);
            } else if (wanted) {
              record_error(a.err, kErrLayout);               // reads as zeros
#pragma unroll 1
              for (int x = 0; x < bytes; x += 16) *reinterpret_cast<uint4*>(dst + x) = make_uint4(0, 0, 0, 0);
              fence_proxy_async_smem();
            }
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(&full[s]);
        }
        continue;
      }
      // ---- products
      const int h = warp % heads, sub = warp / heads, quad = lane & 3, row = lane >> 2, kvh = head0 + h;
      const bool busy = sub < per_head && h < here;
      float m[NT][2], l[NT][2];
      uint4 q[NT][DH / 32];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        m[nt][0] = m[nt][1] = -INFINITY;
        l[nt][0] = l[nt][1] = 0.f;
        const int col = nt * 8 + row;
        const int qr = busy && col < cols ? query_row(a, r, b, col / g, false) : -1;
        const uint4* src = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.q) + (qr < 0 ? 0 : qr * a.ld_q + static_cast<long>(kvh * g + col % g) * DH));
#pragma unroll
        for (int j = 0; j < DH / 32; ++j) q[nt][j] = qr < 0 ? make_uint4(0, 0, 0, 0) : src[4 * j + quad];
      }
      const int free_to = r.kv - r.look;                     // keys up to it are seen by every row
      const uint8_t* mine = ring + (sub * GROUP + row) * pitch + h * DH * 2 + quad * 16;
#pragma unroll 1
      for (int i = 0; i < steps; ++i, ++step) {
        const int s = step % kStages, gi = group0 + i * per_head + sub, t = gi * GROUP + row;
        if (!warp_wait(&full[s], (step / kStages) & 1, abort_flag, a.err)) {
          ok = false;
          break;
        }
        uint4 lo[DH / 32], hi[DH / 32];
        if (busy) {
#pragma unroll
          for (int j = 0; j < DH / 32; ++j) {
            lo[j] = *reinterpret_cast<const uint4*>(mine + s * stage + j * 64);
            hi[j] = *reinterpret_cast<const uint4*>(mine + s * stage + 8 * pitch + j * 64);
          }
        }
        __syncwarp();
        if (!busy || gi >= groups) {
          if (lane == 0) mbar_arrive(&empty[s]);
          continue;
        }
        float d[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          d[nt][0] = d[nt][1] = d[nt][2] = d[nt][3] = 0.f;
#pragma unroll
          for (int j = 0; j < DH / 32; ++j) {
            mma16816<F16>(d[nt], lo[j].x, hi[j].x, lo[j].y, hi[j].y, q[nt][j].x, q[nt][j].y);
            mma16816<F16>(d[nt], lo[j].z, hi[j].z, lo[j].w, hi[j].w, q[nt][j].z, q[nt][j].w);
          }
        }
        if (lane == 0) mbar_arrive(&empty[s]);               // (the fragments are in registers)
        float* out = w.scores + (static_cast<size_t>(first[b] + (gi >> 2)) * hk + kvh) * cc * KEYS + (gi & 3) * GROUP + row;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int col = nt * 8 + 2 * quad + e;
            float s0 = __fmul_rn(d[nt][e], scale), s1 = __fmul_rn(d[nt][2 + e], scale);   // as they are kept
            if (col < cols) {
              out[col * KEYS] = s0;
              out[col * KEYS + 8] = s1;
            }
            if (t + 8 > free_to) {              // (column col sees keys up to free_to + col / g)
              const int last = free_to + col / g;
              if (t > last) s0 = -INFINITY;
              if (t + 8 > last) s1 = -INFINITY;
            }
            const float top = max3(m[nt][e], s0, s1), base = top == -INFINITY ? 0.f : top;
            l[nt][e] = l[nt][e] * ex2(m[nt][e] - base) + ex2(s0 - base) + ex2(s1 - base);
            m[nt][e] = top;
          }
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float2 x = make_float2(m[nt][e], l[nt][e]);
#pragma unroll
          for (int off = 4; off < 32; off <<= 1)
            x = join(x, make_float2(__shfl_xor_sync(0xffffffffu, x.x, off), __shfl_xor_sync(0xffffffffu, x.y, off)));
          if (row == 0) shares[warp][nt * 8 + 2 * quad + e] = x;
        }
      if (any_of_multipliers(!ok)) {                         // all of them give up together, or a barrier would miss some
        ok = false;
        continue;
      }
      float2* out = w.stats + (static_cast<size_t>(run) + b) * hk * cc;
#pragma unroll 1
      for (int x = tid; x < here * cols; x += kThreads) {
        const int head = x / cols, col = x - head * cols;
        float2 st = shares[head][col];
        for (int e = 1; e < per_head; ++e) st = join(st, shares[head + e * heads][col]);
        out[static_cast<size_t>(head0 + head) * cc + col] = st;
      }
      asm volatile("bar.sync 1, %0;" ::"r"(kThreads) : "memory");
    }
  }
  if (warp >= kWarps && *abort_flag && lane == 0)            // copies still in flight land before the memory is released
    for (unsigned j = step > kStages ? step - kStages : 0; j <= step; ++j) mbar_wait_drain(&full[j % kStages], (j / kStages) & 1, 20000000ull);
}

// A tile a block, two threads a key with every second 16 columns.  Bound by latency, so a
// thread's first scores are loaded before it is known whose the tile is (any tile's memory is
// there; of a capacity far above the keys that there are, only a GPU's worth of tiles is), and the code is kept short: its first instructions come from memory too.
constexpr int kEarly = 16, kSumThreads = 2 * KEYS;
template <bool F32>
__global__ void __launch_bounds__(kSumThreads) mass_sums_kernel(const MassArgs a) {
  pdl_enter();
  extern __shared__ float2 stat[];              // (m, 1 / l) of every column
  __shared__ float sums[kSumThreads];
  const int tid = threadIdx.x, part = tid / KEYS, key = tid % KEYS;
  const int hk = a.pages.n_kv, g = a.n_heads / hk, cc = g * a.window, all = hk * cc;
  uint8_t* row_of = reinterpret_cast<uint8_t*>(stat + all + kEarly);      // a column's row among those that look
  const ScoreWork w = score_work(a, F32);
  int tile = blockIdx.x;
  float s[kEarly];
  const auto load_from = [&](int column) {
    const float* src = w.scores + (static_cast<size_t>(tile) * all + column) * KEYS + key;
#pragma unroll
    for (int e = 0; e < kEarly; ++e) s[e] = column + e < all ? src[e * KEYS] : 0.f;
  };
  load_from(part * kEarly);
  const int total = w.first[a.B];
  const int blocks = unit_blocks(a.n_heads, hk, a.window), units = F32 ? hk * blocks : 1, length = run_length(total * units, a.runs);
  if (tid < kEarly) stat[all + tid] = make_float2(0.f, 0.f);
#pragma unroll 1
  while (tile < total) {
    const int b = request_at(w.first, a.B, tile);
    const int t0 = w.first[b], tiles = w.first[b + 1] - t0;
    const MassRequest r = read_request(a, b);
    const int t = (tile - t0) * KEYS + key;
    const float old = tid < KEYS && t < r.kv ? old_mass(a, r, b, t) : 0.f;
#pragma unroll 1
    for (int x = tid; x < all; x += kSumThreads) {
      float2 f = make_float2(-INFINITY, 0.f);
      const int col = x % cc;
      if (col < r.look * g) {
        const int kvh = x / cc, unit = F32 ? kvh * blocks + col / COLS : 0, place = t0 * units + unit * tiles;
        const int c0 = place / length, c1 = (place + tiles - 1) / length, hop = F32 ? COLS : all;
        const float2* from = w.stats + (static_cast<size_t>(b) * units + unit + c0) * hop + (F32 ? col % COLS : x);
#pragma unroll 1
        for (int c = c0; c <= c1; c += 8) {     // in order of the keys, eight loads under way
          float2 piece[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) piece[e] = c + e <= c1 ? from[e * hop] : make_float2(-INFINITY, 0.f);
          f = join8(f, piece);
          from += 8 * hop;
        }
        f = query_row(a, r, b, col / g, x < cc && tile == t0) < 0 ? make_float2(0.f, 0.f) : finish(f);
      }
      stat[x] = f;                              // (no weights: 1 / l is 0)
      row_of[x] = static_cast<uint8_t>(col / g);
    }
    __syncthreads();
    const int behind = t - (r.kv - r.look);     // > 0: only columns from that row on see it
    float sum = 0.f;
#pragma unroll 1
    for (int x0 = part * kEarly; x0 < all; x0 += kSumThreads / KEYS * kEarly) {
#pragma unroll
      for (int e = 0; e < kEarly; ++e) {
        const float2 st = stat[x0 + e];
        const bool seen = st.y != 0.f && (behind <= 0 || behind <= row_of[x0 + e]);
        sum += seen ? ex2(s[e] - st.x) * st.y : 0.f;
      }
      load_from(x0 + kSumThreads / KEYS * kEarly);
    }
    sums[tid] = sum;
    __syncthreads();
    if (tid < KEYS && t < r.kv) store_mass(a, r, b, t, sums[tid] + sums[KEYS + tid], old);
    tile += gridDim.x;
    if (tile < total) load_from(part * kEarly);
  }
}

int score_runs(bool f32, int num_sms) { return (f32 ? 4 : 2) * num_sms; }
bool few_columns(int n_heads, int n_kv, int window) {
  return n_heads / n_kv * window <= kFewCols && n_heads * window <= kFewAll;
}

}  // namespace

bool mass_on_tensor_cores(int type, int n_heads, int n_kv, int window) { return type != kF32 && !few_columns(n_heads, n_kv, window); }

size_t mass_workspace(int type, int B, int T_kv_cap, int n_heads, int n_kv, int head_dim, int window, int num_sms) {
  if (mass_on_tensor_cores(type, n_heads, n_kv, window)) return tc_mass_workspace(B, T_kv_cap, n_heads, n_kv, window, num_sms);
  const bool f32 = type == kF32;
  return first_bytes(B) + 8 * stat_count(f32, B, score_runs(f32, num_sms), n_heads, n_kv, window) +
         4 * KEYS * static_cast<size_t>(n_heads) * window * (static_cast<size_t>(T_kv_cap) / KEYS + B);
}

cudaError_t launch_mass(int type, const MassArgs& args, int num_sms, cudaStream_t st) {
  MassArgs a = args;
  const bool f32 = type == kF32;
  const float scale = 1.4426950408889634f / sqrtf(static_cast<float>(a.pages.head_dim));
  const int line = (a.B + 1) * static_cast<int>(sizeof(int)), most_line = (kPageTableMaxB + 1) * static_cast<int>(sizeof(int));
  const int most_tiles = tile_capacity(a), sums_smem = 9 * (columns(a) + kEarly);
  const dim3 sums(most_tiles < 16 * num_sms ? most_tiles : 16 * num_sms);
  a.runs = score_runs(f32, num_sms);
  cudaError_t e = cudaErrorInvalidValue;
  if (f32) {
    static bool set0[64] = {}, set1[64] = {};
    const long places = static_cast<long>(most_tiles) * a.pages.n_kv * unit_blocks(a.n_heads, a.pages.n_kv, a.window);
    const dim3 grid(static_cast<unsigned>(places < a.runs ? places : a.runs));
    e = set_smem_limit_once(mass_scores_f32_kernel, static_cast<int>(sizeof(TileShared)) + most_line, set0);
    if (e == cudaSuccess) e = set_smem_limit_once(mass_sums_kernel<true>, 9 * (kMassColumns + kEarly), set1);
    if (e == cudaSuccess) e = launch_kernel(mass_scores_f32_kernel, grid, dim3(kThreads), sizeof(TileShared) + line, st, a, scale);
    if (e == cudaSuccess) e = launch_kernel(mass_sums_kernel<true>, sums, dim3(kSumThreads), sums_smem, st, a);
    return e;
  }
  const dim3 grid(most_tiles < a.runs ? most_tiles : a.runs);
  const int wide = a.n_heads / a.pages.n_kv * a.window > 8;
#define SEER_FEW(F, D, N)                                                                       \
  if ((type == kF16) == F && a.pages.head_dim == D && wide == N - 1) {                          \
    static bool set[64] = {};                                                                   \
    e = set_smem_limit_once(mass_scores_kernel<F, D, N>, ring_bytes(1, D) + most_line, set);    \
    if (e == cudaSuccess)                                                                       \
      e = launch_kernel(mass_scores_kernel<F, D, N>, grid, dim3(kScoreThreads), ring_bytes(a.pages.n_kv, D) + line, st, a, scale); \
  }
  SEER_FEW(false, 64, 1)
  SEER_FEW(false, 64, 2)
  SEER_FEW(false, 128, 1)
  SEER_FEW(false, 128, 2)
  SEER_FEW(true, 64, 1)
  SEER_FEW(true, 64, 2)
  SEER_FEW(true, 128, 1)
  SEER_FEW(true, 128, 2)
#undef SEER_FEW
  if (e == cudaSuccess) e = launch_kernel(mass_sums_kernel<false>, sums, dim3(kSumThreads), sums_smem, st, a);
  return e;
}

}  // namespace seer
