// fp32 attention of grouped heads on the CUDA cores (the tensor cores have no fp32-input
// mode): causal over packed prompts, and new rows over a paged cache.
//   o_i = sum_j p_ij v_j / sum_j p_ij,  p_ij = exp(q_i k_j / sqrt(dh) - max),  over the keys j that row i sees
// A block has 32 (few blocks: 16) of the n * g (token, head of the group) rows that share a
// key/value head, 128 threads with 4 (2) rows x 4 keys each; keys in tiles of 64 with an online softmax (expf),
// K, V and Q in shared memory by cp.async, the next K under way during a tile's PV and the
// next V during the next scores.  Lanes as in the fp32 kernels of simt.cu.
// Bound, at 4 x 4 values a thread, by shared-memory reads (eight of 16 bytes for 64 multiply-adds)
// and, for few blocks, by latency: 1500 and 700 rows, 8 / 2 heads of 128, 5.6 GFLOP in 172 us (33
// TFLOP/s).
// Few blocks would leave the longest row's tiles in a chain (5 prompts of 1 .. 300 rows, 34 us
// with one block per tile of rows), so its keys are shared: causal, by a cluster of blocks
// that merge through distributed shared memory; paged, by blocks whose unnormalised sums
// gqa_merge_kernel joins.
#include <math.h>

#include "common.cuh"
#include "paged.h"

namespace seer {
namespace {

constexpr int TY = 8, NTH = 16 * TY;
constexpr int KT = 64;                        // keys per tile
constexpr int PS = KT + 16;                   // floats per row of probabilities
constexpr int MAX_PARTS = 8;                  // blocks of a cluster
// Staged rows hold 64 or 128 dims, zeros past head_dim, so that every address is a constant
// away from a thread's own; an odd number of 16-byte words meets no bank twice.
__host__ __device__ constexpr int row_ld(int dims) { return dims + 4; }
__host__ __device__ constexpr int smem_floats(int rows, int dims) { return (rows + 2 * KT) * row_ld(dims) + rows * PS + 2 * rows; }

__device__ __forceinline__ void copy16(float* dst, const float* src, bool valid) {   // zeros where !valid
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(valid ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
// acc.x += a0 * b0, acc.y += a1 * b1.
__device__ __forceinline__ void fma_pair(float2& acc, float a0, float a1, float b0, float b1) {
  asm("{\n\t.reg .b64 ra, rb, rc;\n\t"
      "mov.b64 ra, {%2, %3};\n\t"
      "mov.b64 rb, {%4, %5};\n\t"
      "mov.b64 rc, {%0, %1};\n\t"
      "fma.rn.f32x2 rc, ra, rb, rc;\n\t"
      "mov.b64 {%0, %1}, rc;\n\t}"
      : "+f"(acc.x), "+f"(acc.y) : "f"(a0), "f"(a1), "f"(b0), "f"(b1));
}
__device__ __forceinline__ float ld_cluster(uint32_t addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr));
  return v;
}
__device__ __forceinline__ float4 ld_cluster4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr));
  return v;
}

// A request's rows and keys, checked against the buffers before anything follows them.
struct Span {
  int q0, n, ctx;                             // first new row, new rows, keys that every row sees
  bool good;
};
template <bool PAGED>
__device__ __forceinline__ Span read_span(const GqaParams& p, int b) {
  Span s;
  s.q0 = p.cu[b];
  const int end = p.cu[b + 1];
  s.good = s.q0 >= 0 && end >= s.q0 && end <= p.T_cap;
  s.n = s.good ? end - s.q0 : 0;
  s.ctx = 0;
  if (PAGED) {
    const int kv = p.kv_len[b];
    s.good = s.good && s.n <= p.max_new && kv >= s.n && kv <= kMaxKeys && kv <= (static_cast<long long>(p.max_pages) << p.page_shift);
    s.ctx = kv - s.n;
  }
  return s;
}

// Tiles of a causal call at most.
__host__ __device__ __forceinline__ long causal_units(const GqaParams& p, int rows) {
  return (static_cast<long>(p.T_cap) * (p.n_heads / p.n_kv) / rows + p.B) * p.n_kv;
}
// Slots of sequence b start at cu[b] * G / BQ + b, at least as far apart as its tiles: the last
// sequence that starts by `slot`.  Offsets ascend, so a warp looks at 32 at once (2 us of a
// short call were bisection's loads).
template <int BQ>
__device__ __forceinline__ int sequence_at(const GqaParams& p, int G, int slot) {
  int lo = 0, hi = p.B;
  while (hi - lo > 1) {
    const int step = (hi - lo + 31) / 32, at = lo + static_cast<int>(threadIdx.x & 31) * step;
    const bool before = at < hi && (at == lo || static_cast<long long>(p.cu[at]) * G / BQ + at <= slot);
    lo += (__popc(__ballot_sync(0xffffffffu, before)) - 1) * step;
    hi = min(hi, lo + step);
  }
  return lo;
}

// Where some offset falls: the sequence and tile of the slot-th tile, counted over the sequences
// that lie in the buffers; b = B past the last.  By a whole block.
template <int BQ>
__device__ __forceinline__ int2 tile_at(const GqaParams& p, int G, long slot, long* sums) {
  const auto tiles = [&](int b) -> long {
    const Span s = read_span<false>(p, b);
    return s.good ? (static_cast<long>(s.n) * G + BQ - 1) / BQ : 0;
  };
  const int each = (p.B + NTH - 1) / NTH;
  long mine = 0;
  for (int b = threadIdx.x * each; b < min(p.B, (static_cast<int>(threadIdx.x) + 1) * each); ++b) mine += tiles(b);
  sums[threadIdx.x] = mine;
  __syncthreads();
  int t = 0;
  while (t < NTH && slot >= sums[t]) slot -= sums[t++];
  __syncthreads();                            // the sums' memory is free again
  int b = min(p.B, t * each);
  for (; b < p.B; ++b) {
    const long n = tiles(b);
    if (slot < n) break;
    slot -= n;
  }
  return make_int2(b, static_cast<int>(slot));
}

// Rows [R0, R0 + BQ) of request b's (token, head) rows.  CLUSTER: the blocks of a cluster share
// the tile's keys.
template <bool PAGED, bool CLUSTER, int BQ, int HALVES>
__device__ __forceinline__ void attend_tile(const GqaParams& p, int b, int kvh, int R0, int split) {
  const Span sp = read_span<PAGED>(p, b);
  if (!sp.good) {
    if (threadIdx.x == 0) record_error(p.err, kErrLayout);
    return;
  }
  constexpr int TM = BQ / TY, DIMS = 64 * HALVES, ld = row_ld(DIMS);
  const int dh = p.head_dim, G = p.n_heads / p.n_kv, parts = p.splits;
  const long long all_rows = static_cast<long long>(sp.n) * G;
  if (R0 >= all_rows) return;
  const int rows = static_cast<int>(all_rows - R0 < BQ ? all_rows - R0 : BQ);
  // keys of this tile's last row; every row sees the first `common`
  const int last_tok = (R0 + rows - 1) / G, first_tok = R0 / G;
  const bool chain = !PAGED || p.mask == nullptr;
  const int kv_end = sp.ctx + (chain ? last_tok + 1 : sp.n);
  const int common = sp.ctx + (chain ? first_tok + 1 : 0);
  int k_begin = 0, k_end = kv_end;
  if (parts > 1) {
    const int tiles = (kv_end + KT - 1) / KT;
    k_begin = static_cast<int>(static_cast<long long>(tiles) * split / parts) * KT;
    k_end = min(kv_end, static_cast<int>(static_cast<long long>(tiles) * (split + 1) / parts) * KT);
  }

  extern __shared__ float4 gqa_smem[];
  float* Qs = reinterpret_cast<float*>(gqa_smem);
  float* Ks = Qs + BQ * ld;
  float* Vs = Ks + KT * ld;
  float* Ps = Vs + KT * ld;
  float* Ms = Ps + BQ * PS;                   // [BQ][2] max and weight of a row (clusters)
  const int tx = (threadIdx.x & 31) >> 1, ty = (threadIdx.x >> 5) * 2 + (threadIdx.x & 1);
  const float *q = static_cast<const float*>(p.q), *kp = static_cast<const float*>(p.k), *vp = static_cast<const float*>(p.v);

  // a warp stages a row of 128 dims or two of 64 at a time
  constexpr int ROWS = 32 / (DIMS / 4);
  const int srow = (threadIdx.x >> 5) * ROWS + (threadIdx.x & 31) / (DIMS / 4), scol = (threadIdx.x & 31) % (DIMS / 4) * 4;
  const bool in_head = scol < dh;
  // a K or V tile; zeros past k_end and on pages outside the pool
  const auto load = [&](float* dst, const float* src, long row_step, int k0, bool report) {
    if (k0 < k_end)
#pragma unroll 4
      for (int r = srow; r < KT; r += NTH / 32 * ROWS) {
        bool have = k0 + r < k_end;
        size_t row = 0;
        if (PAGED) {
          const int page = have ? p.table[static_cast<size_t>(b) * p.max_pages + ((k0 + r) >> p.page_shift)] : 0;
          if (page < 0 || page >= p.n_pages) {
            if (report) record_error(p.err, kErrLayout);
            have = false;
          }
          if (have) row = (static_cast<size_t>(page) << p.page_shift) + ((k0 + r) & ((1 << p.page_shift) - 1));
        } else if (have) {
          row = static_cast<size_t>(sp.q0 + k0 + r);
        }
        copy16(dst + r * ld + scol, have && in_head ? src + row * row_step + kvh * dh + scol : src, have && in_head);
      }
    copy_commit();
  };
  for (int r = srow; r < BQ; r += NTH / 32 * ROWS) {
    const bool have = r < rows && in_head;
    const int tok_r = have ? (R0 + r) / G : 0;
    copy16(Qs + r * ld + scol, have ? q + static_cast<size_t>(sp.q0 + tok_r) * p.ld_q + (kvh * G + R0 + r - tok_r * G) * dh + scol : q, have);
  }
  load(Ks, kp, p.ld_k, k_begin, true);        // Q is part of this group
  load(Vs, vp, p.ld_v, k_begin, false);

  const float scale = 1.0f / sqrtf(static_cast<float>(dh));
  int tok[TM];
  uint64_t bits[TM];
  float m[TM], l[TM], o[TM][4 * HALVES];
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    tok[i] = (R0 + min(ty + TY * i, rows - 1)) / G;
    bits[i] = chain ? 0 : p.mask[sp.q0 + tok[i]];
    m[i] = -INFINITY;
    l[i] = 0.f;
#pragma unroll
    for (int c = 0; c < 4 * HALVES; ++c) o[i][c] = 0.f;
  }
  const int c0 = 4 * tx;
  for (int k0 = k_begin; k0 < k_end; k0 += KT) {
    const int valid = min(KT, k_end - k0);
    const bool masked = k0 + valid > common;  // some row does not see some key of the tile
    copy_wait<1>();                           // K of the tile (its V is the group after)
    __syncthreads();
    // a score is summed in blocks of 16 dims, each two packed chains of 8
    float sc[TM][4] = {};
#pragma unroll 1
    for (int d0 = 0; d0 < dh; d0 += 16) {
      float2 part[TM][4] = {};
#pragma unroll
      for (int d = 0; d < 16; d += 4) {
        float4 kk[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) kk[j] = *reinterpret_cast<const float4*>(Ks + (tx + 16 * j) * ld + d0 + d);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
          const float4 qq = *reinterpret_cast<const float4*>(Qs + (ty + TY * i) * ld + d0 + d);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            fma_pair(part[i][j], qq.x, qq.y, kk[j].x, kk[j].y);
            fma_pair(part[i][j], qq.z, qq.w, kk[j].z, kk[j].w);
          }
        }
      }
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) sc[i][j] += part[i][j].x + part[i][j].y;
    }
    __syncthreads();                          // every warp is done with K
    load(Ks, kp, p.ld_k, k0 + KT, true);
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      float mx = m[i];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int a = k0 + tx + 16 * j - sp.ctx;
        const bool seen = tx + 16 * j < valid && (a < 0 || (chain ? a <= tok[i] : ((bits[i] >> a) & 1) != 0));
        sc[i][j] = seen ? sc[i][j] * scale : -INFINITY;
        mx = fmaxf(mx, sc[i][j]);
      }
#pragma unroll
      for (int off = 16; off > 1; off >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
      const float base = mx == -INFINITY ? 0.f : mx;   // nothing seen so far: every term is 0
      const float alpha = expf(m[i] - base);
      m[i] = mx;
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float e = expf(sc[i][j] - base);
        sum += e;
        Ps[(ty + TY * i) * PS + tx + 16 * j] = e;
      }
      l[i] = l[i] * alpha + sum;
#pragma unroll
      for (int c = 0; c < 4 * HALVES; ++c) o[i][c] *= alpha;
    }
    copy_wait<1>();                           // V of the tile
    int odd = 0;                              // an infinity or a NaN among values that not every row sees
    if (masked) {
      __syncthreads();
      for (int r = srow; r < valid; r += NTH / 32 * ROWS) {
        const float4 v = *reinterpret_cast<const float4*>(Vs + r * ld + scol);
        odd |= !(isfinite(v.x) && isfinite(v.y) && isfinite(v.z) && isfinite(v.w));
      }
      odd = __syncthreads_or(odd);
    } else {
      __syncthreads();
    }
    const auto add = [&](int i, float w, const float* vrow) {
#pragma unroll
      for (int h2 = 0; h2 < HALVES; ++h2) {
        const float4 v = *reinterpret_cast<const float4*>(vrow + c0 + 64 * h2);
        o[i][4 * h2 + 0] = fmaf(w, v.x, o[i][4 * h2 + 0]);
        o[i][4 * h2 + 1] = fmaf(w, v.y, o[i][4 * h2 + 1]);
        o[i][4 * h2 + 2] = fmaf(w, v.z, o[i][4 * h2 + 2]);
        o[i][4 * h2 + 3] = fmaf(w, v.w, o[i][4 * h2 + 3]);
      }
    };
    if (odd) {                                // a key that a row does not see adds nothing, whatever its value
      for (int k = 0; k < valid; ++k) {       // (a seen one adds even with a weight of 0)
        const int a = k0 + k - sp.ctx;
#pragma unroll
        for (int i = 0; i < TM; ++i)
          if (a < 0 || (chain ? a <= tok[i] : ((bits[i] >> a) & 1) != 0)) add(i, Ps[(ty + TY * i) * PS + k], Vs + k * ld);
      }
    } else {
      const int keys = min(KT, (valid + 3) & ~3);   // past the valid keys P is 0 and V zero-filled
#pragma unroll 2
      for (int k = 0; k < keys; k += 4) {
        float4 pr[TM];
#pragma unroll
        for (int i = 0; i < TM; ++i) pr[i] = *reinterpret_cast<const float4*>(Ps + (ty + TY * i) * PS + k);
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int i = 0; i < TM; ++i) add(i, e == 0 ? pr[i].x : (e == 1 ? pr[i].y : (e == 2 ? pr[i].z : pr[i].w)), Vs + (k + e) * ld);
      }
    }
    __syncthreads();                          // every warp is done with V and P
    load(Vs, vp, p.ld_v, k0 + KT, false);
  }
  float sum[TM];
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    sum[i] = l[i];
#pragma unroll
    for (int off = 16; off > 1; off >>= 1) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], off);
  }
  float* out = static_cast<float*>(p.o);
  const auto out_row = [&](int r) { return out + static_cast<size_t>(sp.q0 + (R0 + r) / G) * p.ld_o + (kvh * G + (R0 + r) % G) * dh; };
  if constexpr (CLUSTER) {
    // every block leaves its sums, maxima and weights in its own shared memory and writes
    // BQ / parts of the rows from all blocks' shares, in order of their keys
    copy_wait<0>();
    __syncthreads();
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int r = ty + TY * i;
#pragma unroll
      for (int h2 = 0; h2 < HALVES; ++h2)
        *reinterpret_cast<float4*>(Vs + r * ld + c0 + 64 * h2) = make_float4(o[i][4 * h2], o[i][4 * h2 + 1], o[i][4 * h2 + 2], o[i][4 * h2 + 3]);
      if (tx == 0) *reinterpret_cast<float2*>(Ms + 2 * r) = make_float2(m[i], sum[i]);
    }
    cluster_sync();
    const int each = BQ / parts;
    for (int i = threadIdx.x; i < each * (DIMS / 4); i += NTH) {
      const int r = split * each + i / (DIMS / 4), c = i % (DIMS / 4) * 4;
      if (r >= rows || c >= dh) continue;
      float top = -INFINITY, total = 0.f;
#pragma unroll
      for (int k = 0; k < MAX_PARTS; ++k)
        if (k < parts) top = fmaxf(top, ld_cluster(cluster_addr(Ms + 2 * r, k)));
      const float base = top == -INFINITY ? 0.f : top;
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < MAX_PARTS; ++k)
        if (k < parts) {
          const uint32_t ml = cluster_addr(Ms + 2 * r, k);
          const float weight = ld_cluster(ml + 4), w = weight == 0.f ? 0.f : expf(ld_cluster(ml) - base);
          total += weight * w;
          if (weight != 0.f) {                // a share without a seen key adds nothing
            const float4 v = ld_cluster4(cluster_addr(Vs + r * ld + c, k));
            acc = make_float4(fmaf(w, v.x, acc.x), fmaf(w, v.y, acc.y), fmaf(w, v.z, acc.z), fmaf(w, v.w, acc.w));
          }
        }
      const float inv = total == 0.f ? 0.f : 1.f / total;
      *reinterpret_cast<float4*>(out_row(r) + c) = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
    }
    cluster_sync();                           // no block leaves while its rows are read
  } else {
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      const int r = ty + TY * i;
      if (r >= rows) continue;
      if (PAGED && parts > 1) {
        // rows of dh + 4 floats: the sums, their max and their weight
        const size_t at = (static_cast<size_t>(b) * p.n_kv + kvh) * (static_cast<size_t>(p.max_new) * G) + R0 + r;
        float* part = p.part + (at * parts + split) * (dh + 4);
#pragma unroll
        for (int h2 = 0; h2 < HALVES; ++h2)
          if (c0 + 64 * h2 < dh)
            *reinterpret_cast<float4*>(part + c0 + 64 * h2) = make_float4(o[i][4 * h2], o[i][4 * h2 + 1], o[i][4 * h2 + 2], o[i][4 * h2 + 3]);
        if (tx == 0) *reinterpret_cast<float2*>(part + dh) = make_float2(m[i], sum[i]);
      } else {
        const float inv = sum[i] == 0.f ? 0.f : 1.f / sum[i];   // a row that sees nothing is 0
#pragma unroll
        for (int h2 = 0; h2 < HALVES; ++h2)
          if (c0 + 64 * h2 < dh)
            *reinterpret_cast<float4*>(out_row(r) + c0 + 64 * h2) = make_float4(o[i][4 * h2] * inv, o[i][4 * h2 + 1] * inv, o[i][4 * h2 + 2] * inv, o[i][4 * h2 + 3] * inv);
      }
    }
  }
  copy_wait<0>();
}

// The blocks ahead of a causal call's look through all offsets.  Where one falls, the others' slots
// may have led past some sequences' tiles, so these blocks take all tiles in turn.
template <bool CLUSTER, int BQ, int HALVES>
__device__ __noinline__ void take_all_if_one_falls(const GqaParams& p, int worker, int scouts, int split) {
  int falls = 0;
#pragma unroll 4
  for (int i = threadIdx.x; i < p.B; i += NTH) falls |= p.cu[i] > p.cu[i + 1];
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i < p.B; i += NTH)
      if (!read_span<false>(p, i).good) record_error(p.err, kErrLayout);
  if (!__syncthreads_or(falls)) return;
  extern __shared__ float4 gqa_smem[];
  for (long i = worker;; i += scouts) {
    const int2 at = tile_at<BQ>(p, p.n_heads / p.n_kv, i / p.n_kv, reinterpret_cast<long*>(gqa_smem));
    if (at.x >= p.B) return;
    attend_tile<false, CLUSTER, BQ, HALVES>(p, at.x, static_cast<int>(i % p.n_kv), at.y * BQ, split);
    __syncthreads();
  }
}

// (32 rows of up to 64 dims: shared memory lets four blocks in, so registers have to, too.  600
// prompts of 1 .. 40 rows 39.6 us, 43 with three)
template <bool PAGED, bool CLUSTER, int BQ, int HALVES>
__global__ void __launch_bounds__(NTH, HALVES == 1 && BQ == 32 ? 4 : 1) gqa_simt_kernel(const GqaParams p) {
  pdl_enter();
  const int G = p.n_heads / p.n_kv, parts = p.splits;
  const int split = CLUSTER ? static_cast<int>(cluster_ctarank()) : (PAGED ? static_cast<int>(blockIdx.x) % parts : 0);
  if constexpr (PAGED) {
    const int tiles = (p.max_new * G + BQ - 1) / BQ, unit = blockIdx.x / parts;
    const int R0 = (unit % tiles) * BQ, kvh = unit / tiles % p.n_kv, b = unit / tiles / p.n_kv;
    attend_tile<PAGED, CLUSTER, BQ, HALVES>(p, b, kvh, R0, split);
  } else {
    const int units = static_cast<int>(causal_units(p, BQ)), worker = blockIdx.x / parts, scouts = gridDim.x / parts - units;
    if (worker >= scouts) {
      const int unit = units - 1 - (worker - scouts);    // a sequence's last rows, which see the most keys, first
      const int slot = unit / p.n_kv, kvh = unit % p.n_kv, b = sequence_at<BQ>(p, G, slot);
      const long tile = slot - (static_cast<long>(p.cu[b]) * G / BQ + b);
      if (tile < 0 || tile > 0x7fffffff / BQ) return;
      attend_tile<PAGED, CLUSTER, BQ, HALVES>(p, b, kvh, static_cast<int>(tile) * BQ, split);
      return;
    }
    take_all_if_one_falls<CLUSTER, BQ, HALVES>(p, worker, scouts, split);
  }
}

// A warp per (request, key/value head, row): its shares' sums, weighted by exp(max - largest max).
__global__ void __launch_bounds__(256) gqa_merge_kernel(const GqaParams p) {
  pdl_enter();
  const int G = p.n_heads / p.n_kv, dh = p.head_dim, lane = threadIdx.x & 31;
  const long per_req = static_cast<long>(p.max_new) * G;
  const long unit = (blockIdx.x * 256l + threadIdx.x) >> 5;
  if (unit >= per_req * p.n_kv * p.B) return;
  const int r = static_cast<int>(unit % per_req), kvh = static_cast<int>(unit / per_req % p.n_kv);
  const int b = static_cast<int>(unit / per_req / p.n_kv);
  const Span sp = read_span<true>(p, b);
  if (!sp.good || r >= static_cast<long>(sp.n) * G) return;
  const float* part = p.part + unit * p.splits * (dh + 4);
  float m = -INFINITY, sum = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int s = 0; s < p.splits; ++s) {
    const float* ps = part + s * (dh + 4);
    const float2 ml = *reinterpret_cast<const float2*>(ps + dh);
    const float4 v = 4 * lane < dh ? *reinterpret_cast<const float4*>(ps + 4 * lane) : make_float4(0.f, 0.f, 0.f, 0.f);
    if (ml.y == 0.f) continue;                // a share without a seen key adds nothing
    const float top = fmaxf(m, ml.x), base = top == -INFINITY ? 0.f : top;
    const float old = expf(m - base), w = expf(ml.x - base);
    m = top;
    sum = fmaf(sum, old, ml.y * w);
    acc = make_float4(fmaf(acc.x, old, w * v.x), fmaf(acc.y, old, w * v.y), fmaf(acc.z, old, w * v.z), fmaf(acc.w, old, w * v.w));
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  if (4 * lane < dh)
    *reinterpret_cast<float4*>(static_cast<float*>(p.o) + static_cast<size_t>(sp.q0 + r / G) * p.ld_o + (kvh * G + r % G) * dh + 4 * lane) =
        make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
}

long paged_units(int B, int n_heads, int n_kv, int max_new, int rows) {
  return static_cast<long>(B) * n_kv * ((static_cast<long>(max_new) * (n_heads / n_kv) + rows - 1) / rows);
}
// Rows of a block: 32, or 16 where blocks of 32 would leave SMs idle.  us at 32 / 16: prompts of
// 1 .. 300 rows, 4 heads of 64 (96 blocks) 16.5 / 14.2; eight drafts of 8 rows over 300 .. 3000
// (16) 48 / 41; one prompt of 2000, 4 heads of 128 (251) 141 / 152; eight of 300, 8 heads of 64
// (664) 43.3 / 45.8.
int block_rows(long units_of_32, int num_sms) { return units_of_32 <= num_sms ? 16 : 32; }

template <bool PAGED, bool CLUSTER, int BQ, int HALVES>
cudaError_t launch_typed(const GqaParams& p, int num_sms, cudaStream_t st) {
  // (causal: some more ahead, for offsets that fall)
  const long units = PAGED ? paged_units(p.B, p.n_heads, p.n_kv, p.max_new, BQ) : causal_units(p, BQ) + (num_sms / 4 + p.splits - 1) / p.splits;
  const long blocks = units * p.splits;
  if (blocks > 0x7fffffffL) return cudaErrorInvalidValue;
  constexpr int smem = 4 * smem_floats(BQ, 64 * HALVES);
  static bool attr_set[64] = {};
  cudaError_t e = set_smem_limit_once(gqa_simt_kernel<PAGED, CLUSTER, BQ, HALVES>, smem, attr_set);
  if (e != cudaSuccess) return e;
  e = launch_kernel_overlap(launch_overlap_enabled(), CLUSTER ? p.splits : 1, gqa_simt_kernel<PAGED, CLUSTER, BQ, HALVES>,
                            dim3(static_cast<unsigned>(blocks)), dim3(NTH), smem, st, p);
  if (e != cudaSuccess || !PAGED || p.splits == 1) return e;
  const long warps = static_cast<long>(p.B) * p.max_new * p.n_heads;
  return launch_kernel(gqa_merge_kernel, dim3(static_cast<unsigned>((warps + 7) / 8)), dim3(256), 0, st, p);
}
template <bool PAGED, bool CLUSTER, int BQ>
cudaError_t launch_halves(const GqaParams& p, int num_sms, cudaStream_t st) {
  return p.head_dim <= 64 ? launch_typed<PAGED, CLUSTER, BQ, 1>(p, num_sms, st) : launch_typed<PAGED, CLUSTER, BQ, 2>(p, num_sms, st);
}
template <bool PAGED, bool CLUSTER>
cudaError_t launch_rows(const GqaParams& p, int rows, int num_sms, cudaStream_t st) {
  return rows == 16 ? launch_halves<PAGED, CLUSTER, 16>(p, num_sms, st) : launch_halves<PAGED, CLUSTER, 32>(p, num_sms, st);
}

}  // namespace

int gqa_simt_splits(int B, int n_heads, int n_kv, int max_new, int num_sms) {
  const int rows = block_rows(paged_units(B, n_heads, n_kv, max_new, 32), num_sms);
  const long units = paged_units(B, n_heads, n_kv, max_new, rows);
  const long s = (4l * num_sms + units - 1) / units;
  return static_cast<int>(s < 1 ? 1 : (s > 32 ? 32 : s));
}

size_t gqa_simt_part_bytes(int B, int n_heads, int n_kv, int head_dim, int max_new, int num_sms) {
  const int s = gqa_simt_splits(B, n_heads, n_kv, max_new, num_sms);
  return s == 1 ? 0 : static_cast<size_t>(B) * max_new * n_heads * s * (head_dim + 4) * sizeof(float);
}

cudaError_t launch_gqa_simt(bool paged, const GqaParams& args, int num_sms, cudaStream_t st) {
  GqaParams p = args;
  if (p.T_cap <= 0) return cudaSuccess;
  if (paged)
    return launch_rows<true, false>(p, block_rows(paged_units(p.B, p.n_heads, p.n_kv, p.max_new, 32), num_sms), num_sms, st);
  const int rows = block_rows(causal_units(p, 32), num_sms);
  // causal: blocks that share a tile's keys, as many as the SMs hold at once, where
  // prompts have the tiles to share on average
  const long units = causal_units(p, rows);
  p.splits = 1;
  while (p.splits < MAX_PARTS && units * p.splits * 2 <= 4l * num_sms && p.T_cap / p.B >= KT * p.splits) p.splits *= 2;
  return p.splits > 1 ? launch_rows<false, true>(p, rows, num_sms, st) : launch_rows<false, false>(p, rows, num_sms, st);
}

}  // namespace seer
