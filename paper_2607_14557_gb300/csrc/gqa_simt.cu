// CUDA-core attention of grouped heads: causal over packed prompts, and new rows
// over a paged cache.
//   o_i = sum_j p_ij v_j / sum_j p_ij,  p_ij = exp(q_i k_j / sqrt(dh) - max),  over the keys j that row i sees
// A tile is BQ of the n * g (token, head of the group) rows that share a key/value head,
// keys in tiles of 64 with an online softmax in fp32 (expf).  Paged: the keys of a request
// may be shared by several blocks, whose unnormalised sums gqa_merge_kernel joins.
#include <math.h>

#include "common.cuh"
#include "paged.h"

namespace seer {
namespace {

constexpr int KT = 64;                        // keys per tile
constexpr int PS = KT + 16;                   // floats per row of probabilities
__host__ __device__ constexpr int row_ld(int dh) { return 4 * ((dh / 4) | 1); }

template <int T>
__device__ __forceinline__ float4 load4(const void* p, size_t i) {
  if (T == kF32) return *reinterpret_cast<const float4*>(static_cast<const float*>(p) + i);
  const uint2 w = *reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(p) + i);
  constexpr bool F16 = T == kF16;
  return make_float4(lo16(w.x, F16), hi16(w.x, F16), lo16(w.y, F16), hi16(w.y, F16));
}
template <int T>
__device__ __forceinline__ void store4(void* p, size_t i, float4 v) {
  if (T == kF32) {
    *reinterpret_cast<float4*>(static_cast<float*>(p) + i) = v;
  } else {
    constexpr bool F16 = T == kF16;
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(p) + i) = make_uint2(pack2(v.x, v.y, F16), pack2(v.z, v.w, F16));
  }
}
__device__ __forceinline__ bool finite4(float4 v) {
  return isfinite(v.x) && isfinite(v.y) && isfinite(v.z) && isfinite(v.w);
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
  s.n = p.cu[b + 1] - s.q0;
  s.good = s.q0 >= 0 && s.n >= 0 && s.n <= p.T_cap - s.q0;
  s.ctx = 0;
  if (PAGED) {
    const int kv = p.kv_len[b];
    s.good = s.good && s.n <= p.max_new && kv >= s.n && kv <= (static_cast<long long>(p.max_pages) << p.page_shift);
    s.ctx = kv - s.n;
  }
  return s;
}

template <int T, bool PAGED, int BQ, int TY, int HALVES>
__global__ void __launch_bounds__(16 * TY) gqa_simt_kernel(const GqaParams p) {
  pdl_enter();
  constexpr int TM = BQ / TY, NTH = 16 * TY;
  const int dh = p.head_dim, G = p.n_heads / p.n_kv;
  int b, kvh, R0, split = 0;
  if (PAGED) {
    const int tiles = (p.max_new * G + BQ - 1) / BQ;
    int u = blockIdx.x;
    split = u % p.splits;
    u /= p.splits;
    R0 = (u % tiles) * BQ;
    u /= tiles;
    kvh = u % p.n_kv;
    b = u / p.n_kv;
  } else {
    // slots of request b start at cu[b] * G / BQ + b, at least as far apart as its tiles
    const int slot = blockIdx.x / p.n_kv;
    kvh = blockIdx.x % p.n_kv;
    int lo = 0, hi = p.B;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (static_cast<long long>(p.cu[mid]) * G / BQ + mid <= slot) lo = mid; else hi = mid;
    }
    b = lo;
    const long long tile = slot - (static_cast<long long>(p.cu[b]) * G / BQ + b);
    if (blockIdx.x == gridDim.x - 1)          // requests that no block's slot leads to
      for (int i = threadIdx.x; i < p.B; i += NTH)
        if (!read_span<PAGED>(p, i).good) record_error(p.err, kErrLayout);
    if (tile < 0 || tile > 0x7fffffff / BQ) return;
    R0 = static_cast<int>(tile) * BQ;
  }
  const Span sp = read_span<PAGED>(p, b);
  if (!sp.good) {
    if (threadIdx.x == 0) record_error(p.err, kErrLayout);
    return;
  }
  const long long all_rows = static_cast<long long>(sp.n) * G;
  if (R0 >= all_rows) return;
  const int rows = static_cast<int>(all_rows - R0 < BQ ? all_rows - R0 : BQ);
  // keys of this tile's last row; every row sees the first `common`
  const int last_tok = (R0 + rows - 1) / G, first_tok = R0 / G;
  const bool chain = !PAGED || p.mask == nullptr;
  const int kv_end = sp.ctx + (chain ? last_tok + 1 : sp.n);
  const int common = sp.ctx + (chain ? first_tok + 1 : 0);
  int k_begin = 0, k_end = kv_end;
  if (PAGED && p.splits > 1) {
    const int tiles = (kv_end + KT - 1) / KT;
    k_begin = static_cast<int>(static_cast<long long>(tiles) * split / p.splits) * KT;
    k_end = min(kv_end, static_cast<int>(static_cast<long long>(tiles) * (split + 1) / p.splits) * KT);
  }

  const int ld = row_ld(dh), per_row = dh / 4;
  extern __shared__ float4 gqa_smem[];
  float* Qs = reinterpret_cast<float*>(gqa_smem);
  float* Ks = Qs + BQ * ld;
  float* Vs = Ks + KT * ld;
  float* Ps = Vs + KT * ld;
  __shared__ int odd_values;                  // the V tile holds an infinity or a NaN
  const int tx = (threadIdx.x & 31) >> 1, ty = (threadIdx.x >> 5) * 2 + (threadIdx.x & 1);

  for (int i = threadIdx.x; i < BQ * per_row; i += NTH) {
    const int r = i / per_row, c = (i - r * per_row) * 4;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    if (r < rows) {
      const int tok = (R0 + r) / G, head = kvh * G + (R0 + r) % G;
      v = load4<T>(p.q, static_cast<size_t>(sp.q0 + tok) * p.ld_q + head * dh + c);
    }
    *reinterpret_cast<float4*>(Qs + r * ld + c) = v;
  }
  const float scale = 1.0f / sqrtf(static_cast<float>(dh));
  int tok[TM];
  uint64_t bits[TM];
  float m[TM], l[TM], o[TM][4 * HALVES];
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    const int r = ty + TY * i;
    tok[i] = (R0 + min(r, rows - 1)) / G;
    bits[i] = chain ? 0 : p.mask[sp.q0 + tok[i]];
    m[i] = -INFINITY;
    l[i] = 0.f;
#pragma unroll
    for (int c = 0; c < 4 * HALVES; ++c) o[i][c] = 0.f;
  }
  const int c0 = 4 * tx;
  for (int k0 = k_begin; k0 < k_end; k0 += KT) {
    __syncthreads();                          // the tile before is done with K, V and P
    if (threadIdx.x == 0) odd_values = 0;
    __syncthreads();
    const int valid = min(KT, k_end - k0);
    const bool masked = k0 + valid > common;  // some row does not see some key of the tile
    for (int i = threadIdx.x; i < KT * per_row; i += NTH) {
      const int r = i / per_row, c = (i - r * per_row) * 4;
      float4 kk = make_float4(0.f, 0.f, 0.f, 0.f), vv = kk;
      if (r < valid) {
        size_t row;
        bool have = true;
        if (PAGED) {
          const int page = p.table[static_cast<size_t>(b) * p.max_pages + ((k0 + r) >> p.page_shift)];
          have = page >= 0 && page < p.n_pages;
          if (!have) record_error(p.err, kErrLayout);
          row = (static_cast<size_t>(page) << p.page_shift) + ((k0 + r) & ((1 << p.page_shift) - 1));
        } else {
          row = static_cast<size_t>(sp.q0 + k0 + r);
        }
        if (have) {                           // a page outside the pool reads as zeros
          kk = load4<T>(p.k, row * p.ld_k + kvh * dh + c);
          vv = load4<T>(p.v, row * p.ld_v + kvh * dh + c);
        }
      }
      if (masked && !finite4(vv)) odd_values = 1;
      *reinterpret_cast<float4*>(Ks + r * ld + c) = kk;
      *reinterpret_cast<float4*>(Vs + r * ld + c) = vv;
    }
    __syncthreads();
    float sc[TM][4] = {};
    for (int d0 = 0; d0 < dh; d0 += 16) {     // a score is summed in blocks of 16 dims
      float part[TM][4] = {};
      for (int d = d0; d < min(d0 + 16, dh); d += 4) {
        float4 kk[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) kk[j] = *reinterpret_cast<const float4*>(Ks + (tx + 16 * j) * ld + d);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
          const float4 q = *reinterpret_cast<const float4*>(Qs + (ty + TY * i) * ld + d);
#pragma unroll
          for (int j = 0; j < 4; ++j)
            part[i][j] = fmaf(q.x, kk[j].x, fmaf(q.y, kk[j].y, fmaf(q.z, kk[j].z, fmaf(q.w, kk[j].w, part[i][j]))));
        }
      }
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) sc[i][j] += part[i][j];
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
      float mx = m[i];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int key = k0 + tx + 16 * j, a = key - sp.ctx;
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
    __syncthreads();
    const bool skip = odd_values != 0;        // a key that a row does not see adds nothing, whatever its value
    for (int k = 0; k < valid; ++k) {
      const float* vrow = Vs + k * ld;
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const float w = Ps[(ty + TY * i) * PS + k];
        if (skip && w == 0.f) continue;
#pragma unroll
        for (int h2 = 0; h2 < HALVES; ++h2) {
          if (c0 + 64 * h2 >= dh) continue;
          const float4 v = *reinterpret_cast<const float4*>(vrow + c0 + 64 * h2);
          o[i][4 * h2 + 0] = fmaf(w, v.x, o[i][4 * h2 + 0]);
          o[i][4 * h2 + 1] = fmaf(w, v.y, o[i][4 * h2 + 1]);
          o[i][4 * h2 + 2] = fmaf(w, v.z, o[i][4 * h2 + 2]);
          o[i][4 * h2 + 3] = fmaf(w, v.w, o[i][4 * h2 + 3]);
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < TM; ++i) {
    float sum = l[i];
#pragma unroll
    for (int off = 16; off > 1; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
    const int r = ty + TY * i;
    if (r >= rows) continue;
    if (PAGED && p.splits > 1) {
      // rows of dh + 2 floats: the sums, their max and their weight
      const size_t unit = (static_cast<size_t>(b) * p.n_kv + kvh) * (static_cast<size_t>(p.max_new) * G) + R0 + r;
      float* part = p.part + (unit * p.splits + split) * (dh + 4);
#pragma unroll
      for (int h2 = 0; h2 < HALVES; ++h2)
        if (c0 + 64 * h2 < dh)
          *reinterpret_cast<float4*>(part + c0 + 64 * h2) =
              make_float4(o[i][4 * h2], o[i][4 * h2 + 1], o[i][4 * h2 + 2], o[i][4 * h2 + 3]);
      if (tx == 0) *reinterpret_cast<float2*>(part + dh) = make_float2(m[i], sum);
    } else {
      const float inv = sum == 0.f ? 0.f : 1.f / sum;   // a row that sees nothing is 0
      const size_t out = static_cast<size_t>(sp.q0 + (R0 + r) / G) * p.ld_o + (kvh * G + (R0 + r) % G) * dh;
#pragma unroll
      for (int h2 = 0; h2 < HALVES; ++h2)
        if (c0 + 64 * h2 < dh)
          store4<T>(p.o, out + c0 + 64 * h2, make_float4(o[i][4 * h2] * inv, o[i][4 * h2 + 1] * inv, o[i][4 * h2 + 2] * inv, o[i][4 * h2 + 3] * inv));
    }
  }
}

// A warp per (request, key/value head, row): its shares' sums, weighted by exp(max - largest max).
template <int T>
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
  float top = -INFINITY;
  for (int s = 0; s < p.splits; ++s) top = fmaxf(top, part[s * (dh + 4) + dh]);
  const float base = top == -INFINITY ? 0.f : top;
  float sum = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int s = 0; s < p.splits; ++s) {
    const float* ps = part + s * (dh + 4);
    const float l = ps[dh + 1], w = l == 0.f ? 0.f : expf(ps[dh] - base);
    sum += l * w;
    if (4 * lane < dh && w != 0.f) {
      const float4 v = *reinterpret_cast<const float4*>(ps + 4 * lane);
      acc = make_float4(fmaf(w, v.x, acc.x), fmaf(w, v.y, acc.y), fmaf(w, v.z, acc.z), fmaf(w, v.w, acc.w));
    }
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  if (4 * lane < dh)
    store4<T>(p.o, static_cast<size_t>(sp.q0 + r / G) * p.ld_o + (kvh * G + r % G) * dh + 4 * lane,
              make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv));
}

constexpr int kRows = 32, kThreadsY = 8;

template <int T, bool PAGED, int HALVES>
cudaError_t launch_typed(const GqaParams& p, cudaStream_t st) {
  const int G = p.n_heads / p.n_kv;
  const long blocks = PAGED ? static_cast<long>(p.B) * p.n_kv * ((static_cast<long>(p.max_new) * G + kRows - 1) / kRows) * p.splits
                            : (static_cast<long>(p.T_cap) * G / kRows + p.B) * p.n_kv;
  if (blocks > 0x7fffffffL) return cudaErrorInvalidValue;
  const int smem = 4 * ((kRows + 2 * KT) * row_ld(p.head_dim) + kRows * PS);
  static bool attr_set[64] = {};
  cudaError_t e = set_smem_limit_once(gqa_simt_kernel<T, PAGED, kRows, kThreadsY, HALVES>, 4 * ((kRows + 2 * KT) * row_ld(64 * HALVES) + kRows * PS), attr_set);
  if (e != cudaSuccess) return e;
  e = launch_kernel(gqa_simt_kernel<T, PAGED, kRows, kThreadsY, HALVES>, dim3(static_cast<unsigned>(blocks)), dim3(16 * kThreadsY), smem, st, p);
  if (e != cudaSuccess || !PAGED || p.splits == 1) return e;
  const long warps = static_cast<long>(p.B) * p.n_kv * p.max_new * G;
  return launch_kernel(gqa_merge_kernel<T>, dim3(static_cast<unsigned>((warps + 7) / 8)), dim3(256), 0, st, p);
}
template <int T>
cudaError_t launch_type(bool paged, const GqaParams& p, cudaStream_t st) {
  if (paged) return p.head_dim <= 64 ? launch_typed<T, true, 1>(p, st) : launch_typed<T, true, 2>(p, st);
  return p.head_dim <= 64 ? launch_typed<T, false, 1>(p, st) : launch_typed<T, false, 2>(p, st);
}

}  // namespace

int gqa_simt_splits(int B, int n_heads, int n_kv, int max_new, int num_sms) {
  const long units = static_cast<long>(B) * n_kv * ((static_cast<long>(max_new) * (n_heads / n_kv) + kRows - 1) / kRows);
  long s = (4l * num_sms + units - 1) / units;
  return static_cast<int>(s < 1 ? 1 : (s > 32 ? 32 : s));
}

size_t gqa_simt_part_bytes(int B, int n_heads, int n_kv, int head_dim, int max_new, int num_sms) {
  const int s = gqa_simt_splits(B, n_heads, n_kv, max_new, num_sms);
  return s == 1 ? 0 : static_cast<size_t>(B) * max_new * n_heads * s * (head_dim + 4) * sizeof(float);
}

cudaError_t launch_gqa_simt(int type, bool paged, const GqaParams& p, int num_sms, cudaStream_t st) {
  (void)num_sms;
  if (p.T_cap <= 0) return cudaSuccess;
  switch (type) {
    case kF32: return launch_type<kF32>(paged, p, st);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace seer
