// Rotary positions of either pair layout, of part of a head: rows of heads, and rows on
// their way into a paged cache.
//   (a, b) -> m (a cos - b sin, b cos + a sin),  angle = position * rate_i,
// pairs (i, i + rd/2) or (2i, 2i + 1) of a head's first rd values, the others copied.
// The angle is taken in turns, position * rate modulo 1 in 64-bit integers (exact; the rate
// comes from the host in fp64), and its fraction goes to sincospif.
#include "budget.h"
#include "common.cuh"

namespace seer {
namespace {

constexpr int kRotThreads = 256;
constexpr int kRotRows = 4;
constexpr int kUnroll = 3;

// W 32-bit words at once.
template <int W>
struct Words {
  uint32_t w[W];
};
template <int W>
__device__ __forceinline__ Words<W> load_words(const uint8_t* p) {
  Words<W> v;
  if constexpr (W == 4) {
    const uint4 x = *reinterpret_cast<const uint4*>(p);
    v.w[0] = x.x;
    v.w[1] = x.y;
    v.w[2] = x.z;
    v.w[3] = x.w;
  } else if constexpr (W == 2) {
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    v.w[0] = x.x;
    v.w[1] = x.y;
  } else {
    v.w[0] = *reinterpret_cast<const uint32_t*>(p);
  }
  return v;
}
template <int W>
__device__ __forceinline__ void store_words(uint8_t* p, const Words<W>& v) {
  if constexpr (W == 4) *reinterpret_cast<uint4*>(p) = make_uint4(v.w[0], v.w[1], v.w[2], v.w[3]);
  else if constexpr (W == 2) *reinterpret_cast<uint2*>(p) = make_uint2(v.w[0], v.w[1]);
  else *reinterpret_cast<uint32_t*>(p) = v.w[0];
}
template <int T, int W, int N>
__device__ __forceinline__ void unpack(const Words<W>& v, float (&f)[N]) {
#pragma unroll
  for (int i = 0; i < W; ++i) {
    if constexpr (T == kF32) {
      f[i] = __uint_as_float(v.w[i]);
    } else {
      f[2 * i] = lo16(v.w[i], T == kF16);
      f[2 * i + 1] = hi16(v.w[i], T == kF16);
    }
  }
}
template <int T, int W, int N>
__device__ __forceinline__ Words<W> pack(const float (&f)[N]) {
  Words<W> v;
#pragma unroll
  for (int i = 0; i < W; ++i) {
    if constexpr (T == kF32) v.w[i] = __float_as_uint(f[i]);
    else v.w[i] = pack2(f[2 * i], f[2 * i + 1], T == kF16);
  }
  return v;
}

// The request that holds `row`, or -1: a warp narrows the offsets 32-fold a step, so that
// a batch of 1024 costs two dependent loads (bisection ten).
__device__ __forceinline__ int request_of(const int* cu, int B, int row, int lane) {
  int lo = 0, n = B;                            // among cu[lo .. lo + n - 1]
  while (n > 1) {
    const int step = (n + 31) / 32;
    const int at = lane * step;
    const unsigned below = __ballot_sync(0xffffffffu, at < n && cu[lo + at] <= row);
    const int last = below == 0 ? 0 : 31 - __clz(below);
    lo += last * step;
    n = min(step, n - last * step);
  }
  return cu[lo] <= row && row < cu[lo + 1] ? lo : -1;
}

// One pass: a row is read once and written once (turned heads to `out`, stored ones to their
// cache row); where out is x itself only the turned part moves.  Bound by HBM for many rows.
// A thread's item is 2 W words of one head: the two sides of W words' pairs, or 2 W words
// that stay as they are.  UNROLL items' loads are under way before the angles are made; the
// rows' sines lie in groups of four, neighbouring lanes' groups side by side.  17.9k rows of 32
// heads of 128, half of each turned in interleaved pairs, 293 MB, 51 us (5.8 TB/s; two items a
// thread 66, four 57); 24k rows of 32 + 8 + 8 heads into the cache, 479 MB, 77 us (6.2 TB/s); a step
// of 64 rows 2.8 and 3.6 (a call's host part is more).  The registers of three items leave four blocks on an SM; held to five or
// six blocks they spill (68, 98 us).  A pair's width is the whole head's: 17.9k rows of 32 heads of 80, ten
// pairs of each turned in halves (4-byte words), 183 MB, 87 us; 32 heads of 128 in fp32, 587 MB, 90.
// seer_kv_append keeps its own kernel (whole heads, half layout, no shift): of 1000 rows into the cache
// 6.4 us where this one takes 7.0 (64 rows 4.1 and 3.7, 17.9k rows 73.2 and 73.8).
template <int T, int W, bool INTER>
__global__ void __launch_bounds__(kRotThreads) rotate_kernel(const RotateArgs a, const __grid_constant__ TurnRates rates) {
  pdl_enter();
  constexpr int es = T == kF32 ? 4 : 2, N = 4 * W / es;      // values of W words
  constexpr int Q = N < 4 ? N : 4, UNROLL = kUnroll, ROW = 64;
  __shared__ __align__(16) float cosines[kRotRows][ROW], sines[kRotRows][ROW];
  __shared__ long long positions[kRotRows];
  __shared__ int slots[kRotRows];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int M = a.M_dev ? *a.M_dev : a.T_cap;
  if (M < 0 || M > a.T_cap) {
    if (blockIdx.x == 0 && threadIdx.x == 0) record_error(a.err, kErrRows);
    M = M < 0 ? 0 : a.T_cap;
  }
  const int dh = a.head_dim, turning = (a.half + N - 1) / N;  // items of a head that turn
  const bool in_place = a.out == a.x;
  // in place without a cache nothing but the turning items is needed
  const int per_head = in_place && a.n_plain == 0 && a.slot == nullptr ? turning : dh / (2 * N);
  const int items = (a.n_turned + a.n_plain) * per_head;
  const long kv_row = static_cast<long>(a.n_turned + a.n_plain - a.first_stored) * dh * es;
  const int G = a.rows_per_block;
  for (int row0 = blockIdx.x * G; row0 < M; row0 += gridDim.x * G) {
    const int rows = min(G, M - row0);
    bool tables = false;
    for (int j0 = threadIdx.x; !tables || j0 - static_cast<int>(threadIdx.x) < rows * items; j0 += UNROLL * kRotThreads) {
      Words<W> lo[UNROLL], hi[UNROLL];
      int row[UNROLL], head[UNROLL], chunk[UNROLL];
      const auto offsets = [&](int h, int c, long& x, long& y) {
        if (!INTER && c < turning && h < a.n_turned) {
          x = static_cast<long>(c) * N;
          y = x + a.half;
        } else {
          x = !INTER && h < a.n_turned ? 2l * a.half + 2l * (c - turning) * N : 2l * c * N;
          y = x + N;
        }
        x = (x + static_cast<long>(h) * dh) * es;
        y = (y + static_cast<long>(h) * dh) * es;
      };
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) {
        const int j = j0 + u * kRotThreads;
        row[u] = j / items;
        const int it = j - row[u] * items;
        head[u] = it / per_head;
        chunk[u] = it - head[u] * per_head;
        const bool turned = head[u] < a.n_turned && chunk[u] < turning;
        const bool wanted = row[u] < rows && (turned || (head[u] < a.n_turned && a.out && !in_place) || (a.slot && head[u] >= a.first_stored));
        if (!wanted) {
          row[u] = -1;
          continue;
        }
        long x, y;
        offsets(head[u], chunk[u], x, y);
        const uint8_t* src = a.x + static_cast<size_t>(row0 + row[u]) * a.ld;
        lo[u] = load_words<W>(src + x);
        hi[u] = load_words<W>(src + y);
      }
      if (!tables) {
        tables = true;
        __syncthreads();                          // the rows before are done with the tables
        if (warp < rows) {
          const int r = row0 + warp;
          long long p = a.position ? a.position[r] : 0;
          int s = a.slot ? a.slot[r] : -1;
          if (a.shift) {
            const int b = request_of(a.cu, a.B, r, lane);
            if (b >= 0) p += a.shift[b];
          }
          if (s < -1 || s >= a.pool_rows) {
            if (lane == 0) record_error(a.err, kErrLayout);
            s = -1;
          }
          if (lane == 0) {
            positions[warp] = p;
            slots[warp] = s;
          }
        }
        __syncthreads();
        for (int j = threadIdx.x; j < rows * a.half; j += kRotThreads) {
          const int r = j / a.half, i = j - r * a.half, c = i / N, e = i % N;
          const uint64_t part = static_cast<uint64_t>(positions[r]) * rates.rate[i];
          float sn, cs;
          sincospif(static_cast<float>(static_cast<int64_t>(part)) * 0x1p-63f, &sn, &cs);
          const int at = (e / Q) * (ROW / N * Q) + c * Q + e % Q;
          cosines[r][at] = cs * a.magnitude;
          sines[r][at] = sn * a.magnitude;
        }
        __syncthreads();
      }
#pragma unroll
      for (int u = 0; u < UNROLL; ++u) {
        if (row[u] < 0) continue;
        const int r = row[u], c = chunk[u];
        const bool turned = head[u] < a.n_turned;
        if (turned && c < turning) {
          float x[N], y[N];
          unpack<T>(lo[u], x);
          unpack<T>(hi[u], y);
#pragma unroll
          for (int e = 0; e < N; ++e) {
            const int at = (e / Q) * (ROW / N * Q) + c * Q + e % Q;
            const float cs = cosines[r][at], sn = sines[r][at];
            // interleaved: pair e of the item lies in its first or second half
            float& p = INTER ? (2 * e < N ? x[2 * e % N] : y[2 * e % N]) : x[e];
            float& w = INTER ? (2 * e < N ? x[2 * e % N + 1] : y[2 * e % N + 1]) : y[e];
            const float p0 = p, w0 = w;
            if (!INTER || c * N + e < a.half) {    // an interleaved item may end behind the last pair
              p = fmaf(p0, cs, -w0 * sn);
              w = fmaf(w0, cs, p0 * sn);
            }
          }
          lo[u] = pack<T, W>(x);
          hi[u] = pack<T, W>(y);
          if (INTER && (c + 1) * N > a.half) {
            // what does not turn keeps its bits, a NaN's too: read again, as few items end so and holding
            // every item's words cost a quarter of the speed
            long xo, yo;
            offsets(head[u], c, xo, yo);
            const uint8_t* src = a.x + static_cast<size_t>(row0 + r) * a.ld;
#pragma unroll
            for (int i = 0; i < W; ++i) {
              if (c * N + i * 4 / (2 * es) >= a.half) lo[u].w[i] = *reinterpret_cast<const uint32_t*>(src + xo + 4 * i);
              if (c * N + (W + i) * 4 / (2 * es) >= a.half) hi[u].w[i] = *reinterpret_cast<const uint32_t*>(src + yo + 4 * i);
            }
          }
        }
        long xo, yo;
        offsets(head[u], c, xo, yo);
        if (turned && a.out && (!in_place || c < turning)) {
          uint8_t* dst = a.out + static_cast<size_t>(row0 + r) * a.ld_out;
          store_words<W>(dst + xo, lo[u]);
          store_words<W>(dst + yo, hi[u]);
        }
        if (head[u] >= a.first_stored && slots[r] >= 0) {
          uint8_t* dst = static_cast<uint8_t*>(a.kv) + static_cast<size_t>(slots[r]) * kv_row - static_cast<long>(a.first_stored) * dh * es;
          store_words<W>(dst + xo, lo[u]);
          store_words<W>(dst + yo, hi[u]);
        }
      }
    }
  }
}

}  // namespace

cudaError_t launch_rotate(int type, bool interleaved, const RotateArgs& args, const TurnRates& rates, int num_sms,
                          cudaStream_t st) {
  if (args.T_cap <= 0) return cudaSuccess;
  RotateArgs a = args;
  // the widest words that both sides of a pair are aligned to
  const int es = type == kF32 ? 4 : 2, side = a.half * es;
  const int words = interleaved || side % 16 == 0 ? 4 : (side % 8 == 0 ? 2 : 1);
  // rows of a block: those whose items fill its threads' loads best (32 heads of 128: three rows 51
  // us, four 53)
  a.rows_per_block = 1;
  if (a.T_cap >= 2 * kRotRows * num_sms) {
    const int pair = 2 * 4 * words / es, round = kUnroll * kRotThreads;
    const bool turning = a.out == a.x && a.n_plain == 0 && a.slot == nullptr;
    const int items = (a.n_turned + a.n_plain) * (turning ? (2 * a.half + pair - 1) / pair : a.head_dim / pair);
    double best = 0;
    for (int rows = kRotRows; rows >= 1; --rows) {
      const double used = static_cast<double>(rows * items) / ((rows * items + round - 1) / round * round);
      if (used > best + 0.01) {
        best = used;
        a.rows_per_block = rows;
      }
    }
  }
  const int groups = (a.T_cap + a.rows_per_block - 1) / a.rows_per_block;
  const dim3 grid(groups < 8 * num_sms ? groups : 8 * num_sms);
#define SEER_ROTATE(T, W, I) \
  if (type == T && words == W && interleaved == I) return launch_kernel(rotate_kernel<T, W, I>, grid, dim3(kRotThreads), 0, st, a, rates);
#define SEER_ROTATE_TYPE(T) \
  SEER_ROTATE(T, 4, true)   \
  SEER_ROTATE(T, 4, false)  \
  SEER_ROTATE(T, 2, false)  \
  SEER_ROTATE(T, 1, false)
  SEER_ROTATE_TYPE(kF32)
  SEER_ROTATE_TYPE(kBF16)
  SEER_ROTATE_TYPE(kF16)
#undef SEER_ROTATE_TYPE
#undef SEER_ROTATE
  return cudaErrorInvalidValue;
}

}  // namespace seer
