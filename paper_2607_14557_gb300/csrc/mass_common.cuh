// What the kernels of the attention mass share: requests as they check them, the line of key
// tiles that runs are cut from, and the arithmetic of joined softmax sums.
#pragma once

#include <math.h>

#include "attn_math.cuh"
#include "budget.h"
#include "common.cuh"

namespace seer {

struct MassRequest {
  int q0, rows;           // its first row of q, and how many the batch gives it
  int n, look, kv;        // new rows, those that look, keys
  bool good;
};
__device__ __forceinline__ MassRequest read_request(const MassArgs& a, int b) {
  MassRequest r{};
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

// A request's keys in one 64-bit sum with what its last tile lacks of TILE keys (at most 127 of each
// of 16384 requests: 21 bits), from which both the keys of all requests and their tiles follow.  The keys
// of 1024 requests, each at most kMaxKeys, and a sum that was cut stay below 2^63.
constexpr int kLackBits = 21;
template <int TILE>
__device__ __forceinline__ long long pack_keys(int kv) {
  return static_cast<long long>(kv) << kLackBits | (-kv & (TILE - 1));
}
template <int TILE>
__device__ __forceinline__ long long tiles_in(long long sum) {
  return static_cast<unsigned long long>((sum >> kLackBits) + (sum & ((1 << kLackBits) - 1))) / TILE;
}
__device__ __forceinline__ bool within(long long sum, int T_kv_cap) { return (sum >> kLackBits) <= T_kv_cap; }
// A sum past the capacity stays past it, and is let grow no further.
__device__ __forceinline__ long long cut_sum(long long sum, int T_kv_cap) { return min(sum, (T_kv_cap + 1ll) << kLackBits); }

// The request of place x on a line, first[b] the places before request b: by a whole warp, the
// prefix sums narrowed 128-fold a step (four loads a lane, one after the other's heels).
__device__ __forceinline__ int request_at(const int* first, int B, int x) {
  const int lane = threadIdx.x & 31;
  int b = 0, left = B;
#pragma unroll 1
  while (left > 1) {
    const int hop = (left + 127) / 128;
    int below = 0;                              // of 128 starts, those at or before x
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int k = (4 * lane + e) * hop;
      below += k < left && first[b + k] <= x;
    }
    const int last = __reduce_add_sync(0xffffffffu, below) - 1;     // (first[b] <= x)
    b += last * hop;
    left = min(hop, left - last * hop);
  }
  return b;
}
// Places of a run: `total` places cut into at most n equal runs, the last one shorter.  Run c holds
// places [c * run, (c + 1) * run), so a place's run is one 32-bit division (total < 2^31).
__device__ __forceinline__ int run_length(int total, int n) { return max(1, (total + n - 1) / n); }

// Row of q of a request's i-th looking row, or -1 (an accepted entry outside the draft).
__device__ __forceinline__ int query_row(const MassArgs& a, const MassRequest& r, int b, int i, bool report) {
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
// Eight more at once: one maximum, then independent terms.
__device__ __forceinline__ float2 join8(float2 x, const float2 (&y)[8]) {
  float m = x.x;
#pragma unroll
  for (int e = 0; e < 8; ++e) m = fmaxf(m, y[e].x);
  const float base = m == -INFINITY ? 0.f : m;
  float l = x.y * ex2(x.x - base);
#pragma unroll
  for (int e = 0; e < 8; ++e) l = fmaf(y[e].y, ex2(y[e].x - base), l);
  return make_float2(m, l);
}
// (m, 1 / l) as the weights take it: 2^(s - m) / l.  The reciprocal is off by at most 2^-23 of itself.
__device__ __forceinline__ float2 finish(float2 x) {
  float inv;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(x.y));
  return make_float2(x.x == -INFINITY ? 0.f : x.x, inv);
}

// Key t's new weight into the matrices; what it adds to is read before.
__device__ __forceinline__ float old_mass(const MassArgs& a, const MassRequest& r, int b, int t) {
  return t < r.kv - r.n && a.keep != 0.f ? a.mass_in[static_cast<size_t>(b) * a.ld_mass + t] : 0.f;
}
__device__ __forceinline__ void store_mass(const MassArgs& a, const MassRequest& r, int b, int t, float w, float old) {
  const size_t at = static_cast<size_t>(b) * a.ld_mass + t;
  a.mass_out[at] = fmaf(a.keep, old, w);
  if (a.birth && t >= r.kv - r.n) a.birth[at] = t + (a.gone ? a.gone[b] : 0);
}

}  // namespace seer
