// Arithmetic of the tensor-core attention kernels' softmax warps.
#pragma once

#include <math.h>

#include "common.cuh"

namespace seer {

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float y;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}

// 2^x of two packed f16 values in one MUFU operation.
__device__ __forceinline__ uint32_t ex2_h2(uint32_t x) {
  uint32_t y;
  asm("ex2.approx.f16x2 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// acc + the low / high 16-bit half of v (f16 or bf16), in fp32: one mixed-precision
// addition each.
template <bool F16>
__device__ __forceinline__ float add_lo16(uint32_t v, float acc) {
  float d;
  if (F16) asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tadd.rn.f32.f16 %0, l, %2;\n\t}" : "=f"(d) : "r"(v), "f"(acc));
  else asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tadd.rn.f32.bf16 %0, l, %2;\n\t}" : "=f"(d) : "r"(v), "f"(acc));
  return d;
}
template <bool F16>
__device__ __forceinline__ float add_hi16(uint32_t v, float acc) {
  float d;
  if (F16) asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tadd.rn.f32.f16 %0, h, %2;\n\t}" : "=f"(d) : "r"(v), "f"(acc));
  else asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tadd.rn.f32.bf16 %0, h, %2;\n\t}" : "=f"(d) : "r"(v), "f"(acc));
  return d;
}

// Two fp32 fused multiply-adds in one instruction (packed f32x2, sm_100+).
__device__ __forceinline__ void ffma2(float a0, float a1, float b0, float b1, float c0, float c1, float& d0, float& d1) {
  asm("{\n\t.reg .b64 ra, rb, rc, rd;\n\t"
      "mov.b64 ra, {%2, %3};\n\t"
      "mov.b64 rb, {%4, %5};\n\t"
      "mov.b64 rc, {%6, %7};\n\t"
      "fma.rn.f32x2 rd, ra, rb, rc;\n\t"
      "mov.b64 {%0, %1}, rd;\n\t}"
      : "=f"(d0), "=f"(d1) : "f"(a0), "f"(a1), "f"(b0), "f"(b1), "f"(c0), "f"(c1));
}

// (s0, s1) += (a0, a1) in one instruction.
__device__ __forceinline__ void fadd2(float& s0, float& s1, float a0, float a1) {
  asm("{\n\t.reg .b64 ra, rb;\n\t"
      "mov.b64 ra, {%0, %1};\n\t"
      "mov.b64 rb, {%2, %3};\n\t"
      "add.rn.f32x2 ra, ra, rb;\n\t"
      "mov.b64 {%0, %1}, ra;\n\t}"
      : "+f"(s0), "+f"(s1) : "f"(a0), "f"(a1));
}

// The largest magnitude of the 16-bit values seen, NaN included, two at a time.
template <bool F16>
__device__ __forceinline__ uint32_t max_abs2(uint32_t m, uint32_t w) {
  uint32_t d;
  w &= 0x7fff7fffu;
  if (F16) asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(d) : "r"(m), "r"(w));
  else asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(m), "r"(w));
  return d;
}

// A key of a row: its key and value heads, or zeros where k is null.
struct KeyAt {
  const uint16_t *k, *v;
  bool seen;
};
// A row's running maximum (log2 units), weight and unnormalised sums; a lane holds columns
// [lane * DH / 32, (lane + 1) * DH / 32).
template <int DH>
struct RowSums {
  float m = -INFINITY, l = 0.f;
  float acc[DH / 32] = {};
};
template <bool F16, int DH>
__device__ __forceinline__ void load_columns(const uint16_t* row, int lane, float (&f)[DH / 32]) {
  static_assert(DH == 64 || DH == 128, "two or four columns a lane");
  uint32_t w[DH / 64];
  if constexpr (DH == 128) *reinterpret_cast<uint2*>(w) = reinterpret_cast<const uint2*>(row)[lane];
  else w[0] = reinterpret_cast<const uint32_t*>(row)[lane];
#pragma unroll
  for (int e = 0; e < DH / 64; ++e) {
    f[2 * e] = lo16(w[e], F16);
    f[2 * e + 1] = hi16(w[e], F16);
  }
}

// One row over keys [begin, end) by a warp, in fp32 from global memory: for rows whose tile
// holds a value that is infinite or NaN and that not every row sees, which the MMA would
// multiply by the hidden rows' P = 0.  at(j): key j.  One pass, eight keys' loads at a time; it
// ends early where nothing but NaN can come out.  47 ms for 256 rows of 11.8k keys on one SM.
template <bool F16, int DH, typename At>
__device__ __forceinline__ RowSums<DH> attend_row(const uint16_t* q, int begin, int end, const At& at, int lane) {
  constexpr int N = DH / 32, KEYS = 8;
  const float scale_log2 = 1.4426950408889634f / sqrtf(static_cast<float>(DH));
  RowSums<DH> r;
  float qf[N];
  load_columns<F16, DH>(q, lane, qf);
  for (int j0 = begin; j0 < end; j0 += KEYS) {
    float s[KEYS], v[KEYS][N];
    bool seen[KEYS];
#pragma unroll
    for (int e = 0; e < KEYS; ++e) {
      const KeyAt key = j0 + e < end ? at(j0 + e) : KeyAt{nullptr, nullptr, false};
      float k[N] = {};
      seen[e] = key.seen;
#pragma unroll
      for (int n = 0; n < N; ++n) v[e][n] = 0.f;
      if (key.k != nullptr) {
        load_columns<F16, DH>(key.k, lane, k);
        load_columns<F16, DH>(key.v, lane, v[e]);
      }
      s[e] = 0.f;
#pragma unroll
      for (int n = 0; n < N; ++n) s[e] = fmaf(qf[n], k[n], s[e]);
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1)
#pragma unroll
      for (int e = 0; e < KEYS; ++e) s[e] += __shfl_xor_sync(0xffffffffu, s[e], off);
    float top = r.m;
#pragma unroll
    for (int e = 0; e < KEYS; ++e) {
      s[e] = seen[e] ? s[e] * scale_log2 : -INFINITY;
      top = fmaxf(top, s[e]);
    }
    const float base = top == -INFINITY ? 0.f : top;       // nothing seen so far: every term is 0
    const float alpha = ex2(r.m - base);
    r.m = top;
    r.l *= alpha;
#pragma unroll
    for (int n = 0; n < N; ++n) r.acc[n] *= alpha;
#pragma unroll
    for (int e = 0; e < KEYS; ++e) {
      if (!seen[e]) continue;                              // a hidden value is not even multiplied
      const float w = ex2(s[e] - base);
      r.l += w;
#pragma unroll
      for (int n = 0; n < N; ++n) r.acc[n] = fmaf(w, v[e][n], r.acc[n]);
    }
    bool lost = true;                                      // every column is NaN, and stays so
#pragma unroll
    for (int n = 0; n < N; ++n) lost = lost && isnan(r.acc[n]);
    if (__all_sync(0xffffffffu, lost || isnan(r.l))) {
      r.l = __int_as_float(0x7fffffff);
      break;
    }
  }
  return r;
}

// A warp's 32 output rows, a row per lane, stored 32 columns at a time: the four lanes of a
// quad trade 16-byte pieces by shuffles, so that one instruction stores 64 bytes of each of
// eight rows.  Every lane storing its own row touched 32 lines an instruction (a ragged
// causal batch 114 us, so 104); through shared memory instead of shuffles the pieces wait
// for the MMAs' operand reads (4 KB a warp: 107, its epilogue 2.0 us against 1.3).
struct RowStore {
  uint16_t* row[4];                   // the quad's rows at this lane's 16 bytes, or null

  // out + off: the lane's row, where ok.
  __device__ __forceinline__ void set(void* out, long long off, bool ok, int lane) {
    const uint32_t stored = __ballot_sync(0xffffffffu, ok);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int src = (lane & ~3) + q;
      const long long at = __shfl_sync(0xffffffffu, off, src);
      row[q] = (stored >> src) & 1u ? static_cast<uint16_t*>(out) + at + 8 * (lane & 3) : nullptr;
    }
  }
  // v: columns [col, col + 32) of the lane's row.
  __device__ __forceinline__ void put(uint4 (&v)[4], int col, int lane) const {
    const auto trade = [&](uint4& a, uint4& b, int bit) {
      const bool up = (lane & bit) != 0;
      const uint4 give = up ? a : b;
      uint4 got;
      got.x = __shfl_xor_sync(0xffffffffu, give.x, bit);
      got.y = __shfl_xor_sync(0xffffffffu, give.y, bit);
      got.z = __shfl_xor_sync(0xffffffffu, give.z, bit);
      got.w = __shfl_xor_sync(0xffffffffu, give.w, bit);
      if (up) a = got;
      else b = got;
    };
    trade(v[0], v[1], 1);
    trade(v[2], v[3], 1);
    trade(v[0], v[2], 2);
    trade(v[1], v[3], 2);
#pragma unroll
    for (int q = 0; q < 4; ++q)       // v[q]: piece lane % 4 of the quad's row q
      if (row[q]) *reinterpret_cast<uint4*>(row[q] + col) = v[q];
  }
};

}  // namespace seer
