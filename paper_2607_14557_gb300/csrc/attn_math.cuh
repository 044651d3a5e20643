// Arithmetic of the tensor-core attention kernels' softmax warps.
#pragma once

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

// The largest magnitude of the 16-bit values seen, NaN included, two at a time.
template <bool F16>
__device__ __forceinline__ uint32_t max_abs2(uint32_t m, uint32_t w) {
  uint32_t d;
  w &= 0x7fff7fffu;
  if (F16) asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(d) : "r"(m), "r"(w));
  else asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(m), "r"(w));
  return d;
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
