// Causal attention over packed prompts with grouped heads on tcgen05 for sm_103a
// (head_dim 64 or 128; q, k, v, the probabilities P and the output all f16, or all bf16).
//   o_i = sum_{j <= i} p_ij v_j / sum_{j <= i} p_ij,  p_ij = 2^(s_ij - m_i),
//   s_ij = q_i k_j log2(e) / sqrt(dh),  m_i a running maximum
//
// The g = n_heads / n_kv query heads that share a key/value head are rows of one tile: a
// tile is the g heads of floor(128 / g) consecutive tokens (row = token * g + head, a
// three-dimensional TMA box of q), so a key tile is read once for all of them and the
// causal edge costs a tile of 128 / g tokens, not of 128.  A unit is two such tiles and
// the key tiles up to its last token; both tiles run over the same key tiles, and scores
// past a row's token are dropped in the last ones.
//
// Persistent CTAs, one per SM; the pipeline is that of the bidirectional kernel
// (tc_attn.cu), whose comments give the reasons for its parts:
//   warp 0      TMA producer: Q tiles of a unit, then K_j and V_j in turn (2-deep rings)
//   warps 1, 2  MMA issuers of the two tiles, passing a turn token
//   warp 3      scheduler: decodes this CTA's units and publishes them in a shared ring
//   warps 4-11  softmax of the two tiles, a thread per row; O rescaled in tensor memory
//               only where a row's maximum grew by more than 2^8
// Units in order of descending token group g (their cost grows with g alone), dealt to the
// CTAs in alternating direction: no list, counter or workspace, and concurrent or captured
// calls share nothing.  The scheduler walks the groups once, counting the sequences that
// reach each.
//
// Bound by the softmax chain of the two tiles (a round of both takes 1.36 us against 1.09 of
// MMA work) and ~2.4 us at a unit's end: one prompt of 11792 rows, 32 / 8 heads of 128, 1.14
// TFLOP in 0.64 to 0.76 ms over boxes and power (1510 to 1770 TFLOP/s), 16 prompts of 83 .. 1693
// rows, 0.11 TFLOP, in 103 to 109 us.
//
// P is exponentiated in fp32 and rounded to the 16-bit type that the PV MMA reads; the row
// sums add the rounded values, so numerator and normaliser carry the same rounding.
// A key that a row does not see has P = 0, which an infinite or NaN value row would still
// turn into NaN in the MMA.  So value rows past the unit's last token are cleared, and the
// rows of a unit with a non-finite value in a masked tile are left to recompute_units() after
// the last unit, when no wait with a time limit is pending.
#include <math.h>

#include "attn_math.cuh"
#include "common.cuh"
#include "paged.h"

namespace seer {
namespace {

constexpr int BQ = 128;                     // rows of a tile
constexpr int BKV = 128;                    // keys of a tile
constexpr int NT = 2;                       // tiles of a unit
constexpr int THREADS = 128 + 128 * NT;
constexpr int PANEL = 16384;                // 128 rows x 64 values, 128-byte swizzle
constexpr int STAGES = 2;                   // K ring and V ring
constexpr int BAR_BYTES = 512;
constexpr uint32_t TMEM_COLS = 512;
constexpr uint32_t TM_S = 0;                // S_t at TM_S + 128 t
constexpr uint32_t TM_O = 256;              // O_t at TM_O + 128 t
constexpr float RESCALE_THRESHOLD = 8.0f;   // log2 units
constexpr int U_SLOTS = 4;                  // units published ahead
constexpr int U_READERS = 1 + NT + 4 * NT;  // producer, issuers, softmax warps

template <int DH>
struct Layout {
  static constexpr int TILE = 128 * DH * 2;
  static constexpr int OFF_Q = 0;
  static constexpr int OFF_K = NT * TILE;
  static constexpr int OFF_V = OFF_K + STAGES * TILE;
  static constexpr int OFF_BAR = OFF_V + STAGES * TILE;
  static constexpr int BYTES = OFF_BAR + BAR_BYTES + 1024;
};
// up to 199680 bytes leave 60 KB of the SM to L1
static_assert(Layout<128>::BYTES <= 199680, "L1 carve-out");
// barriers, the unit ring, the odd-value marks, the TMEM base and the abort flag
static_assert(8 * (2 + 4 * STAGES + 6 * NT + 2 * U_SLOTS) + 16 * U_SLOTS + 16 * NT + 8 <= BAR_BYTES, "barrier block");

// seq0 < 0: no more units.
struct Unit {
  int seq0, L, tok0, kvh;
};
struct Span {
  int nt, nkv, kend;                        // tiles, key tiles, keys
};
__device__ __forceinline__ Span span_of(const Unit& u, int tpt) {
  Span s;
  s.nt = u.tok0 + tpt < u.L ? 2 : 1;
  s.kend = min(u.L, u.tok0 + s.nt * tpt);
  s.nkv = (s.kend + BKV - 1) / BKV;
  return s;
}

// This CTA's i-th unit from the ring, by a whole warp (see read_unit in tc_attn.cu).
__device__ __forceinline__ Unit read_unit(uint64_t* u_full, uint64_t* u_empty, const int4* ring, int i,
                                          volatile int* abort, int* err, int lane) {
  const int s = i % U_SLOTS;
  const bool ok = warp_wait(&u_full[s], (i / U_SLOTS) & 1, abort, err);
  const int4 w = ok ? ring[s] : make_int4(-1, 0, 0, 0);
  __syncwarp();
  if (lane == 0 && ok) mbar_arrive(&u_empty[s]);
  return Unit{w.x, w.y, w.z, w.w};
}

// This CTA's units, by a whole warp: units in order of descending token group, the sequences that
// reach a group counted once on the way.
struct UnitWalk {
  int span, H, lane;
  int mine;                                 // units per head of sequence `lane`: the first 32 stay in registers
  long total;
  int g;                                    // units of group g: [base, base + count)
  long base = 0, count = 0;
  int b0 = 0, passed = 0;                   // sequences b0 .. hold the next unit; so many before them reach g

  // Units of sequence b per head; 0 where it leaves the buffers.
  __device__ __forceinline__ int groups_of(const GqaParams& p, int b, bool report) const {
    if (b >= p.B) return 0;
    const int c0 = p.cu[b], c1 = p.cu[b + 1];
    const bool good = c0 >= 0 && c1 >= c0 && c1 <= p.T_cap;
    if (!good && report) record_error(p.err, kErrLayout);
    return good ? (c1 - c0 + span - 1) / span : 0;
  }
  // Which of sequences x .. x + 31 have a group g.
  __device__ __forceinline__ uint32_t reach(const GqaParams& p, int x) const {
    const int n = x == 0 ? mine : groups_of(p, x + lane, false);
    return __ballot_sync(0xffffffffu, n > g);
  }
  __device__ __forceinline__ UnitWalk(const GqaParams& p, int tpt, int lane_, bool report) : span(NT * tpt), H(p.n_kv), lane(lane_) {
    mine = groups_of(p, lane, report);
    int most = mine, sum = mine;
    for (int b = lane + 32; b < p.B; b += 32) {
      const int n = groups_of(p, b, report);
      most = max(most, n);
      sum += n;
    }
    g = __reduce_max_sync(0xffffffffu, most);
    total = static_cast<long>(__reduce_add_sync(0xffffffffu, sum)) * H;
  }
  // The CTA's i-th unit, i ascending; seq0 < 0 past its last.
  __device__ __forceinline__ int4 unit(const GqaParams& p, int i) {
    const int grid = gridDim.x;
    const long u = (i & 1) ? (i + 1l) * grid - 1 - blockIdx.x : static_cast<long>(i) * grid + blockIdx.x;
    if (u >= total) return make_int4(-1, 0, 0, 0);
    while (u >= base + count) {
      base += count;
      --g;
      int n = 0;
      for (int x = 0; x < p.B; x += 32) n += __popc(reach(p, x));
      count = static_cast<long>(n) * H;
      b0 = passed = 0;
    }
    const int k = static_cast<int>(u - base), nth = k / H;
    int b = 0;
    for (; b0 < p.B; b0 += 32) {            // a group's units come in order, so this goes on where it stopped
      const uint32_t m = reach(p, b0);
      if (nth - passed < __popc(m)) {
        b = b0 + __fns(m, 0, nth - passed + 1);
        break;
      }
      passed += __popc(m);
    }
    return make_int4(p.cu[b], p.cu[b + 1] - p.cu[b], g * span, k % H);
  }
};

// The rows that a non-finite value in a masked tile may have reached, from global memory by
// every warp of the CTA.  Its units are looked over once more, so that none need be remembered.
template <bool F16, int DH>
__device__ __noinline__ void recompute_units(const GqaParams& p) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int G = p.n_heads / p.n_kv, TPT = BQ / G;
  UnitWalk walk(p, TPT, lane, false);
  uint32_t nonfinite = 0;
  for (int i = 0;; ++i) {
    const int4 w = walk.unit(p, i);
    if (w.x < 0) break;
    const Unit u{w.x, w.y, w.z, w.w};
    const Span d = span_of(u, TPT);
    const uint16_t* k = static_cast<const uint16_t*>(p.k) + static_cast<size_t>(u.seq0) * p.ld_k + u.kvh * DH;
    const uint16_t* v = static_cast<const uint16_t*>(p.v) + static_cast<size_t>(u.seq0) * p.ld_v + u.kvh * DH;
    for (int t = 0; t < d.nt; ++t) {
      const int first = u.tok0 + t * TPT, tokens = min(TPT, u.L - first);
      const int masked = (first + 1) / BKV * BKV;          // first key of the masked key tiles
      uint32_t bad = 0;
      for (int x = threadIdx.x; x < (d.kend - masked) * (DH / 8); x += THREADS) {
        const uint4 a = reinterpret_cast<const uint4*>(v + static_cast<size_t>(masked + x / (DH / 8)) * p.ld_v)[x % (DH / 8)];
        bad |= nonfinite_term(a.x, F16) | nonfinite_term(a.y, F16) | nonfinite_term(a.z, F16) | nonfinite_term(a.w, F16);
      }
      if (!__syncthreads_or((bad & 0x80008000u) != 0)) continue;
      for (int r = warp; r < tokens * G; r += THREADS / 32) {
        const int tok = first + r / G, head = u.kvh * G + r % G;
        const uint16_t* q = static_cast<const uint16_t*>(p.q) + static_cast<size_t>(u.seq0 + tok) * p.ld_q + head * DH;
        const auto at = [&](int j) { return KeyAt{k + static_cast<size_t>(j) * p.ld_k, v + static_cast<size_t>(j) * p.ld_v, true}; };
        const RowSums<DH> sums = attend_row<F16, DH>(q, 0, tok + 1, at, lane);
        const float inv = sums.l == 0.f ? 0.f : 1.f / sums.l;
        uint32_t* o = reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(p.o) + static_cast<size_t>(u.seq0 + tok) * p.ld_o + head * DH);
#pragma unroll
        for (int e = 0; e < DH / 64; ++e) {
          const uint32_t x = pack2(sums.acc[2 * e] * inv, sums.acc[2 * e + 1] * inv, F16);
          nonfinite |= nonfinite_term(x, F16);
          o[lane * (DH / 64) + e] = x;
        }
      }
    }
  }
  report_range(nonfinite, p.err);
}

template <bool F16, int DH>
__global__ void __launch_bounds__(THREADS, 1)
    tc_causal_kernel(const __grid_constant__ CUtensorMap mQ, const __grid_constant__ CUtensorMap mK,
                     const __grid_constant__ CUtensorMap mV, const GqaParams p) {
  using Lay = Layout<DH>;
  constexpr int TILE = Lay::TILE, PANELS = DH / 64;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + Lay::OFF_BAR);
  uint64_t* q_full = bars + 0;
  uint64_t* q_empty = bars + 1;
  uint64_t* k_full = bars + 2;               // [STAGES]
  uint64_t* k_empty = k_full + STAGES;
  uint64_t* v_full = k_empty + STAGES;
  uint64_t* v_empty = v_full + STAGES;
  uint64_t* s_full = v_empty + STAGES;       // [NT] S_t,j written (and O_t += P_t,j-1 V done)
  uint64_t* p_full = s_full + NT;            // [NT] P_t,j of keys 0..63 in tensor memory
  uint64_t* p_full2 = p_full + NT;           // [NT] P_t,j of keys 64..127 in tensor memory
  uint64_t* o_done = p_full2 + NT;           // [NT] last PV of a unit's tile complete
  uint64_t* o_free = o_done + NT;            // [NT] O_t read out by the softmax warps
  uint64_t* turn = o_free + NT;              // [NT] issuer t may enqueue its next round
  uint64_t* u_full = turn + NT;              // [U_SLOTS]
  uint64_t* u_empty = u_full + U_SLOTS;      // [U_SLOTS]
  int4* ring = reinterpret_cast<int4*>(u_empty + U_SLOTS);       // [U_SLOTS]
  // [NT][4]: i + 1 in slot i % 4 where the CTA's i-th unit met a non-finite value in a
  // masked tile (a warp is at most one unit ahead of the others of its tile)
  volatile int* odd = reinterpret_cast<volatile int*>(ring + U_SLOTS);
  uint32_t* tmem_slot = const_cast<uint32_t*>(reinterpret_cast<volatile uint32_t*>(odd + 4 * NT));
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

  const int warp = threadIdx.x >> 5;
  const int lane = threadIdx.x & 31;
  const int G = p.n_heads / p.n_kv, TPT = BQ / G;

  // barriers and tensor memory, before the kernels ahead are waited for
  if (threadIdx.x == 0) {
    tma_prefetch_desc(&mQ);
    tma_prefetch_desc(&mK);
    tma_prefetch_desc(&mV);
    mbar_init(q_full, 1);
    mbar_init(q_empty, NT);
    for (int i = 0; i < STAGES; ++i) {
      mbar_init(&k_full[i], 1);
      mbar_init(&k_empty[i], NT);
      mbar_init(&v_full[i], 1);
      mbar_init(&v_empty[i], NT);
    }
    for (int t = 0; t < NT; ++t) {
      mbar_init(&s_full[t], 1);
      mbar_init(&p_full[t], 4);
      mbar_init(&p_full2[t], 4);
      mbar_init(&o_done[t], 1);
      mbar_init(&o_free[t], 4);
      mbar_init(&turn[t], 1);
    }
    for (int i = 0; i < U_SLOTS; ++i) {
      mbar_init(&u_full[i], 1);
      mbar_init(&u_empty[i], U_READERS);
    }
    for (int i = 0; i < 4 * NT; ++i) odd[i] = 0;
    *abort_flag = 0;
    fence_barrier_init();
  }
  if (warp == 1) tmem_alloc(tmem_slot, TMEM_COLS);
  pdl_enter();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  if (warp == 3) {
    // -------------------------------------------------- scheduler
    UnitWalk walk(p, TPT, lane, blockIdx.x == 0);
    for (int i = 0;; ++i) {
      const int s = i % U_SLOTS;
      if (i >= U_SLOTS && !warp_wait(&u_empty[s], (i / U_SLOTS - 1) & 1, abort_flag, p.err)) break;
      const int4 w = walk.unit(p, i);
      if (lane == 0) {
        ring[s] = w;
        mbar_arrive(&u_full[s]);
      }
      __syncwarp();
      if (w.x < 0) break;
    }
  } else if (warp == 0) {
    // -------------------------------------------------- TMA producer
    const bool leader = elect_one();
    int q_issued = 0, k_issued = 0, v_issued = 0;
    bool ok = true;
    for (int i = 0; ok; ++i) {
      const Unit u = read_unit(u_full, u_empty, ring, i, abort_flag, p.err, lane);
      if (u.seq0 < 0) break;
      const Span d = span_of(u, TPT);
      if (i > 0 && !warp_wait(q_empty, (i - 1) & 1, abort_flag, p.err)) break;
      if (leader) {
        mbar_arrive_expect_tx(q_full, d.nt * PANELS * TPT * G * 128);
        for (int t = 0; t < d.nt; ++t)
          for (int c = 0; c < PANELS; ++c)
            tma_load_3d(smem + Lay::OFF_Q + t * TILE + c * PANEL, &mQ, q_full, 64 * c, u.kvh * G, u.seq0 + u.tok0 + t * TPT);
      }
      __syncwarp();
      ++q_issued;
      for (int j = 0; j < d.nkv; ++j) {
        const int ks = k_issued % STAGES, ku = k_issued / STAGES;
        if (ku > 0 && !warp_wait(&k_empty[ks], (ku - 1) & 1, abort_flag, p.err)) { ok = false; break; }
        if (leader) {
          mbar_arrive_expect_tx(&k_full[ks], TILE);
          for (int c = 0; c < PANELS; ++c)
            tma_load_3d(smem + Lay::OFF_K + ks * TILE + c * PANEL, &mK, &k_full[ks], 64 * c, u.kvh, u.seq0 + j * BKV);
        }
        __syncwarp();
        ++k_issued;
        const int vs = v_issued % STAGES, vu = v_issued / STAGES;
        if (vu > 0 && !warp_wait(&v_empty[vs], (vu - 1) & 1, abort_flag, p.err)) { ok = false; break; }
        if (leader) {
          mbar_arrive_expect_tx(&v_full[vs], TILE);
          for (int c = 0; c < PANELS; ++c)
            tma_load_3d(smem + Lay::OFF_V + vs * TILE + c * PANEL, &mV, &v_full[vs], 64 * c, u.kvh, u.seq0 + j * BKV);
        }
        __syncwarp();
        ++v_issued;
      }
    }
    if (*abort_flag && leader) {
      // let copies still in flight land before the CTA's shared memory is released
      if (q_issued > 0) mbar_wait_drain(q_full, (q_issued - 1) & 1, 200000000ull);
      for (int j = k_issued > STAGES ? k_issued - STAGES : 0; j < k_issued; ++j)
        mbar_wait_drain(&k_full[j % STAGES], (j / STAGES) & 1, 200000000ull);
      for (int j = v_issued > STAGES ? v_issued - STAGES : 0; j < v_issued; ++j)
        mbar_wait_drain(&v_full[j % STAGES], (j / STAGES) & 1, 200000000ull);
    }
  } else if (warp == 1 || warp == 2) {
    // -------------------------------------------------- MMA issuer of tile t
    const int t = warp - 1;
    const bool leader = elect_one();
    constexpr uint32_t idesc_qk = make_idesc(BQ, BKV, 0, F16);
    constexpr uint32_t idesc_pv = make_idesc(BQ, DH, 1, F16);
    const uint64_t dq = make_sdesc_sw128(smem_u32(smem + Lay::OFF_Q + t * TILE), 16, 1024);
    const uint64_t dk0 = make_sdesc_sw128(smem_u32(smem + Lay::OFF_K), 16, 1024);
    const uint64_t dv0 = make_sdesc_sw128(smem_u32(smem + Lay::OFF_V), PANEL, 1024);
    const uint32_t dS = tmem + TM_S + 128 * t, dO = tmem + TM_O + 128 * t;
    unsigned kc = 0, vc = 0;       // K / V tiles consumed
    unsigned pc = 0, tc = 0;       // P tiles consumed, turn waits
    unsigned oc = 0;               // units of this tile finished
    bool paired_before = false;
    bool ok = true;
    auto qk = [&](unsigned c) {
      if (leader) {
        const uint64_t dk = dk0 + static_cast<uint64_t>((c & 1u) * (TILE >> 4));
#pragma unroll
        for (int k = 0; k < DH / 16; ++k) {
          const uint64_t off = static_cast<uint64_t>(((k >> 2) * PANEL + (k & 3) * 32) >> 4);
          tc_mma_f16(dS, dq + off, dk + off, idesc_qk, k > 0 ? 1u : 0u);
        }
        tc_commit(&s_full[t]);
        tc_commit(&k_empty[c & 1u]);
      }
      __syncwarp();
    };
    auto pv = [&](unsigned c, int vt, int half) {
      if (leader) {
        const uint64_t dv = dv0 + static_cast<uint64_t>((c & 1u) * (TILE >> 4));
#pragma unroll
        for (int kk = 0; kk < BKV / 32; ++kk) {
          const int k = half * (BKV / 32) + kk;
          tc_mma_f16_tmem_a(dO, dS + 8 * k, dv + static_cast<uint64_t>(k * 128), idesc_pv, (vt > 0 || k > 0) ? 1u : 0u);
        }
        if (half == 1) tc_commit(&v_empty[c & 1u]);
      }
      __syncwarp();
    };
    auto arrive = [&](uint64_t* bar) {
      if (leader) mbar_arrive(bar);
      __syncwarp();
    };
    for (int i = 0; ok; ++i) {
      const Unit u = read_unit(u_full, u_empty, ring, i, abort_flag, p.err, lane);
      if (u.seq0 < 0) break;
      const Span d = span_of(u, TPT);
      if (!warp_wait(q_full, i & 1, abort_flag, p.err)) break;
      if (t >= d.nt) {
        // idle this unit: release Q and every K / V stage as they pass
        arrive(q_empty);
        for (int j = 0; j < d.nkv; ++j, ++kc, ++vc) {
          if (!warp_wait(&k_full[kc & 1u], (kc >> 1) & 1u, abort_flag, p.err) ||
              !warp_wait(&v_full[vc & 1u], (vc >> 1) & 1u, abort_flag, p.err)) {
            ok = false;
            break;
          }
          arrive(&k_empty[kc & 1u]);
          arrive(&v_empty[vc & 1u]);
        }
        continue;
      }
      const bool pair = d.nt > 1;
      const int nkv = d.nkv;
      if (!warp_wait(&k_full[kc & 1u], (kc >> 1) & 1u, abort_flag, p.err)) break;
      if (pair && (t == 1 || paired_before)) {
        if (!warp_wait(&turn[t], tc & 1u, abort_flag, p.err)) break;
        ++tc;
      }
      tc_fence_after();
      qk(kc);
      ++kc;
      if (nkv == 1 && leader) tc_commit(q_empty);
      if (pair) arrive(&turn[t ^ 1]);
      if (oc > 0 && !warp_wait(&o_free[t], (oc - 1) & 1u, abort_flag, p.err)) break;
      for (int j = 1; j < nkv; ++j) {
        if (!warp_wait(&v_full[vc & 1u], (vc >> 1) & 1u, abort_flag, p.err) ||
            !warp_wait(&k_full[kc & 1u], (kc >> 1) & 1u, abort_flag, p.err) ||
            !warp_wait(&p_full[t], pc & 1u, abort_flag, p.err) ||
            (pair && !warp_wait(&turn[t], tc & 1u, abort_flag, p.err))) {
          ok = false;
          break;
        }
        tc += pair ? 1u : 0u;
        tc_fence_after();
        pv(vc, j - 1, 0);
        if (!warp_wait(&p_full2[t], pc & 1u, abort_flag, p.err)) {
          ok = false;
          break;
        }
        tc_fence_after();
        pv(vc, j - 1, 1);
        qk(kc);
        ++vc;
        ++pc;
        ++kc;
        if (pair) arrive(&turn[t ^ 1]);
      }
      if (!ok) break;
      if (nkv > 1 && leader) tc_commit(q_empty);
      if (!warp_wait(&v_full[vc & 1u], (vc >> 1) & 1u, abort_flag, p.err) ||
          !warp_wait(&p_full[t], pc & 1u, abort_flag, p.err) ||
          (pair && !warp_wait(&turn[t], tc & 1u, abort_flag, p.err)))
        break;
      tc += pair ? 1u : 0u;
      tc_fence_after();
      pv(vc, nkv - 1, 0);
      if (!warp_wait(&p_full2[t], pc & 1u, abort_flag, p.err)) break;
      tc_fence_after();
      pv(vc, nkv - 1, 1);
      if (leader) tc_commit(&o_done[t]);
      __syncwarp();
      ++vc;
      ++pc;
      if (pair) arrive(&turn[t ^ 1]);
      if (pair) paired_before = true;
      ++oc;
    }
  } else {
    // -------------------------------------------------- softmax warps 4..11
    const int t = (warp - 4) >> 2;
    const int r = (warp & 3) * 32 + lane;         // row of the tile == TMEM lane
    const int rt = r / G, rh = r - rt * G;        // its token and head inside the tile
    const uint32_t lane_off = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t tS = tmem + lane_off + TM_S + 128 * t;
    const uint32_t tO = tmem + lane_off + TM_O + 128 * t;
    const float scale_log2 = 1.4426950408889634f / sqrtf(static_cast<float>(DH));
    int cs = 0, co = 0, cv = 0;                   // S tiles seen, units done (this tile), V tiles before the unit
    uint32_t nonfinite = 0;
    bool ok = true;
    for (int i = 0; ok; ++i) {
      const Unit u = read_unit(u_full, u_empty, ring, i, abort_flag, p.err, lane);
      if (u.seq0 < 0) break;
      const Span d = span_of(u, TPT);
      if (t >= d.nt) {
        cv += d.nkv;
        continue;
      }
      const int first = u.tok0 + t * TPT, tok = first + rt;
      float m_ref = -INFINITY;
      float l = 0.f;
      for (int j = 0; ok && j < d.nkv; ++j) {
        if (!__all_sync(0xffffffffu, mbar_wait(&s_full[t], cs & 1, abort_flag, p.err))) { ok = false; break; }
        ++cs;
        tc_fence_after();
        float s[BKV];
        {
          uint32_t ra[BKV / 32][32];
#pragma unroll
          for (int cc = 0; cc < BKV / 32; ++cc) tmem_ld32(tS + 32 * cc, ra[cc]);
          tmem_ld_wait();
#pragma unroll
          for (int cc = 0; cc < BKV / 32; ++cc)
#pragma unroll
            for (int e = 0; e < 32; ++e) s[32 * cc + e] = __uint_as_float(ra[cc][e]);
        }
        const bool masked = first + 1 - j * BKV < BKV;   // the tile's first row does not see all keys
        if (masked) {
          const int seen = tok + 1 - j * BKV;
#pragma unroll
          for (int cc = 0; cc < BKV; ++cc) s[cc] = cc < seen ? s[cc] : -INFINITY;
        }
        float mx[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) mx[e] = fmaxf(s[e], s[e + 8]);
#pragma unroll
        for (int cc = 16; cc < BKV; cc += 16)
#pragma unroll
          for (int e = 0; e < 8; ++e) mx[e] = max3(mx[e], s[cc + e], s[cc + 8 + e]);
#pragma unroll
        for (int w = 4; w >= 1; w >>= 1)
#pragma unroll
          for (int e = 0; e < w; ++e) mx[e] = fmaxf(mx[e], mx[e + w]);
        const float m_new = fmaxf(m_ref, mx[0] * scale_log2);
        const bool need = (j == 0) || (m_new > m_ref + RESCALE_THRESHOLD);
        const bool any_need = __any_sync(0xffffffffu, need);
        float alpha = 1.f;
        if (need) {
          alpha = j == 0 ? 0.f : ex2(m_ref - m_new);
          m_ref = m_new;
        }
        const float neg = m_ref == -INFINITY ? 0.f : -m_ref;   // only scores of -inf so far: every term is 0
        float rs[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
#pragma unroll
          for (int cc = 2 * hf; cc < 2 * hf + 2; ++cc) {
            uint32_t pk[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              float x0, x1;
              ffma2(s[32 * cc + 2 * e], s[32 * cc + 2 * e + 1], scale_log2, scale_log2, neg, neg, x0, x1);
              pk[e] = pack2(ex2(x0), ex2(x1), F16);
              rs[(2 * e) & 3] = add_lo16<F16>(pk[e], rs[(2 * e) & 3]);
              rs[(2 * e + 1) & 3] = add_hi16<F16>(pk[e], rs[(2 * e + 1) & 3]);
            }
            tmem_st16(tS + 16 * cc, pk);
          }
          if (hf == 0) {
            if (j > 0 && any_need) {
#pragma unroll 1
              for (int cc = 0; cc < DH / 32; ++cc) {
                uint32_t rr[32];
                tmem_ld32(tO + 32 * cc, rr);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 32; ++e) rr[e] = __float_as_uint(__uint_as_float(rr[e]) * alpha);
                tmem_st32(tO + 32 * cc, rr);
              }
            }
            if (masked) {
              // value rows past the unit's keys are cleared; a non-finite one before
              // them marks the unit
              const int vsi = cv + j, vst = vsi % STAGES;
              if (!__all_sync(0xffffffffu, mbar_wait(&v_full[vst], (vsi / STAGES) & 1, abort_flag, p.err))) {
                ok = false;
                break;
              }
              const int valid = d.kend - j * BKV;
              uint4* v = reinterpret_cast<uint4*>(smem + Lay::OFF_V + vst * TILE);
              uint32_t bad = 0;
#pragma unroll 4
              for (int c = r; c < TILE / 16; c += 128) {
                if (((c >> 3) & 127) < valid) {
                  const uint4 w = v[c];
                  bad |= nonfinite_term(w.x, F16) | nonfinite_term(w.y, F16) | nonfinite_term(w.z, F16) |
                         nonfinite_term(w.w, F16);
                } else {
                  v[c] = make_uint4(0, 0, 0, 0);
                }
              }
              if (bad & 0x80008000u) odd[4 * t + (i & 3)] = i + 1;
              fence_proxy_async_smem();
            }
          }
          tmem_st_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(hf == 0 ? &p_full[t] : &p_full2[t]);
        }
        if (!ok) break;
        l = l * alpha + ((rs[0] + rs[1]) + (rs[2] + rs[3]));
      }
      if (!ok) break;
      if (!__all_sync(0xffffffffu, mbar_wait(&o_done[t], co & 1, abort_flag, p.err))) break;
      tc_fence_after();
      const float inv_l = l == 0.f ? 0.f : 1.f / l;
      const bool valid_row = rt < TPT && tok < u.L;
      const int head = u.kvh * G + rh;
      if (odd[4 * t + (i & 3)] != i + 1) {        // (else the rows are left to recompute_units())
        RowStore store;
        store.set(p.o, static_cast<long long>(u.seq0 + tok) * p.ld_o + head * DH, valid_row, lane);
        uint32_t top = 0;
#pragma unroll 1
        for (int cc = 0; cc < DH / 32; ++cc) {
          uint32_t rr[32];
          tmem_ld32(tO + 32 * cc, rr);
          tmem_ld_wait();
          uint4 v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            uint32_t q[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              float x0, x1;
              ffma2(__uint_as_float(rr[8 * e + 2 * k]), __uint_as_float(rr[8 * e + 2 * k + 1]), inv_l, inv_l, 0.f, 0.f, x0, x1);
              q[k] = pack2(x0, x1, F16);
              top = max_abs2<F16>(top, q[k]);
            }
            v[e] = make_uint4(q[0], q[1], q[2], q[3]);
          }
          store.put(v, 32 * cc, lane);
        }
        if (valid_row) nonfinite |= nonfinite_term(top, F16);
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&o_free[t]);
      ++co;
      cv += d.nkv;
    }
    report_range(nonfinite, p.err);
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, TMEM_COLS);
  }
  int any = 0;
  for (int i = 0; i < 4 * NT; ++i) any |= odd[i];
  if (any != 0 && !*abort_flag) recompute_units<F16, DH>(p);
}

template <bool F16, int DH>
cudaError_t launch_typed(const CUtensorMap& mQ, const CUtensorMap& mK, const CUtensorMap& mV, const GqaParams& p,
                         int grid, cudaStream_t st) {
  static bool attr_set[64] = {};
  cudaError_t e = set_smem_limit_once(tc_causal_kernel<F16, DH>, Layout<DH>::BYTES, attr_set);
  if (e != cudaSuccess) return e;
  return launch_kernel(tc_causal_kernel<F16, DH>, dim3(grid), dim3(THREADS), Layout<DH>::BYTES, st, mQ, mK, mV, p);
}

}  // namespace

cudaError_t launch_tc_causal(const CUtensorMap& mQ, const CUtensorMap& mK, const CUtensorMap& mV, const GqaParams& p,
                             bool f16, int num_sms, cudaStream_t st) {
  const int tpt = BQ / (p.n_heads / p.n_kv);
  const long units = (static_cast<long>(p.T_cap) / (NT * tpt) + p.B) * p.n_kv;   // at least as many as there are
  if (units > 0x7fffffffL) return cudaErrorInvalidValue;
  const int grid = static_cast<int>(units < num_sms ? units : num_sms);
  if (p.head_dim == 128) return f16 ? launch_typed<true, 128>(mQ, mK, mV, p, grid, st) : launch_typed<false, 128>(mQ, mK, mV, p, grid, st);
  return f16 ? launch_typed<true, 64>(mQ, mK, mV, p, grid, st) : launch_typed<false, 64>(mQ, mK, mV, p, grid, st);
}

}  // namespace seer
