// Attention of a few new rows per request over a paged key/value cache on tcgen05 for
// sm_103a (head_dim 64 or 128; q, the cache, P and the output all f16, or all bf16).
//   o_i = sum_j p_ij v_j / sum_j p_ij,  p_ij = 2^(s_ij - m_i),  s_ij = q_i k_j log2(e) / sqrt(dh)
// over the cached rows and the new rows whose bit is set in the row's mask.
//
// Bound by HBM: a key/value row is read once for the g = n_heads / n_kv query heads that
// share it and for all of a request's new rows, which together are the rows of one 128-row
// tile (128 / g tokens, row = token * g + head; more tokens: more tiles).  The MMAs of a
// mostly empty tile cost no more than its K and V take to arrive.
//
// A unit is (request, key/value head, row tile); its work the 128-key tiles of its cache.
// All units' key tiles form one line, cut into equal runs, one per CTA, so lengths may
// differ as they like and one long request fills the GPU.  A CTA takes its run as pieces of
// units; a piece that is not a whole unit leaves its unnormalised sums, maximum and weight
// in the workspace, and tree_merge_kernel joins a unit's pieces in order of their keys.
// Where the runs start follows from the lengths by a prefix sum that every CTA makes.
//
// Two CTAs per SM (192 threads, 256 columns of tensor memory), so one's loads and MMAs run
// beside the other's softmax:
//   warp 0     producer: decodes the pieces, publishes them in a shared ring, and loads Q,
//              then K_j and V_j; a box per page, a lane per box
//   warp 1     MMA issuer: S = Q K_j^T, then O += P V_j with P written over S
//   warps 2-5  softmax, a thread per row; warps without a row of the tile only pass on
// Measured (32 / 8 heads of 128): one token for each of 64 requests over 200 .. 8000 cached rows,
// 539 MB, 98 us (5.5 TB/s); 12 trees of 16 .. 64 rows over 500 .. 12000, 179 MB, 60 us; one token
// over 12000 rows 21 us, two over 700 and 433 13.3.  The softmax warps spill 180 .. 230 bytes.
// Hidden keys and non-finite values are treated as in tc_causal.cu: scores dropped, value
// rows past the request's end cleared, and the rows of a piece whose masked tile holds a
// non-finite value left to recompute_pieces() after the last piece.
#include <math.h>

#include "attn_math.cuh"
#include "common.cuh"
#include "paged.h"

namespace seer {
namespace {

constexpr int BQ = 128;                     // rows of a tile
constexpr int BKV = 128;                    // keys of a tile
constexpr int THREADS = 192;
constexpr int PANEL = 16384;
constexpr int BAR_BYTES = 512;
constexpr uint32_t TMEM_COLS = 256;
constexpr uint32_t TM_O = 128;              // S at column 0, O at 128
constexpr float RESCALE_THRESHOLD = 8.0f;   // log2 units
constexpr int U_SLOTS = 4;
constexpr int U_READERS = 1 + 4;            // issuer, softmax warps

// Shared memory of a CTA: QROWS rows of Q, then one ring of SLOTS key and value tiles in turn.
// The MMA reads 128 rows from Q; those past QROWS are other bytes of this memory, in rows of S
// that nobody looks at.  Few rows leave room for a third slot, so that loads go on across a
// tile's softmax (a second Q buffer on top gained nothing).  Where Q fills 32 KB the ring is
// one key slot and three halves of value tiles (64 keys; SLOTS = 0): half of the next V is
// under way before this V is used up.
template <int DH_, int SLOTS_, int QROWS_>
struct Config {
  static constexpr int DH = DH_, SLOTS = SLOTS_, QROWS = QROWS_;
  static constexpr bool HALVES = SLOTS == 0;
  static constexpr int BARS = HALVES ? 4 : SLOTS;         // K, then the halves; or the slots
  static constexpr int TILE = 128 * DH * 2;
  static constexpr int V_PANEL = HALVES ? PANEL / 2 : PANEL;   // 64 columns of a V tile or half
  static constexpr int Q_PANEL = QROWS * 128, Q_BYTES = DH / 64 * Q_PANEL;
  static constexpr int OFF_RING = Q_BYTES;
  static constexpr int RING = HALVES ? TILE + 3 * TILE / 2 : SLOTS * TILE;
  static constexpr int OFF_BAR = OFF_RING + RING;
  static constexpr int BOX = HALVES ? 64 : 128;           // most rows of a box of the pool
  static constexpr int BYTES = OFF_BAR + BAR_BYTES;
  static_assert(Q_PANEL % 1024 == 0, "the 128-byte swizzle repeats every 8 rows");
  static_assert(2 * (BYTES + 1024) <= 228 * 1024, "two CTAs per SM");
  static_assert(Q_BYTES + RING >= (DH / 64 - 1) * Q_PANEL + PANEL, "128 rows from any Q panel");
};
using Dims64 = Config<64, 5, 128>;
using Few128 = Config<128, 3, 48>;
using Wide128 = Config<128, 0, 128>;

// A piece: keys [tile0 * 128, tile1 * 128) of a unit.  n < 0: no more pieces.
struct Piece {
  int q0, tok0, n, kv;                      // request's first row, the tile's first token, its new rows, its keys
  int b, kvh, tile0, tile1;
  int part;                                 // slot of its partial result, or -1: a whole unit
};
static_assert(sizeof(Piece) == 36, "ring entries");

// Places of a unit on the line besides its key tiles: what a piece costs beyond them (Q, the
// first and last round, its result, the join), in key tiles.  Measured, us, at 1 / 2 / 3 places
// of few rows: 64 single tokens 103 / 98 / 98, 12 requests' 32-row drafts 42 / 40 / 40, heads of
// 64 71 / 67 / 69; at 2 / 4 / 6 / 8 of many rows: 12 trees 66 / 59 / 59 / 62.
__device__ __forceinline__ int unit_extra(int part_rows) { return part_rows <= 32 ? 2 : 5; }

struct Request {
  int q0, n, kv;
  bool good;
};
__device__ __forceinline__ Request read_request(const GqaParams& p, int b) {
  Request r{0, 0, 0, true};
  if (b >= p.B) return r;
  r.q0 = p.cu[b];
  const int end = p.cu[b + 1];
  r.kv = p.kv_len[b];
  r.good = r.q0 >= 0 && end >= r.q0 && end <= p.T_cap;
  r.n = r.good ? end - r.q0 : 0;
  r.good = r.good && r.n <= p.max_new && r.kv >= r.n && r.kv <= kMaxKeys &&
           r.kv <= (static_cast<long long>(p.max_pages) << p.page_shift);
  if (!r.good) r.n = r.kv = 0;
  return r;
}
__device__ __forceinline__ int key_tiles(int kv) { return static_cast<int>((kv + static_cast<unsigned>(BKV) - 1) / BKV); }
// Places of all units of a request.
__device__ __forceinline__ long long line_length(const GqaParams& p, const Request& r, int tpt, int extra) {
  return r.n == 0 ? 0 : static_cast<long long>(p.n_kv) * ((r.n + tpt - 1) / tpt) * (key_tiles(r.kv) + extra);
}
// a / b for a >= 0, b > 0, by a 32-bit division where that is enough.
__device__ __forceinline__ int quotient(long long a, int b) {
  return static_cast<int>((a >> 32) == 0 ? static_cast<unsigned>(a) / static_cast<unsigned>(b) : a / b);
}

// Run c of n over a line of `total`: [cut(c), cut(c + 1)), and the run that holds x.
__device__ __forceinline__ long long cut(long long total, int c, int n) {
  const long long x = total * c;
  return (x >> 32) == 0 ? static_cast<unsigned>(x) / static_cast<unsigned>(n) : x / n;
}
__device__ __forceinline__ int run_of(long long total, long long x, int n) {
  return static_cast<int>(((x + 1) * n - 1) / total);
}

// Units that begin in a run and do not end there (at most one per run).
struct Join {
  int q0, tok0, n, kvh;                     // n = 0: none
  int first, last;                          // runs: its pieces are slot 2 first + 1, then 2 c of the later ones
  int pad[2];
};

// This CTA's i-th piece, or null when there are no more; by a whole warp, which gives the
// entry back with release_piece() when it has done with it.
__device__ __forceinline__ const Piece* read_piece(uint64_t* u_full, const Piece* ring, int i, volatile int* abort, int* err) {
  const int s = i % U_SLOTS;
  if (!warp_wait(&u_full[s], (i / U_SLOTS) & 1, abort, err) || ring[s].n < 0) return nullptr;
  return ring + s;
}
__device__ __forceinline__ void release_piece(uint64_t* u_empty, int i, int lane) {
  __syncwarp();
  if (lane == 0) mbar_arrive(&u_empty[i % U_SLOTS]);
}

// Bits of the keys that new row `tok` sees among the request's new rows.
__device__ __forceinline__ uint64_t visible(const GqaParams& p, const Piece& u, int tok) {
  const uint64_t all = u.n >= 64 ? ~0ull : (1ull << u.n) - 1;
  const uint64_t bits = p.mask ? p.mask[u.q0 + tok] : (tok >= 63 ? ~0ull : (2ull << tok) - 1);
  return bits & all;
}

// Where a row's result goes: the output, divided by its weight, or its partial slot.
// A slot holds the sums as [column / 4][row] float4, so that a warp stores 512 bytes in one
// piece (a row's 512 bytes one after the other took 2 us for 128 rows), then each row's
// (max, weight).
struct RowOut {
  uint16_t* o = nullptr;
  float4* part = nullptr;                   // the row's first float4; the next is `rows` on
  float2* stats = nullptr;
  int rows = 0;
};
template <int DH>
__device__ __forceinline__ RowOut row_out(const GqaParams& p, const Piece& u, int tok, int head, int r, int rows) {
  RowOut w;
  if (u.part < 0) {
    w.o = static_cast<uint16_t*>(p.o) + static_cast<size_t>(u.q0 + tok) * p.ld_o + head * DH;
  } else {
    float* slot = p.part + static_cast<size_t>(u.part) * rows * (DH + 4);
    w.part = reinterpret_cast<float4*>(slot) + r;
    w.stats = reinterpret_cast<float2*>(slot + rows * DH) + r;
    w.rows = rows;
  }
  return w;
}
// 8 columns from c on, scaled by inv (output only).
template <bool F16>
__device__ __forceinline__ uint32_t store8(const RowOut& w, int c, const float (&v)[8], float inv) {
  if (w.o == nullptr) {
    w.part[(c / 4) * w.rows] = make_float4(v[0], v[1], v[2], v[3]);
    w.part[(c / 4 + 1) * w.rows] = make_float4(v[4], v[5], v[6], v[7]);
    return 0;
  }
  uint32_t q[4], bad = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    q[e] = pack2(v[2 * e] * inv, v[2 * e + 1] * inv, F16);
    bad |= nonfinite_term(q[e], F16);
  }
  *reinterpret_cast<uint4*>(w.o + c) = make_uint4(q[0], q[1], q[2], q[3]);
  return bad;
}

// A CTA's run [run0, run1) of the line, in shared memory.
struct Start {
  long long warp_sum[THREADS / 32];
  long long run0, run1;
  long long off;                            // run0 is so many places into request b
  Request r;
  int b;
};

// The pieces of run blockIdx.x, by a whole warp.
struct PieceWalk {
  int tpt, extra, lane;
  int b;                                    // request of the next place, `off` places into it
  Request r;
  long long off, at, run1;
  int window;                               // requests window .. window + 31 in the lanes' registers
  Request ahead{};
  Join join{};                              // the unit that begins in the run and does not end there
  long long join_end = 0;                   // its last place

  __device__ __forceinline__ PieceWalk(const Start& s, int tpt_, int extra_, int lane_)
      : tpt(tpt_), extra(extra_), lane(lane_), b(s.b), r(s.r), off(s.off), at(s.run0), run1(s.run1), window(s.b - 32) {}

  // The next piece; n < 0: no more.
  __device__ __forceinline__ Piece next(const GqaParams& p) {
    const int run = blockIdx.x;
    Piece u{};
    while (at < run1) {                     // the next stretch that holds key tiles
      const long long len = line_length(p, r, tpt, extra);
      if (off >= len) {                     // on to the next request
        off -= len;
        if (++b >= p.B) {                   // the lengths changed under the call
          at = run1;
          break;
        }
        if (b - window >= 32) {
          window = b;
          ahead = read_request(p, window + lane);
        }
        r.q0 = __shfl_sync(0xffffffffu, ahead.q0, b - window);
        r.n = __shfl_sync(0xffffffffu, ahead.n, b - window);
        r.kv = __shfl_sync(0xffffffffu, ahead.kv, b - window);
        continue;
      }
      const int tiles = key_tiles(r.kv), places = tiles + extra, row_tiles = (r.n + tpt - 1) / tpt;
      const int unit = quotient(off, places);
      const int first = static_cast<int>(off - static_cast<long long>(unit) * places);
      const int last = static_cast<int>(min(static_cast<long long>(places), first + (run1 - at)));
      off += last - first;
      at += last - first;
      u.tile0 = max(first - extra, 0);
      u.tile1 = last - extra;
      if (u.tile1 <= u.tile0) continue;     // only places without a tile
      u.q0 = r.q0;
      u.n = r.n;
      u.kv = r.kv;
      u.b = b;
      u.kvh = unit / row_tiles;
      u.tok0 = (unit - u.kvh * row_tiles) * tpt;
      u.part = u.tile0 > 0 ? 2 * run : (u.tile1 < tiles ? 2 * run + 1 : -1);
      if (u.tile0 == 0 && u.tile1 < tiles) {
        join = Join{u.q0, u.tok0, u.n, u.kvh, run, 0, {0, 0}};
        join_end = at + (places - last) - 1;
      }
      break;
    }
    if (u.tile1 <= u.tile0) u.n = -1;
    return u;
  }
};

// The rows that a non-finite value in a masked tile may have reached, from global memory by
// every warp of the CTA.  Its pieces are looked over once more, so that none need be remembered.
template <bool F16, int DH>
__device__ __forceinline__ void recompute_pieces(const GqaParams& p, const Start& start) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int G = p.n_heads / p.n_kv, TPT = BQ / G, part_rows = min(TPT, p.max_new) * G;
  PieceWalk walk(start, TPT, unit_extra(part_rows), lane);
  uint32_t nonfinite = 0;
  for (;;) {
    const Piece u = walk.next(p);
    if (u.n < 0) break;
    const int ctx = u.kv - u.n, end = min(u.kv, u.tile1 * BKV);
    // key j's heads; null on a page outside the pool (zeros)
    const auto row_of = [&](int j) -> KeyAt {
      const int page = p.table[static_cast<size_t>(u.b) * p.max_pages + (j >> p.page_shift)];
      if (page < 0 || page >= p.n_pages) return KeyAt{nullptr, nullptr, true};
      const size_t row = ((static_cast<size_t>(page) << p.page_shift) + (j & ((1 << p.page_shift) - 1))) * p.ld_k + u.kvh * DH;
      return KeyAt{static_cast<const uint16_t*>(p.k) + row, static_cast<const uint16_t*>(p.v) + row, true};
    };
    const int masked = max(ctx / BKV, u.tile0) * BKV;      // first key of the masked key tiles
    uint32_t bad = 0;
    for (int x = threadIdx.x; x < (end - masked) * (DH / 8); x += THREADS) {
      const KeyAt key = row_of(masked + x / (DH / 8));
      if (key.v == nullptr) continue;
      const uint4 a = reinterpret_cast<const uint4*>(key.v)[x % (DH / 8)];
      bad |= nonfinite_term(a.x, F16) | nonfinite_term(a.y, F16) | nonfinite_term(a.z, F16) | nonfinite_term(a.w, F16);
    }
    if (!__syncthreads_or((bad & 0x80008000u) != 0)) continue;
    const int rows = min(TPT, u.n - u.tok0) * G;
    for (int r = warp; r < rows; r += THREADS / 32) {
      const int tok = u.tok0 + r / G, head = u.kvh * G + r % G;
      const uint64_t bits = visible(p, u, tok);
      const uint16_t* q = static_cast<const uint16_t*>(p.q) + static_cast<size_t>(u.q0 + tok) * p.ld_q + head * DH;
      const auto at = [&](int j) { return j < ctx || ((bits >> (j - ctx)) & 1) != 0 ? row_of(j) : KeyAt{nullptr, nullptr, false}; };
      const RowSums<DH> sums = attend_row<F16, DH>(q, u.tile0 * BKV, end, at, lane);
      const RowOut out = row_out<DH>(p, u, tok, head, r, part_rows);
      const float inv = sums.l == 0.f ? 0.f : 1.f / sums.l;
#pragma unroll
      for (int e = 0; e < DH / 64; ++e) {
        const int c = lane * (DH / 32) + 2 * e;
        if (out.o == nullptr) {
          reinterpret_cast<float2*>(out.part + (c / 4) * out.rows)[c % 4 / 2] = make_float2(sums.acc[2 * e], sums.acc[2 * e + 1]);
        } else {
          const uint32_t x = pack2(sums.acc[2 * e] * inv, sums.acc[2 * e + 1] * inv, F16);
          nonfinite |= nonfinite_term(x, F16);
          *reinterpret_cast<uint32_t*>(out.o + c) = x;
        }
      }
      if (out.stats && lane == 0) *out.stats = make_float2(sums.m, sums.l);
    }
  }
  report_range(nonfinite, p.err);
}

template <bool F16, typename Cfg>
__global__ void __launch_bounds__(THREADS, 2)
    tc_tree_kernel(const __grid_constant__ CUtensorMap mQ, const __grid_constant__ CUtensorMap mKV, const GqaParams p,
                   const int q_box, Join* __restrict__ joins) {
  constexpr int DH = Cfg::DH, TILE = Cfg::TILE, PANELS = DH / 64;
  constexpr int SLOTS = Cfg::HALVES ? 1 : Cfg::SLOTS;
  extern __shared__ __align__(1024) uint8_t smem[];       // all of the CTA's shared memory, so it starts aligned
  if ((smem_u32(smem) & 1023u) != 0) {
    pdl_enter();
    if (threadIdx.x == 0) {
      record_error(p.err, kErrLayout);
      joins[blockIdx.x] = Join{};
    }
    return;
  }
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + Cfg::OFF_BAR);
  uint64_t* s_full = bars + 0;
  uint64_t* p_full = bars + 1;
  uint64_t* p_full2 = bars + 2;
  uint64_t* o_done = bars + 3;
  uint64_t* o_free = bars + 4;
  uint64_t* q_full = bars + 5;
  uint64_t* q_empty = bars + 6;
  uint64_t* r_full = bars + 7;               // [BARS] ring
  uint64_t* r_empty = r_full + Cfg::BARS;
  uint64_t* u_full = r_empty + Cfg::BARS;    // [U_SLOTS]
  uint64_t* u_empty = u_full + U_SLOTS;      // [U_SLOTS]
  Piece* ring = reinterpret_cast<Piece*>(u_empty + U_SLOTS);     // [U_SLOTS]
  volatile int* odd = reinterpret_cast<volatile int*>(ring + U_SLOTS);   // [4], as in tc_causal.cu
  uint32_t* tmem_slot = const_cast<uint32_t*>(reinterpret_cast<volatile uint32_t*>(odd + 4));
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  constexpr int START_AT = (8 * (7 + 2 * Cfg::BARS + 2 * U_SLOTS) + 36 * U_SLOTS + 16 + 8 + 7) & ~7;
  static_assert(START_AT + sizeof(Start) <= BAR_BYTES, "barrier block");
  Start& start = *reinterpret_cast<Start*>(smem + Cfg::OFF_BAR + START_AT);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int G = p.n_heads / p.n_kv, TPT = BQ / G;
  const int part_rows = min(TPT, p.max_new) * G;          // rows of a partial slot
  const int extra = unit_extra(part_rows);

  // Places of the ring.  Of this CTA's g-th key tile, K is ring tile 2 g and V 2 g + 1 (slot
  // x % SLOTS, used x / SLOTS times before); in halves, K is always slot 0 and half h of V is
  // half slot (2 g + h) % 3.
  struct Place {
    int bar, off;
    unsigned use;
  };
  const auto k_place = [](unsigned g) {
    if (Cfg::HALVES) return Place{0, Cfg::OFF_RING, g};
    return Place{static_cast<int>(2 * g % SLOTS), Cfg::OFF_RING + static_cast<int>(2 * g % SLOTS) * TILE, 2 * g / SLOTS};
  };
  const auto v_place = [](unsigned g, int h) {            // half h; of whole tiles, where half h begins
    if (Cfg::HALVES) {
      const unsigned x = 2 * g + h;
      return Place{1 + static_cast<int>(x % 3), Cfg::OFF_RING + TILE + static_cast<int>(x % 3) * (TILE / 2), x / 3};
    }
    const unsigned x = 2 * g + 1;
    return Place{static_cast<int>(x % SLOTS), Cfg::OFF_RING + static_cast<int>(x % SLOTS) * TILE + h * 8192, x / SLOTS};
  };

  // barriers and tensor memory, before the kernels ahead are waited for
  if (threadIdx.x == 0) {
    mbar_init(s_full, 1);
    mbar_init(p_full, 4);
    mbar_init(p_full2, 4);
    mbar_init(o_done, 1);
    mbar_init(o_free, 4);
    mbar_init(q_full, 1);
    mbar_init(q_empty, 1);
    for (int i = 0; i < Cfg::BARS; ++i) {
      mbar_init(&r_full[i], 1);
      mbar_init(&r_empty[i], 1);
    }
    for (int i = 0; i < U_SLOTS; ++i) {
      mbar_init(&u_full[i], 1);
      mbar_init(&u_empty[i], U_READERS);
      odd[i] = 0;
    }
    *abort_flag = 0;
    fence_barrier_init();
    tma_prefetch_desc(&mQ);
    tma_prefetch_desc(&mKV);
  }
  if (warp == 1) tmem_alloc(tmem_slot, TMEM_COLS);
  pdl_enter();

  // ---- the line of key tiles: its length and the request where this CTA's run begins
  const int chunk = (p.B + THREADS - 1) / THREADS;
  const int b_lo = min(p.B, static_cast<int>(threadIdx.x) * chunk), b_hi = min(p.B, b_lo + chunk);
  long long mine = 0;
  for (int b = b_lo; b < b_hi; ++b) {
    const Request r = read_request(p, b);
    if (!r.good && blockIdx.x == 0) record_error(p.err, kErrLayout);
    mine += line_length(p, r, TPT, extra);
  }
  long long inc = mine;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const long long v = __shfl_up_sync(0xffffffffu, inc, off);
    if (lane >= off) inc += v;
  }
  if (lane == 31) start.warp_sum[warp] = inc;
  __syncthreads();
  long long before = inc - mine, total = 0;
#pragma unroll
  for (int w = 0; w < THREADS / 32; ++w) {
    before += w < warp ? start.warp_sum[w] : 0;
    total += start.warp_sum[w];
  }
  const int grid = gridDim.x, c = blockIdx.x;
  const int runs = total < grid ? static_cast<int>(total) : grid;
  const bool idle = c >= runs;                            // the whole CTA
  const long long run0 = idle ? 0 : cut(total, c, runs), run1 = idle ? 0 : cut(total, c + 1, runs);
  if (!idle && mine > 0 && run0 >= before && run0 < before + mine) {
    long long at = before;
    for (int b = b_lo; b < b_hi; ++b) {
      const Request r = read_request(p, b);
      const long long n = line_length(p, r, TPT, extra);
      if (run0 < at + n) {
        start.b = b;
        start.run0 = run0;
        start.run1 = run1;
        start.off = run0 - at;
        start.r = r;
        break;
      }
      at += n;
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  if (idle) {
    if (threadIdx.x == 0) joins[c] = Join{};
  } else if (warp == 0) {
    // -------------------------------------------------- producer
    const bool leader = elect_one();
    const int box_rows = min(Cfg::BOX, 1 << p.page_shift), boxes = BKV / box_rows;
    const int out_of_pool = p.n_pages << p.page_shift;    // a row that the tensor map fills with zeros
    unsigned g = 0;                                       // key tiles loaded
    int pieces = 0;
    bool ok = true;
    PieceWalk walk(start, TPT, extra, lane);
    // pool row of this lane's box of key tile j
    const auto box_row = [&](int bb, int kv, int j) {
      const int key = j * BKV + lane * box_rows;
      if (lane >= boxes || key >= kv) return -1;
      const int page = p.table[static_cast<size_t>(bb) * p.max_pages + (key >> p.page_shift)];
      if (page < 0 || page >= p.n_pages) {
        record_error(p.err, kErrLayout);
        return out_of_pool;
      }
      return (page << p.page_shift) + (key & ((1 << p.page_shift) - 1));
    };
    // Lanes `mine` load their box (row >= 0), columns of head `head` of the row's 2 n_kv, to
    // `place`, whose first row is key `key0` of the tile.
    const auto load = [&](const Place& at_place, int row, bool mine_box, int key0, int head, int panel) {
      const bool go = mine_box && row >= 0;
      const int bytes = __popc(__ballot_sync(0xffffffffu, go)) * box_rows * 128 * PANELS;
      if (at_place.use > 0 && !warp_wait(&r_empty[at_place.bar], (at_place.use - 1) & 1, abort_flag, p.err)) return false;
      if (leader) mbar_arrive_expect_tx(&r_full[at_place.bar], bytes);
      __syncwarp();
      if (go)
        for (int x = 0; x < PANELS; ++x)
          tma_load_3d(smem + at_place.off + x * panel + (lane * box_rows - key0) * 128, &mKV, &r_full[at_place.bar], 64 * x, head, row);
      __syncwarp();
      return true;
    };
    for (int i = 0; ok; ++i) {
      const Piece u = walk.next(p);
      int next_row = u.n < 0 ? -1 : box_row(u.b, u.kv, u.tile0);   // the page of a tile is looked up a tile ahead
      const int s = i % U_SLOTS;
      if (i >= U_SLOTS && !warp_wait(&u_empty[s], (i / U_SLOTS - 1) & 1, abort_flag, p.err)) break;
      if (lane == 0) {
        ring[s] = u;
        mbar_arrive(&u_full[s]);
      }
      __syncwarp();
      if (u.n < 0) break;
      if (i > 0 && !warp_wait(q_empty, (i - 1) & 1, abort_flag, p.err)) break;
      if (leader) {
        mbar_arrive_expect_tx(q_full, PANELS * q_box * G * 128);
        for (int x = 0; x < PANELS; ++x)
          tma_load_3d(smem + x * Cfg::Q_PANEL, &mQ, q_full, 64 * x, u.kvh * G, u.q0 + u.tok0);
      }
      __syncwarp();
      ++pieces;
      for (int j = u.tile0; j < u.tile1; ++j) {
        const int row = next_row;
        if (j + 1 < u.tile1) next_row = box_row(u.b, u.kv, j + 1);
        ok = load(k_place(g), row, true, 0, u.kvh, PANEL);
        if (Cfg::HALVES) {
          const bool high = lane * box_rows >= BKV / 2;
          ok = ok && load(v_place(g, 0), row, !high, 0, p.n_kv + u.kvh, Cfg::V_PANEL) &&
               load(v_place(g, 1), row, high, BKV / 2, p.n_kv + u.kvh, Cfg::V_PANEL);
        } else {
          ok = ok && load(v_place(g, 0), row, true, 0, p.n_kv + u.kvh, Cfg::V_PANEL);
        }
        if (!ok) break;
        ++g;
      }
    }
    if (walk.join.n > 0) walk.join.last = run_of(total, walk.join_end, runs);
    if (lane == 0) joins[c] = walk.join;
    if (*abort_flag && leader) {
      // let copies still in flight land before the CTA's shared memory is released
      if (pieces > 0) mbar_wait_drain(q_full, (pieces - 1) & 1, 20000000ull);
      for (unsigned j = g > 2 ? g - 3 : 0; j <= g; ++j) { // (waits on tiles that were not issued run out)
        mbar_wait_drain(&r_full[k_place(j).bar], k_place(j).use & 1, 20000000ull);
        for (int h = 0; h < 2; ++h) mbar_wait_drain(&r_full[v_place(j, h).bar], v_place(j, h).use & 1, 20000000ull);
      }
    }
  } else if (warp == 1) {
    // -------------------------------------------------- MMA issuer
    const bool leader = elect_one();
    constexpr uint32_t idesc_qk = make_idesc(BQ, BKV, 0, F16);
    constexpr uint32_t idesc_pv = make_idesc(BQ, DH, 1, F16);
    const uint64_t dq = make_sdesc_sw128(smem_u32(smem), 16, 1024);
    const uint64_t dk0 = make_sdesc_sw128(smem_u32(smem), 16, 1024);
    const uint64_t dv0 = make_sdesc_sw128(smem_u32(smem), Cfg::V_PANEL, 1024);
    const uint32_t dS = tmem, dO = tmem + TM_O;
    unsigned g = 0;                                       // key tiles begun
    auto full = [&](const Place& x) { return warp_wait(&r_full[x.bar], x.use & 1u, abort_flag, p.err); };
    auto qk = [&](bool last) {
      if (leader) {
        const Place at = k_place(g);
        const uint64_t dk = dk0 + static_cast<uint64_t>(at.off >> 4);
#pragma unroll
        for (int k = 0; k < DH / 16; ++k) {
          const uint64_t oq = static_cast<uint64_t>(((k >> 2) * Cfg::Q_PANEL + (k & 3) * 32) >> 4);
          const uint64_t ok = static_cast<uint64_t>(((k >> 2) * PANEL + (k & 3) * 32) >> 4);
          tc_mma_f16(dS, dq + oq, dk + ok, idesc_qk, k > 0 ? 1u : 0u);
        }
        tc_commit(s_full);
        tc_commit(&r_empty[at.bar]);
        if (last) tc_commit(q_empty);
      }
      __syncwarp();
      ++g;
    };
    auto pv = [&](const Place& at, bool fresh, int half) {   // half of the tile's 128 keys
      if (leader) {
        const uint64_t dv = dv0 + static_cast<uint64_t>(at.off >> 4);
#pragma unroll
        for (int kk = 0; kk < BKV / 32; ++kk)
          tc_mma_f16_tmem_a(dO, dS + 8 * (half * (BKV / 32) + kk), dv + static_cast<uint64_t>(kk * 128), idesc_pv,
                            (!fresh || half > 0 || kk > 0) ? 1u : 0u);
        if (half == 1 || Cfg::HALVES) tc_commit(&r_empty[at.bar]);
      }
      __syncwarp();
    };
    bool ok = true;
    for (int i = 0; ok; ++i) {
      const Piece* u = read_piece(u_full, ring, i, abort_flag, p.err);
      if (u == nullptr) break;
      const int tiles = u->tile1 - u->tile0;
      release_piece(u_empty, i, lane);
      if (!warp_wait(q_full, i & 1, abort_flag, p.err) || !full(k_place(g))) break;
      tc_fence_after();
      qk(tiles == 1);
      for (int j = 0; j < tiles; ++j) {
        const unsigned pc = (g - 1) & 1u;                 // the tile whose scores were issued last
        const Place v0 = v_place(g - 1, 0), v1 = v_place(g - 1, 1);
        if ((j == 0 && i > 0 && !warp_wait(o_free, (i - 1) & 1u, abort_flag, p.err)) ||   // the piece before is read out
            !full(v0) || !warp_wait(p_full, pc, abort_flag, p.err)) {
          ok = false;
          break;
        }
        tc_fence_after();
        pv(v0, j == 0, 0);
        if ((Cfg::HALVES && !full(v1)) || !warp_wait(p_full2, pc, abort_flag, p.err)) {
          ok = false;
          break;
        }
        tc_fence_after();
        pv(v1, j == 0, 1);
        if (j + 1 < tiles) {
          if (!full(k_place(g))) {
            ok = false;
            break;
          }
          tc_fence_after();
          qk(j + 2 == tiles);
        } else {
          if (leader) tc_commit(o_done);
          __syncwarp();
        }
      }
    }
  } else {
    // -------------------------------------------------- softmax warps 2..5
    const int r = (warp & 3) * 32 + lane;                 // row of the tile == TMEM lane
    const int rt = r / G;
    const uint32_t lane_off = static_cast<uint32_t>((warp & 3) * 32) << 16;
    const uint32_t tS = tmem + lane_off, tO = tmem + lane_off + TM_O;
    const float scale_log2 = 1.4426950408889634f / sqrtf(static_cast<float>(DH));
    unsigned g = 0;                                       // key tiles seen
    uint32_t nonfinite = 0;
    bool ok = true;
    for (int i = 0; ok; ++i) {
      const Piece* u = read_piece(u_full, ring, i, abort_flag, p.err);
      if (u == nullptr) break;
      const int ntok = min(TPT, u->n - u->tok0), tile0 = u->tile0, tile1 = u->tile1;
      const bool valid_row = rt < ntok;
      const bool busy = (warp & 3) * 32 < ntok * G;       // the warp holds rows of the tile
      const int first_masked = (u->kv - u->n) / BKV;      // tiles from here on hold new rows' keys
      float m_ref = -INFINITY, l = 0.f;
      for (int j = tile0; ok && j < tile1; ++j, ++g) {
        if (!__all_sync(0xffffffffu, mbar_wait(s_full, g & 1u, abort_flag, p.err))) { ok = false; break; }
        tc_fence_after();
        const bool masked = j >= first_masked;
        float s[BKV];
        float alpha = 1.f, neg = 0.f;
        bool any_need = false;
        if (busy) {
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
          if (masked) {
            // new row 0 is key `sh` of the tile: keys before it are seen, then the row's bits
            const uint64_t bits = valid_row ? visible(p, *u, u->tok0 + rt) : 0;
            const int sh = u->kv - u->n - j * BKV;
            const auto word = [&](int at) -> uint32_t {   // keys at .. at + 31
              const int x = at - sh;                      // index of key `at` among the new rows
              if (x >= 64) return 0u;
              if (x >= 0) return static_cast<uint32_t>(bits >> x);
              if (x <= -32) return ~0u;
              return (static_cast<uint32_t>(bits) << -x) | ((1u << -x) - 1);
            };
#pragma unroll
            for (int w = 0; w < BKV / 32; ++w) {
              const uint32_t see = word(32 * w);
#pragma unroll
              for (int e = 0; e < 32; ++e) s[32 * w + e] = (see >> e) & 1u ? s[32 * w + e] : -INFINITY;
            }
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
          const bool need = j == tile0 || m_new > m_ref + RESCALE_THRESHOLD;
          any_need = __any_sync(0xffffffffu, need);
          if (need) {
            alpha = m_ref == -INFINITY ? 0.f : ex2(m_ref - m_new);
            m_ref = m_new;
          }
          neg = m_ref == -INFINITY ? 0.f : -m_ref;        // nothing seen so far: every term is 0
        }
        float rs[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          if (busy) {
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
          }
          if (hf == 0) {
            if (busy && j > tile0 && any_need) {
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
              const int valid = u->kv - j * BKV;
              uint32_t bad = 0;
#pragma unroll 1
              for (int h = 0; h < (Cfg::HALVES ? 2 : 1); ++h) {
                const Place at = v_place(g, h);
                if (!__all_sync(0xffffffffu, mbar_wait(&r_full[at.bar], at.use & 1u, abort_flag, p.err))) {
                  ok = false;
                  break;
                }
                uint4* v = reinterpret_cast<uint4*>(smem + at.off);
                constexpr int KEYS = Cfg::HALVES ? 64 : 128;
#pragma unroll 4
                for (int x = r; x < KEYS * DH / 8; x += 128) {   // 16 bytes: 8 to a key of a panel
                  if (((x >> 3) & (KEYS - 1)) + h * KEYS < valid) {
                    const uint4 w = v[x];
                    bad |= nonfinite_term(w.x, F16) | nonfinite_term(w.y, F16) | nonfinite_term(w.z, F16) |
                           nonfinite_term(w.w, F16);
                  } else {
                    v[x] = make_uint4(0, 0, 0, 0);
                  }
                }
              }
              if (!ok) break;
              if (bad & 0x80008000u) odd[i & 3] = i + 1;
              fence_proxy_async_smem();
            }
          }
          tmem_st_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(hf == 0 ? p_full : p_full2);
        }
        if (!ok) break;
        l = l * alpha + ((rs[0] + rs[1]) + (rs[2] + rs[3]));
      }
      if (!ok) break;
      if (!__all_sync(0xffffffffu, mbar_wait(o_done, i & 1, abort_flag, p.err))) break;
      tc_fence_after();
      const int tok = u->tok0 + rt, head = u->kvh * G + r - rt * G;
      if (busy && odd[i & 3] != i + 1) {      // (else the rows are left to recompute_pieces())
        const float inv_l = l == 0.f ? 0.f : 1.f / l;
        RowOut out;
        if (valid_row) out = row_out<DH>(p, *u, tok, head, r, part_rows);
#pragma unroll 1
        for (int cc = 0; cc < DH / 32; ++cc) {
          uint32_t rr[32];
          tmem_ld32(tO + 32 * cc, rr);
          tmem_ld_wait();
          if (valid_row) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              float v[8];
#pragma unroll
              for (int k = 0; k < 8; ++k) v[k] = __uint_as_float(rr[8 * e + k]);
              nonfinite |= store8<F16>(out, 32 * cc + 8 * e, v, inv_l);
            }
          }
        }
        if (valid_row && out.stats) *out.stats = make_float2(m_ref, l);
      }
      tc_fence_before();
      release_piece(u_empty, i, lane);
      if (lane == 0) mbar_arrive(o_free);
    }
    report_range(nonfinite, p.err);
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, TMEM_COLS);
  }
  if ((odd[0] | odd[1] | odd[2] | odd[3]) != 0 && !*abort_flag) recompute_pieces<F16, DH>(p, start);
}

// Joins the pieces of the unit that begins in run blockIdx.x and ends in a later one, in order
// of their keys: sums and weights relative to a running maximum, so that a piece's numbers
// are read once and several pieces' reads are under way.  A thread takes 16 columns of one of
// 32 rows of the tile (8 columns: twice the threads, 12 trees 60 us instead of 58); fewer rows leave threads to share the pieces among (one token over
// 12000 keys has 38 of them: 39 us with one thread a row and column group), whose results
// then meet in shared memory.
constexpr int MERGE_THREADS = 256, MERGE_COLS = 16;

template <bool F16, int DH>
__global__ void __launch_bounds__(MERGE_THREADS) tree_merge_kernel(const GqaParams p, const Join* __restrict__ joins) {
  constexpr int CHUNKS = DH / MERGE_COLS;
  static_assert(32 * CHUNKS <= MERGE_THREADS, "a thread for every row and column group");
  __shared__ float shares[MERGE_THREADS][MERGE_COLS + 3]; // max, weight, sums
  const int G = p.n_heads / p.n_kv, TPT = BQ / G, part_rows = min(TPT, p.max_new) * G;
  pdl_enter();
  const Join u = joins[blockIdx.x];
  const int rows = min(TPT, u.n - u.tok0) * G, row0 = blockIdx.y * 32;
  if (u.n == 0 || row0 >= rows) return;
  const int left = rows - row0, side = left > 16 ? 32 : (left > 8 ? 16 : (left > 4 ? 8 : (left > 2 ? 4 : 2)));
  const int pieces = u.last - u.first + 1, most = MERGE_THREADS / (side * CHUNKS), subs = pieces < most ? pieces : most;
  const int r = row0 + static_cast<int>(threadIdx.x) % side, col = static_cast<int>(threadIdx.x) / side % CHUNKS * MERGE_COLS;
  const int sub = threadIdx.x / (side * CHUNKS);
  const bool mine = r < rows && sub < subs;
  const size_t stride = static_cast<size_t>(part_rows) * (DH + 4);
  float m = -INFINITY, sum = 0.f, acc[MERGE_COLS] = {};
  const auto add = [&](float m1, float sum1, const float (&f)[MERGE_COLS]) {
    if (sum1 == 0.f) return;                              // a share without a seen key adds nothing
    const float top = fmaxf(m, m1), base = top == -INFINITY ? 0.f : top;
    const float old = ex2(m - base), w = ex2(m1 - base);
    m = top;
    sum = fmaf(sum, old, sum1 * w);
#pragma unroll
    for (int e = 0; e < MERGE_COLS; ++e) acc[e] = fmaf(acc[e], old, w * f[e]);
  };
  if (mine) {
    const int c1 = pieces * (sub + 1) / subs;
#pragma unroll 4
    for (int c = pieces * sub / subs; c < c1; ++c) {      // the unit's first piece is in its run's second slot
      const float* slot = p.part + (2 * (u.first + c) + (c == 0 ? 1 : 0)) * stride;
      const float2 ml = reinterpret_cast<const float2*>(slot + part_rows * DH)[r];
      const float4* v = reinterpret_cast<const float4*>(slot) + col / 4 * part_rows + r;
      float f[MERGE_COLS];
#pragma unroll
      for (int e = 0; e < MERGE_COLS / 4; ++e) {
        const float4 a = v[e * part_rows];
        f[4 * e] = a.x;
        f[4 * e + 1] = a.y;
        f[4 * e + 2] = a.z;
        f[4 * e + 3] = a.w;
      }
      add(ml.x, ml.y, f);
    }
  }
  if (subs > 1) {
    float* mine_at = shares[threadIdx.x];
    mine_at[0] = m;
    mine_at[1] = sum;
#pragma unroll
    for (int e = 0; e < MERGE_COLS; ++e) mine_at[2 + e] = acc[e];
    __syncthreads();
    if (sub == 0)
      for (int k = 1; k < subs; ++k) {
        const float* s = shares[threadIdx.x + k * side * CHUNKS];
        float f[MERGE_COLS];
#pragma unroll
        for (int e = 0; e < MERGE_COLS; ++e) f[e] = s[2 + e];
        add(s[0], s[1], f);
      }
  }
  uint32_t nonfinite = 0;
  if (mine && sub == 0) {
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    uint16_t* o = static_cast<uint16_t*>(p.o) + static_cast<size_t>(u.q0 + u.tok0 + r / G) * p.ld_o + (u.kvh * G + r % G) * DH + col;
#pragma unroll
    for (int h = 0; h < MERGE_COLS / 8; ++h) {
      uint32_t q[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        q[e] = pack2(acc[8 * h + 2 * e] * inv, acc[8 * h + 2 * e + 1] * inv, F16);
        nonfinite |= nonfinite_term(q[e], F16);
      }
      reinterpret_cast<uint4*>(o)[h] = make_uint4(q[0], q[1], q[2], q[3]);
    }
  }
  report_range(nonfinite, p.err);
}

constexpr int CTAS_PER_SM = 2;

template <bool F16, typename Cfg>
cudaError_t launch_typed(const CUtensorMap& mQ, const CUtensorMap& mKV, const GqaParams& p, int grid, int q_box, Join* joins,
                         cudaStream_t st) {
  static bool attr_set[64] = {};
  cudaError_t e = set_smem_limit_once(tc_tree_kernel<F16, Cfg>, Cfg::BYTES, attr_set);
  if (e != cudaSuccess) return e;
  e = launch_kernel(tc_tree_kernel<F16, Cfg>, dim3(grid), dim3(THREADS), Cfg::BYTES, st, mQ, mKV, p, q_box, joins);
  if (e != cudaSuccess) return e;
  const int rows = q_box * (p.n_heads / p.n_kv);
  return launch_kernel(tree_merge_kernel<F16, Cfg::DH>, dim3(grid, (rows + 31) / 32), dim3(MERGE_THREADS), 0, st, p,
                       static_cast<const Join*>(joins));
}
template <bool F16>
cudaError_t launch_rows(const CUtensorMap& mQ, const CUtensorMap& mKV, const GqaParams& p, int grid, int q_box, Join* joins,
                        cudaStream_t st) {
  const int rows = q_box * (p.n_heads / p.n_kv);
  if (p.head_dim == 64) return launch_typed<F16, Dims64>(mQ, mKV, p, grid, q_box, joins, st);
  if (rows <= Few128::QROWS) return launch_typed<F16, Few128>(mQ, mKV, p, grid, q_box, joins, st);
  return launch_typed<F16, Wide128>(mQ, mKV, p, grid, q_box, joins, st);
}

int tile_tokens(int n_heads, int n_kv, int max_new) {
  const int tpt = BQ / (n_heads / n_kv);
  return tpt < max_new ? tpt : max_new;
}
size_t part_floats(int n_heads, int n_kv, int head_dim, int max_new, int num_sms) {
  return static_cast<size_t>(2 * CTAS_PER_SM) * num_sms * tile_tokens(n_heads, n_kv, max_new) * (n_heads / n_kv) * (head_dim + 4);
}

}  // namespace

int tc_tree_box_tokens(int n_heads, int n_kv, int max_new) { return tile_tokens(n_heads, n_kv, max_new); }
int tc_tree_box_keys(int n_heads, int n_kv, int head_dim, int max_new, int page_size) {
  const int rows = tile_tokens(n_heads, n_kv, max_new) * (n_heads / n_kv);
  const int most = head_dim == 128 && rows > Few128::QROWS ? Wide128::BOX : Few128::BOX;
  return page_size < most ? page_size : most;
}

size_t tc_tree_part_bytes(int n_heads, int n_kv, int head_dim, int max_new, int num_sms) {
  return ((part_floats(n_heads, n_kv, head_dim, max_new, num_sms) * 4 + 255) & ~size_t(255)) +
         static_cast<size_t>(CTAS_PER_SM) * num_sms * sizeof(Join);
}

cudaError_t launch_tc_tree(const CUtensorMap& mQ, const CUtensorMap& mKV, const GqaParams& p, bool f16, int num_sms, cudaStream_t st) {
  const int q_box = tile_tokens(p.n_heads, p.n_kv, p.max_new), grid = CTAS_PER_SM * num_sms;
  Join* joins = reinterpret_cast<Join*>(reinterpret_cast<uint8_t*>(p.part) +
                                        ((part_floats(p.n_heads, p.n_kv, p.head_dim, p.max_new, num_sms) * 4 + 255) & ~size_t(255)));
  return f16 ? launch_rows<true>(mQ, mKV, p, grid, q_box, joins, st) : launch_rows<false>(mQ, mKV, p, grid, q_box, joins, st);
}

}  // namespace seer
