// Launch interface of the kernels that keep a paged cache within a budget: rotary
// positions (rotary.cu), attention mass (mass.cu), the choice of rows and their moves
// (evict.cu).  Not part of the public ABI.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "paged.h"

namespace seer {

struct RotateArgs {
  const uint8_t* x;       // rows of heads: turned ones, then plain ones
  long ld;                // bytes per row
  uint8_t* out;           // rows of the turned heads, or null
  long ld_out;
  int n_turned, n_plain;  // heads of x
  int first_stored;       // heads from here on go to the cache
  int head_dim;
  int half;               // pairs that turn
  const int* slot;        // [T_cap], or null (no cache)
  const int* position;    // [T_cap], or null (no rotation)
  const int* M_dev;       // rows, or null (T_cap)
  int T_cap;
  const int* cu;          // [B + 1] with shift
  const int* shift;       // [B] added to the positions of a request's rows, or null
  int B;
  float magnitude;
  void* kv;               // the pool's rows
  int pool_rows;
  int rows_per_block;     // set by the launch
  int* err;
};
cudaError_t launch_rotate(int type, bool interleaved, const RotateArgs& a, const TurnRates& rates, int num_sms,
                          cudaStream_t st);

struct MassArgs {
  const void* q;          // [T_cap, ld_q]
  long ld_q;
  const int* cu;          // [B + 1]
  const int* kv_len;      // [B]
  const int* accepted;    // [B, max_draft], or null
  const int* n_accepted;  // [B]
  int max_draft;
  int window;
  int B, T_cap;
  int T_kv_cap;           // keys of all requests
  int n_heads;
  PagedKv pages;
  float keep;
  const int* gone;        // [B], or null
  const float* mass_in;   // [B, ld_mass], or null
  float* mass_out;        // [B, ld_mass]
  int* birth;             // [B, ld_mass], or null
  long ld_mass;
  void* ws;
  int runs;               // runs that the tiles are cut into at most (set by the launch)
  int* err;
};
constexpr int kMassColumns = 16384;          // fp32: n_heads * window at most (their statistics are in a block's shared memory)
size_t mass_workspace(int type, int B, int T_kv_cap, int n_heads, int n_kv, int head_dim, int window, int num_sms);
cudaError_t launch_mass(int type, const MassArgs& a, int num_sms, cudaStream_t st);
// The tensor-core path (tc_mass.cu): 16-bit calls of more columns than launch_mass keeps scores for.
// mQ: q as [T_cap][n_heads][head_dim] in boxes of tc_mass_box_tokens() x n_heads / n_kv x 64 (unused with
// accepted rows); mK: the pool as [rows][2 * n_kv][head_dim] in boxes of tc_mass_box_keys() x 1 x 64, with the 128-byte swizzle.
bool mass_on_tensor_cores(int type, int n_heads, int n_kv, int window);
int tc_mass_box_tokens(int n_heads, int n_kv, int window);
int tc_mass_box_keys(int page_size);
size_t tc_mass_workspace(int B, int T_kv_cap, int n_heads, int n_kv, int window, int num_sms);
cudaError_t launch_tc_mass(const CUtensorMap& mQ, const CUtensorMap& mK, const MassArgs& a, bool f16, int num_sms, cudaStream_t st);

struct SelectArgs {
  const float* mass;      // [B, ld_mass]
  const int* birth;       // [B, ld_mass]
  long ld_mass;
  const int* kv_len;      // [B]
  const int* gone;        // [B], or null
  const int* budget;      // [B]
  int B, sinks, recent;
  int* len_out;           // [B]
  int* gone_out;          // [B]
  int* n_moves;           // [B]
  int* move_from;         // [B, ld_move]
  int* move_to;           // [B, ld_move]
  int ld_move;
  int* err;
};
cudaError_t launch_evict_select(const SelectArgs& a, int num_sms, cudaStream_t st);

struct EvictArgs {
  const int* kv_len;      // [B], or null
  const int* n_moves;     // [B]
  const int* move_from;   // [B, ld_move]
  const int* move_to;     // [B, ld_move]
  int ld_move;
  int B;
  PagedKv pages;
  int row_bytes;
  float* mass;            // [B, ld_mass], or null
  int* birth;             // [B, ld_mass], or null
  long ld_mass;
  int* err;
};
cudaError_t launch_kv_evict(const EvictArgs& a, int num_sms, cudaStream_t st);

}  // namespace seer
