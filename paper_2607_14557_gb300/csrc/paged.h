// Launch interface of the paged K/V cache kernels (paged.cu) and of the
// grouped-head attention kernels that use them.  Not part of the public ABI.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace seer {

// A paged cache: page p owns rows [p << page_shift, (p + 1) << page_shift) of kv,
// and table[b * max_pages + i] is the page of request b's rows from i << page_shift on.
struct PagedKv {
  void* kv;               // [n_pages << page_shift, row_elems] rows K | V
  const int* table;       // [B, max_pages]
  int n_pages;
  int page_shift;
  int max_pages;
  int n_kv;               // key/value heads
  int head_dim;
};

struct PageTableArgs {
  const int* cached;      // [B] rows in the cache
  const int* fresh;       // [B] rows that the step adds
  int B;
  int page_shift;
  int n_pages;
  const int* free_pages;  // [n_free]
  int n_free;
  const int* head;        // [1] free pages taken so far
  int* table;             // [B, max_pages]
  int max_pages;
  int T_cap;
  const int* parent;      // [T_cap] or null
  int* cu;                // [B + 1]
  int* kv_len;            // [B]
  int* slot;              // [T_cap]
  int* position;          // [T_cap]
  uint64_t* mask;         // [T_cap] or null
  int* head_out;          // [1]
  int* err;
};
constexpr int kPageTableMaxB = 16384;
cudaError_t launch_page_tables(const PageTableArgs& a, int num_sms, cudaStream_t st);

// Rotary frequencies of a head's pairs as fractions of a turn per position, times 2^64.
struct TurnRates {
  uint64_t rate[64];
};
struct KvAppendArgs {
  const uint8_t* qkv;     // rows q | k | v
  long ld;                // bytes per row
  uint8_t* rotated;       // rows q | k, or null
  long ld_rot;
  int n_heads;            // query heads
  const int* slot;        // [T_cap]
  const int* position;    // [T_cap], or null (no rotation)
  const int* M_dev;       // rows, or null (T_cap)
  int T_cap;
  PagedKv pages;
  int rows_per_block;     // set by the launch
  int* err;
};
cudaError_t launch_kv_append(int type, const KvAppendArgs& a, const TurnRates& rates, bool rotate, int num_sms,
                             cudaStream_t st);

struct KvAcceptArgs {
  const int* cached;      // [B]
  const int* accepted;    // [B, max_draft]
  const int* n_accepted;  // [B]
  int B;
  int max_draft;
  PagedKv pages;
  int row_bytes;
  int* len_out;           // [B]
  int* err;
};
constexpr int kMaxDraft = 64;
cudaError_t launch_kv_accept(const KvAcceptArgs& a, cudaStream_t st);

// Keys of a request at most, so that a tile past them still has a 32-bit number.
constexpr int kMaxKeys = 0x7fffffff - 1024;
// Attention of grouped heads: query head h reads key/value head h / (n_heads / n_kv).
struct GqaParams {
  const void* q;          // [T_cap, ld_q]
  const void* k;          // packed: [T_cap, ld_k]; paged: the pool, K of a row
  const void* v;
  long ld_q, ld_k, ld_v, ld_o;   // elements
  void* o;                // [T_cap, ld_o]
  const int* cu;          // [B + 1]
  const int* kv_len;      // paged: [B] keys of a request, its new rows included
  const uint64_t* mask;   // paged: [T_cap] visible new rows of each new row, or null (causal)
  int B, T_cap, n_heads, n_kv, head_dim;
  int max_new;            // paged: most new rows of a request
  const int* table;       // paged
  int n_pages, page_shift, max_pages;
  float* part;            // paged: partial results, see gqa_part_floats
  int splits;             // CUDA-core kernel, paged: shares of a request's keys
  int* err;
};
// 16-bit causal attention on the tensor cores.  mQ: q as [T_cap][n_heads][head_dim] in boxes
// of floor(128 / g) x g x 64, g = n_heads / n_kv; mK, mV: [T_cap][n_kv][head_dim] in
// boxes of 128 x 1 x 64; all with the 128-byte swizzle.
cudaError_t launch_tc_causal(const CUtensorMap& mQ, const CUtensorMap& mK, const CUtensorMap& mV, const GqaParams& p,
                             bool f16, int num_sms, cudaStream_t st);
// 16-bit attention of new rows over the pages on the tensor cores.  mQ: as above with boxes of
// tc_tree_box_tokens() rows; mKV: the pool as [rows][2 * n_kv][head_dim] in boxes of
// tc_tree_box_keys() x 1 x 64.  p.part: tc_tree_part_bytes().
int tc_tree_box_tokens(int n_heads, int n_kv, int max_new);
int tc_tree_box_keys(int n_heads, int n_kv, int head_dim, int max_new, int page_size);
size_t tc_tree_part_bytes(int n_heads, int n_kv, int head_dim, int max_new, int num_sms);
cudaError_t launch_tc_tree(const CUtensorMap& mQ, const CUtensorMap& mKV, const GqaParams& p, bool f16, int num_sms,
                           cudaStream_t st);
// CUDA-core kernels (fp32).
cudaError_t launch_gqa_simt(bool paged, const GqaParams& p, int num_sms, cudaStream_t st);
// Shares of the keys, and bytes of partial results, of a paged call on the CUDA-core kernel.
int gqa_simt_splits(int B, int n_heads, int n_kv, int max_new, int num_sms);
size_t gqa_simt_part_bytes(int B, int n_heads, int n_kv, int head_dim, int max_new, int num_sms);

}  // namespace seer
