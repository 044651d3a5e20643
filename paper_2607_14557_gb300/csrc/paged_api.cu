// C ABI of the paged K/V cache (declared in include/seer.h): argument checks and
// launches; the arithmetic runs in paged.cu and the grouped-head attention kernels.
#include <cmath>

#include "api.h"
#include "common.cuh"
#include "kernels.h"
#include "paged.h"

using namespace seer;

static_assert(SEER_MAX_DRAFT == kMaxDraft && SEER_MAX_REQUESTS == kPageTableMaxB, "limits of the paged cache");

namespace {

// Row numbers are 32-bit; a page past the pool's end is one too.
constexpr long long kMaxPoolRows = 0x7fffffffll - 1024;
// Row loops step by a grid's worth of rows in 32 bits.
constexpr int kMaxRows = 1 << 30;
// Key tiles of a tree call at most, by its capacities: places on its line times runs stay in 64 bits.
constexpr double kMaxTreeTiles = 1125899906842624.0;   // 2^50

int log2_exact(int v) {
  int s = 0;
  while ((1 << s) < v) ++s;
  return s;
}

seer_status check_page_size(const char* what, int page_size) {
  if (page_size < 8 || page_size > 1024 || (page_size & (page_size - 1)) != 0)
    return fail(SEER_ERR_UNSUPPORTED, "%s: page_size must be a power of two from 8 to 1024 (got %d)", what, page_size);
  return SEER_OK;
}

seer_status check_requests(const char* what, int B) {
  if (B <= 0) return fail(SEER_ERR_INVALID_ARG, "%s: B must be positive", what);
  if (B > SEER_MAX_REQUESTS) return fail(SEER_ERR_UNSUPPORTED, "%s: at most %d requests", what, SEER_MAX_REQUESTS);
  return SEER_OK;
}

seer_status check_capacity(const char* what, int T_cap) {
  if (T_cap < 0) return fail(SEER_ERR_INVALID_ARG, "%s: bad sizes", what);
  if (T_cap > kMaxRows) return fail(SEER_ERR_UNSUPPORTED, "%s: at most %d rows", what, kMaxRows);
  return SEER_OK;
}

seer_status check_pages(const char* what, const seer_pages* g, seer_dtype dt, PagedKv* out) {
  if (!g) return fail(SEER_ERR_INVALID_ARG, "%s: pages is null", what);
  if (!valid_dt(dt)) return fail(SEER_ERR_INVALID_ARG, "%s: unknown dtype", what);
  if (!g->kv || !g->table) return fail(SEER_ERR_INVALID_ARG, "%s: null page pool or table", what);
  if (g->n_pages <= 0 || g->max_pages <= 0 || g->n_kv_heads <= 0 || g->head_dim <= 0)
    return fail(SEER_ERR_INVALID_ARG, "%s: page counts, heads and head_dim must be positive", what);
  SEER_TRY(check_page_size(what, g->page_size));
  if (static_cast<long long>(g->n_pages) * g->page_size > kMaxPoolRows)
    return fail(SEER_ERR_UNSUPPORTED, "%s: the pool has more than %lld rows", what, kMaxPoolRows);
  const int step = dt == SEER_F32 ? 8 : 16;
  if (g->head_dim > 128 || g->head_dim % step != 0)
    return fail(SEER_ERR_UNSUPPORTED, "%s: head_dim must be a multiple of %d and at most 128 (got %d)", what, step, g->head_dim);
  if (static_cast<long long>(g->n_kv_heads) * g->head_dim > (1 << 20))
    return fail(SEER_ERR_UNSUPPORTED, "%s: rows of more than 2^20 key values", what);
  if (!aligned16(g->kv)) return fail(SEER_ERR_UNSUPPORTED, "%s: the page pool must be 16-byte aligned", what);
  *out = PagedKv{g->kv, g->table, g->n_pages, log2_exact(g->page_size), g->max_pages, g->n_kv_heads, g->head_dim};
  return SEER_OK;
}

// Rows of `cols` values, ld apart, at p.
seer_status check_rows(const char* what, const char* name, const void* p, int ld, long long cols, seer_dtype dt) {
  if (!p) return fail(SEER_ERR_INVALID_ARG, "%s: %s is null", what, name);
  if (ld < cols) return fail(SEER_ERR_INVALID_ARG, "%s: rows of %s hold %lld values, ld is %d", what, name, cols, ld);
  if (!aligned16(p) || static_cast<long long>(ld) * static_cast<long long>(esize(dt)) % 16 != 0)
    return fail(SEER_ERR_UNSUPPORTED, "%s: %s needs 16-byte aligned rows", what, name);
  return SEER_OK;
}

seer_status check_heads(const char* what, int n_heads, int n_kv, int head_dim, seer_dtype dt) {
  if (!valid_dt(dt)) return fail(SEER_ERR_INVALID_ARG, "%s: unknown dtype", what);
  if (n_heads <= 0 || n_kv <= 0 || head_dim <= 0) return fail(SEER_ERR_INVALID_ARG, "%s: heads and head_dim must be positive", what);
  if (n_heads % n_kv != 0)
    return fail(SEER_ERR_INVALID_ARG, "%s: n_heads (%d) must be a multiple of n_kv_heads (%d)", what, n_heads, n_kv);
  if (n_heads / n_kv > 128) return fail(SEER_ERR_UNSUPPORTED, "%s: at most 128 query heads share a key/value head", what);
  if (static_cast<long long>(n_heads) * head_dim > (1 << 20))
    return fail(SEER_ERR_UNSUPPORTED, "%s: rows of more than 2^20 query values", what);
  if (is16(dt) && head_dim != 64 && head_dim != 128)
    return fail(SEER_ERR_UNSUPPORTED, "%s: 16-bit attention needs head_dim 64 or 128 (got %d)", what, head_dim);
  if (head_dim > 128 || head_dim % 4 != 0)
    return fail(SEER_ERR_UNSUPPORTED, "%s: fp32 attention needs head_dim <= 128, %% 4 == 0", what);
  return SEER_OK;
}

// Tensor map of 16-bit heads: rows (ld apart) x heads (dh apart) x dh columns, in boxes of
// box_rows x box_heads x 64 with the 128-byte swizzle.
seer_status map_heads(CUtensorMap* m, const void* base, seer_dtype dt, long rows, long ld, int heads, int dh, int box_rows,
                      int box_heads) {
  const PFN_cuTensorMapEncodeTiled_v12000 encode = tensor_map_encoder();
  if (encode == nullptr) return fail(SEER_ERR_CUDA, "cuTensorMapEncodeTiled is not available from the driver");
  const cuuint64_t dims[3] = {static_cast<cuuint64_t>(dh), static_cast<cuuint64_t>(heads), static_cast<cuuint64_t>(rows)};
  const cuuint64_t strides[2] = {static_cast<cuuint64_t>(dh) * 2, static_cast<cuuint64_t>(ld) * 2};
  const cuuint32_t box[3] = {64, static_cast<cuuint32_t>(box_heads), static_cast<cuuint32_t>(box_rows)};
  const cuuint32_t step[3] = {1, 1, 1};
  const CUresult r = encode(m, dt == SEER_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3,
                            const_cast<void*>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) return fail(SEER_ERR_CUDA, "cuTensorMapEncodeTiled failed (%d)", static_cast<int>(r));
  return SEER_OK;
}

}  // namespace

extern "C" {

seer_status seer_page_tables(const int32_t* cached_len, const int32_t* new_len, int B, int page_size, int n_pages,
                             const int32_t* free_pages, int n_free, const int32_t* free_head, int32_t* table,
                             int max_pages, int T_cap, const int32_t* parent, int32_t* cu_new_out, int32_t* kv_len_out,
                             int32_t* slot_out, int32_t* position_out, uint64_t* mask_out, int32_t* free_head_out,
                             void* stream) {
  SEER_TRY(check_requests("page tables", B));
  SEER_TRY(check_page_size("page tables", page_size));
  if (!cached_len || !new_len || !free_head || !table || !cu_new_out || !kv_len_out || !free_head_out)
    return fail(SEER_ERR_INVALID_ARG, "page tables: null pointer");
  if (n_pages <= 0 || max_pages <= 0 || n_free < 0) return fail(SEER_ERR_INVALID_ARG, "page tables: bad sizes");
  SEER_TRY(check_capacity("page tables", T_cap));
  if (n_free > 0 && !free_pages) return fail(SEER_ERR_INVALID_ARG, "page tables: free_pages is null");
  if (T_cap > 0 && (!slot_out || !position_out)) return fail(SEER_ERR_INVALID_ARG, "page tables: null row output");
  if (static_cast<long long>(n_pages) * page_size > kMaxPoolRows)
    return fail(SEER_ERR_UNSUPPORTED, "page tables: the pool has more than %lld rows", kMaxPoolRows);
  if (reinterpret_cast<uintptr_t>(mask_out) % 8 != 0) return fail(SEER_ERR_UNSUPPORTED, "page tables: mask_out must be 8-byte aligned");
  // every block reads the inputs, so no block's outputs may replace them
  const void* const in[] = {cached_len, new_len, free_head, free_pages, parent};
  const void* const out[] = {cu_new_out, kv_len_out, free_head_out, table, slot_out, position_out, mask_out};
  for (const void* i : in)
    for (const void* o : out)
      if (i != nullptr && i == o) return fail(SEER_ERR_INVALID_ARG, "page tables: an output is also an input");
  DeviceInfo* di;
  SEER_TRY(device_info(&di));
  PageTableArgs a{};
  a.cached = cached_len;
  a.fresh = new_len;
  a.B = B;
  a.page_shift = log2_exact(page_size);
  a.n_pages = n_pages;
  a.free_pages = free_pages;
  a.n_free = n_free;
  a.head = free_head;
  a.table = table;
  a.max_pages = max_pages;
  a.T_cap = T_cap;
  a.parent = parent;
  a.cu = cu_new_out;
  a.kv_len = kv_len_out;
  a.slot = slot_out;
  a.position = position_out;
  a.mask = mask_out;
  a.head_out = free_head_out;
  a.err = di->err;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  Phase ph(PH_KV, st);
  SEER_CUDA(launch_page_tables(a, di->num_sms, st), "page tables launch");
  return SEER_OK;
}

seer_status seer_kv_append(const void* qkv, int ld_qkv, seer_dtype dt, int n_heads, int T_cap, const int32_t* M_dev,
                           const int32_t* slot, const int32_t* position, float theta, void* rotated, int ld_rotated,
                           const seer_pages* pages, void* stream) {
  KvAppendArgs a{};
  SEER_TRY(check_pages("append", pages, dt, &a.pages));
  if (n_heads < 0) return fail(SEER_ERR_INVALID_ARG, "append: bad sizes");
  SEER_TRY(check_capacity("append", T_cap));
  const int dh = pages->head_dim;
  const long long q = static_cast<long long>(n_heads) * dh, k = static_cast<long long>(pages->n_kv_heads) * dh;
  if (q > (1 << 20)) return fail(SEER_ERR_UNSUPPORTED, "append: rows of more than 2^20 query values");
  if (!(theta == 0.f || theta >= 1.f) || !std::isfinite(theta))
    return fail(SEER_ERR_INVALID_ARG, "append: theta must be 0 (off) or a finite base from 1 on");
  if (T_cap == 0) return SEER_OK;             // (empty buffers may have no address)
  SEER_TRY(check_rows("append", "qkv", qkv, ld_qkv, q + 2 * k, dt));
  if (rotated) SEER_TRY(check_rows("append", "rotated", rotated, ld_rotated, q + k, dt));
  if (rotated == qkv && ld_rotated != ld_qkv) return fail(SEER_ERR_INVALID_ARG, "append: in place, rotated has qkv's ld");
  if (!slot) return fail(SEER_ERR_INVALID_ARG, "append: slot is null");
  if (theta > 0.f && !position) return fail(SEER_ERR_INVALID_ARG, "append: rotation needs positions");
  DeviceInfo* di;
  SEER_TRY(device_info(&di));
  const long es = static_cast<long>(esize(dt));
  a.qkv = static_cast<const uint8_t*>(qkv);
  a.ld = ld_qkv * es;
  a.rotated = static_cast<uint8_t*>(rotated);
  a.ld_rot = ld_rotated * es;
  a.n_heads = n_heads;
  a.slot = slot;
  a.position = position;
  a.M_dev = M_dev;
  a.T_cap = T_cap;
  a.err = di->err;
  TurnRates rates{};
  if (theta > 0.f)
    for (int i = 0; i < dh / 2; ++i) {
      // turns per position, less than 1 / 6
      const double turns = std::exp2(-2.0 * i / dh * std::log2(static_cast<double>(theta))) / 6.283185307179586476925;
      rates.rate[i] = static_cast<uint64_t>(turns * 18446744073709551616.0);
    }
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  Phase ph(PH_KV, st);
  SEER_CUDA(launch_kv_append(dt, a, rates, theta > 0.f, di->num_sms, st), "append launch");
  return SEER_OK;
}

seer_status seer_kv_accept(seer_dtype dt, const int32_t* cached_len, const int32_t* accepted, const int32_t* n_accepted,
                           int B, int max_draft, const seer_pages* pages, int32_t* len_out, void* stream) {
  KvAcceptArgs a{};
  SEER_TRY(check_requests("accept", B));
  SEER_TRY(check_pages("accept", pages, dt, &a.pages));
  if (!cached_len || !accepted || !n_accepted || !len_out) return fail(SEER_ERR_INVALID_ARG, "accept: null pointer");
  if (max_draft < 1 || max_draft > SEER_MAX_DRAFT)
    return fail(SEER_ERR_INVALID_ARG, "accept: max_draft must be in [1, %d]", SEER_MAX_DRAFT);
  if (len_out == n_accepted || len_out == cached_len || len_out == accepted)
    return fail(SEER_ERR_INVALID_ARG, "accept: len_out is also an input");
  DeviceInfo* di;
  SEER_TRY(device_info(&di));
  a.cached = cached_len;
  a.accepted = accepted;
  a.n_accepted = n_accepted;
  a.B = B;
  a.max_draft = max_draft;
  a.row_bytes = 2 * pages->n_kv_heads * pages->head_dim * static_cast<int>(esize(dt));
  a.len_out = len_out;
  a.err = di->err;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  Phase ph(PH_KV, st);
  SEER_CUDA(launch_kv_accept(a, st), "accept launch");
  return SEER_OK;
}

seer_status seer_attention_causal(const void* q, int ld_q, const void* k, int ld_k, const void* v, int ld_v, void* o,
                                  int ld_o, seer_dtype dt, const int32_t* cu_seqlens, int B, int T_cap, int n_heads,
                                  int n_kv_heads, int head_dim, void* stream) {
  SEER_TRY(check_requests("causal attention", B));
  SEER_TRY(check_heads("causal attention", n_heads, n_kv_heads, head_dim, dt));
  SEER_TRY(check_capacity("causal attention", T_cap));
  if (!cu_seqlens) return fail(SEER_ERR_INVALID_ARG, "causal attention: cu_seqlens is null");
  if (T_cap == 0) return SEER_OK;
  const long long qc = static_cast<long long>(n_heads) * head_dim, kc = static_cast<long long>(n_kv_heads) * head_dim;
  SEER_TRY(check_rows("causal attention", "q", q, ld_q, qc, dt));
  SEER_TRY(check_rows("causal attention", "k", k, ld_k, kc, dt));
  SEER_TRY(check_rows("causal attention", "v", v, ld_v, kc, dt));
  SEER_TRY(check_rows("causal attention", "o", o, ld_o, qc, dt));
  if (o == q || o == k || o == v) return fail(SEER_ERR_INVALID_ARG, "causal attention: o must not alias q, k or v");
  DeviceInfo* di;
  SEER_TRY(device_info(&di));
  GqaParams p{};
  p.q = q;
  p.k = k;
  p.v = v;
  p.o = o;
  p.ld_q = ld_q;
  p.ld_k = ld_k;
  p.ld_v = ld_v;
  p.ld_o = ld_o;
  p.cu = cu_seqlens;
  p.B = B;
  p.T_cap = T_cap;
  p.n_heads = n_heads;
  p.n_kv = n_kv_heads;
  p.head_dim = head_dim;
  p.err = di->err;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (is16(dt)) {
    const int g = n_heads / n_kv_heads;
    CUtensorMap mq, mk, mv;
    SEER_TRY(map_heads(&mq, q, dt, T_cap, ld_q, n_heads, head_dim, 128 / g, g));
    SEER_TRY(map_heads(&mk, k, dt, T_cap, ld_k, n_kv_heads, head_dim, 128, 1));
    SEER_TRY(map_heads(&mv, v, dt, T_cap, ld_v, n_kv_heads, head_dim, 128, 1));
    Phase ph(PH_ATTN, st);
    SEER_CUDA(launch_tc_causal(mq, mk, mv, p, dt == SEER_F16, di->num_sms, st), "causal attention launch");
    return SEER_OK;
  }
  Phase ph(PH_ATTN, st);
  SEER_CUDA(launch_gqa_simt(false, p, di->num_sms, st), "causal attention launch");
  return SEER_OK;
}

seer_status seer_attention_tree_workspace_size(seer_dtype dt, int B, int n_heads, int n_kv_heads, int head_dim,
                                               int max_draft, size_t* bytes) {
  SEER_TRY(check_requests("tree attention", B));
  SEER_TRY(check_heads("tree attention", n_heads, n_kv_heads, head_dim, dt));
  if (max_draft < 1 || max_draft > SEER_MAX_DRAFT)
    return fail(SEER_ERR_INVALID_ARG, "tree attention: max_draft must be in [1, %d]", SEER_MAX_DRAFT);
  if (!bytes) return fail(SEER_ERR_INVALID_ARG, "tree attention: bytes is null");
  DeviceInfo* di;
  SEER_TRY(device_info(&di));
  *bytes = is16(dt) ? tc_tree_part_bytes(n_heads, n_kv_heads, head_dim, max_draft, di->num_sms)
                    : gqa_simt_part_bytes(B, n_heads, n_kv_heads, head_dim, max_draft, di->num_sms);
  return SEER_OK;
}

seer_status seer_attention_tree(const void* q, int ld_q, void* o, int ld_o, seer_dtype dt, const int32_t* cu_new,
                                const int32_t* kv_len, const uint64_t* mask, int B, int T_cap, int n_heads,
                                int max_draft, const seer_pages* pages, void* ws, size_t ws_bytes, void* stream) {
  PagedKv pg;
  SEER_TRY(check_requests("tree attention", B));
  SEER_TRY(check_pages("tree attention", pages, dt, &pg));
  SEER_TRY(check_heads("tree attention", n_heads, pages->n_kv_heads, pages->head_dim, dt));
  SEER_TRY(check_capacity("tree attention", T_cap));
  if (max_draft < 1 || max_draft > SEER_MAX_DRAFT)
    return fail(SEER_ERR_INVALID_ARG, "tree attention: max_draft must be in [1, %d]", SEER_MAX_DRAFT);
  if (!cu_new || !kv_len) return fail(SEER_ERR_INVALID_ARG, "tree attention: null pointer");
  if (reinterpret_cast<uintptr_t>(mask) % 8 != 0) return fail(SEER_ERR_UNSUPPORTED, "tree attention: mask must be 8-byte aligned");
  if (static_cast<double>(B) * pages->n_kv_heads * max_draft * (static_cast<double>(pages->max_pages) * pages->page_size / 128 + 8) > kMaxTreeTiles)
    return fail(SEER_ERR_UNSUPPORTED, "tree attention: more key tiles than 2^50 fit the tables");
  if (T_cap == 0) return SEER_OK;
  const long long qc = static_cast<long long>(n_heads) * pages->head_dim;
  SEER_TRY(check_rows("tree attention", "q", q, ld_q, qc, dt));
  SEER_TRY(check_rows("tree attention", "o", o, ld_o, qc, dt));
  if (o == q) return fail(SEER_ERR_INVALID_ARG, "tree attention: o must not alias q");
  size_t need = 0;
  SEER_TRY(seer_attention_tree_workspace_size(dt, B, n_heads, pages->n_kv_heads, pages->head_dim, max_draft, &need));
  if (need > 0 && (!ws || ws_bytes < need)) return fail(SEER_ERR_WORKSPACE, "tree attention needs %zu bytes of workspace", need);
  if (need > 0 && !aligned16(ws)) return fail(SEER_ERR_UNSUPPORTED, "tree attention: the workspace must be 16-byte aligned");
  DeviceInfo* di;
  SEER_TRY(device_info(&di));
  GqaParams p{};
  const size_t es = esize(dt);
  p.q = q;
  p.k = pg.kv;
  p.v = static_cast<const uint8_t*>(pg.kv) + static_cast<size_t>(pg.n_kv) * pg.head_dim * es;
  p.o = o;
  p.ld_q = ld_q;
  p.ld_k = p.ld_v = 2l * pg.n_kv * pg.head_dim;
  p.ld_o = ld_o;
  p.cu = cu_new;
  p.kv_len = kv_len;
  p.mask = mask;
  p.B = B;
  p.T_cap = T_cap;
  p.n_heads = n_heads;
  p.n_kv = pg.n_kv;
  p.head_dim = pg.head_dim;
  p.max_new = max_draft;
  p.table = pg.table;
  p.n_pages = pg.n_pages;
  p.page_shift = pg.page_shift;
  p.max_pages = pg.max_pages;
  p.part = static_cast<float*>(ws);
  p.err = di->err;
  const cudaStream_t st = static_cast<cudaStream_t>(stream);
  if (is16(dt)) {
    const int g = n_heads / pg.n_kv, page = 1 << pg.page_shift;
    CUtensorMap mq, mkv;
    SEER_TRY(map_heads(&mq, q, dt, T_cap, ld_q, n_heads, pg.head_dim, tc_tree_box_tokens(n_heads, pg.n_kv, max_draft), g));
    SEER_TRY(map_heads(&mkv, pg.kv, dt, static_cast<long>(pg.n_pages) << pg.page_shift, p.ld_k, 2 * pg.n_kv, pg.head_dim,
                       tc_tree_box_keys(n_heads, pg.n_kv, pg.head_dim, max_draft, page), 1));
    Phase ph(PH_ATTN, st);
    SEER_CUDA(launch_tc_tree(mq, mkv, p, dt == SEER_F16, di->num_sms, st), "tree attention launch");
    return SEER_OK;
  }
  p.splits = gqa_simt_splits(B, n_heads, pg.n_kv, max_draft, di->num_sms);
  Phase ph(PH_ATTN, st);
  SEER_CUDA(launch_gqa_simt(true, p, di->num_sms, st), "tree attention launch");
  return SEER_OK;
}

}  // extern "C"
