// What the C-ABI translation units (seer_api.cu, paged_api.cu) share: error
// reporting, the current device's error word and SM count, argument helpers and
// the per-phase marks of the profiler.  Not part of the public ABI.
#pragma once

#include <cudaTypedefs.h>
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/seer.h"

namespace seer {

struct DeviceInfo {
  int* err = nullptr;
  int num_sms = 0;
};

// Sets this thread's message and returns st.
seer_status fail(seer_status st, const char* fmt, ...);
seer_status cuda_fail(cudaError_t e, const char* where);
seer_status device_info(DeviceInfo** out);
// cuTensorMapEncodeTiled, or null when the driver does not offer it.
PFN_cuTensorMapEncodeTiled_v12000 tensor_map_encoder();

#define SEER_CUDA(call, where)                          \
  do {                                                  \
    cudaError_t e_ = (call);                            \
    if (e_ != cudaSuccess) return cuda_fail(e_, where); \
  } while (0)

#define SEER_TRY(expr)                 \
  do {                                 \
    seer_status s_ = (expr);           \
    if (s_ != SEER_OK) return s_;      \
  } while (0)

inline bool valid_dt(seer_dtype dt) { return dt == SEER_F32 || dt == SEER_BF16 || dt == SEER_F16; }
inline bool is16(seer_dtype dt) { return dt == SEER_BF16 || dt == SEER_F16; }
inline size_t esize(seer_dtype dt) { return dt == SEER_F32 ? 4 : 2; }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

enum { PH_DETECT = 0, PH_SCAN, PH_PACK, PH_NORM1, PH_QKV, PH_ATTN, PH_OPROJ, PH_NORM2, PH_GATEUP, PH_DOWN, PH_KV };

// Marks one kernel launch: an NVTX range on the host timeline (a no-op unless
// a tool such as nsys or ncu --nvtx is attached), and, when profiling is on,
// a pair of CUDA events on the launch's stream.
class Phase {
 public:
  Phase(int ph, cudaStream_t st);
  ~Phase();
  Phase(const Phase&) = delete;
  Phase& operator=(const Phase&) = delete;

 private:
  int ph_;
  cudaStream_t st_;
  cudaEvent_t a_ = nullptr, b_ = nullptr;
};

}  // namespace seer
