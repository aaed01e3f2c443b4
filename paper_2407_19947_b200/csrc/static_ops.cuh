// What the entry points on caller-held buffers (paged.cu, attend.cu, sample.cu) share.
#pragma once
#include <atomic>

#include "../../include/stairs.h"
#include "common.cuh"

namespace stairs {

// Files the text that stairs_last_error(NULL) gives and returns `code`.
int static_fail(int code, const char* fmt, ...);

#define SCK(call)                                                                                       \
  do {                                                                                                  \
    cudaError_t e_ = (call);                                                                            \
    if (e_ != cudaSuccess)                                                                              \
      return stairs::static_fail(STAIRS_ECUDA, "%s failed: %s (%s:%d)", #call, cudaGetErrorString(e_),  \
                                 __FILE__, __LINE__);                                                   \
  } while (0)

// Sets an attribute of a kernel once per device (the call takes the host about a microsecond).
inline int allow_once(std::atomic<unsigned long long>& done, const void* kern, cudaFuncAttribute what, int value) {
  int dev = 0;
  SCK(cudaGetDevice(&dev));
  const unsigned long long bit = 1ull << (dev & 63);
  if (dev < 64 && (done.load(std::memory_order_relaxed) & bit)) return STAIRS_OK;
  SCK(cudaFuncSetAttribute(kern, what, value));
  if (dev < 64) done.fetch_or(bit, std::memory_order_relaxed);
  return STAIRS_OK;
}
inline int allow_shared(std::atomic<unsigned long long>& done, const void* kern, int bytes) {
  return allow_once(done, kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

enum Dtype { DT_F32 = 0, DT_BF16 = 1, DT_F16 = 2 };
inline int dtype_bytes(int dt) { return dt == DT_F32 ? 4 : 2; }

inline bool aligned(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % (size_t)bytes == 0; }
inline bool aligned16(const void* p) { return aligned(p, 16); }

// Checks that every entry point with a cache makes; 0 or a status with its text filed.
int check_paged(const char* who, const stairs_paged* c);

// The checks of stairs_sample_static on what the host can see, without launching anything; `who` goes into the text.
int check_sample(const char* who, const void* logits_dev, int dtype, int vocab, long long ld, int n_req, const int32_t* k_host, const stairs_sampling* params_host,
                 const float* u_dev, const int32_t* draft_dev, int k_max, const int32_t* target_tokens_dev, const int32_t* accept_len_dev);

// PDL: the next kernel of the stream may be set up; wait until the previous one's writes are visible.
__device__ __forceinline__ void launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_prerequisites() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

}  // namespace stairs
