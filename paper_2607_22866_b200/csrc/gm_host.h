// What the translation units of the library share on the host: the last error's text and the allocator hook.
#pragma once
#include <cuda_runtime.h>

#include <cstddef>
#include <string>

#include "gmagnus.h"

namespace gm {

int fail(int code, const std::string& msg);               // keeps the text for gm_last_error, returns the code
void* dev_alloc(size_t bytes, cudaStream_t st);           // the allocator hook, or the device's default pool; nullptr when refused
void dev_free(void* p, cudaStream_t st);
int device_facts_basic(int* num_sms, int* smem_optin);    // of the current device, looked up once

void* page_locked(size_t bytes);                          // host memory that kernels of every device may write to, or nullptr; kept for good

#define GM_CUDA(expr)                                                                              \
  do {                                                                                             \
    cudaError_t e_ = (expr);                                                                       \
    if (e_ != cudaSuccess)                                                                         \
      return fail(GM_ERR_CUDA, std::string(#expr) + ": " + cudaGetErrorString(e_));               \
  } while (0)

#define GM_TRY(expr)                \
  do {                              \
    int rc_ = (expr);               \
    if (rc_ != GM_OK) return rc_;   \
  } while (0)

}  // namespace gm
