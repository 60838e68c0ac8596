// What the library's entry points share about errors and launches.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ws_gemm.h"

namespace wsg {

// Records a failing HIP call for ws_gemm_last_error(); returns WS_ERR_HIP.
ws_status hip_fail(const char* what, hipError_t e);

// Launches kernel(args) on `stream`; the kernel takes one struct by value.
template <typename Args>
ws_status launch(const char* what, void (*kernel)(Args), int64_t grid, int block, int lds, hipStream_t stream,
                 Args args) {
  void* p[] = {&args};
  const hipError_t e = hipLaunchKernel((const void*)kernel, dim3((uint32_t)grid), dim3((uint32_t)block), p,
                                       (size_t)lds, stream);
  return e == hipSuccess ? WS_OK : hip_fail(what, e);
}

}  // namespace wsg
