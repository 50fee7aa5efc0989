// The C ABI's error state, shared by its translation units (api.cu, api_attention.cu).  Internal to libqvla.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

#include "../../include/qvla.h"

namespace qvla {

void clear_error();                                         // the calling thread's message becomes ""
qvla_status fail(qvla_status s, const char* fmt, ...);      // records a message for the calling thread
qvla_status cuda_fail(cudaError_t e, const char* what);
int num_sms(int device);

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace qvla

#define QVLA_CUDA(call, what)                        \
  do {                                               \
    cudaError_t e_ = (call);                         \
    if (e_ != cudaSuccess) return qvla::cuda_fail(e_, what); \
  } while (0)
