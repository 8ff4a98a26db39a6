// Host-side helpers shared by the files that implement the C ABI (tk_api.cu,
// qk_api.cu): error reporting, per-device facts and descriptor checks.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "tk.h"

namespace tk {
namespace api {

// Records the reason for tk_last_error and returns the status.
tk_status fail(tk_status s, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
tk_status cuda_fail(cudaError_t e, const char* what);

// Per-call facts about the current device.
struct DeviceInfo {
  int num_sms = 0;
  int* err = nullptr;  // device address of the device error word
};
tk_status device_info(DeviceInfo* out);

bool aligned16(const void* p);
bool pow2(int x);
int log2i(int x);
bool supported_r(int r);
bool supported_dv(int d);

tk_status check_desc(const tk_cache_desc* d);
tk_status check_cache_ptrs(const tk_cache_desc* d, const void* k, const void* v, const void* ks,
                           const void* pt);

// Key format index used by the kernels: 0 bf16, 1 int8, 2 int4.
int key_format(int32_t k_dtype);

}  // namespace api
}  // namespace tk
