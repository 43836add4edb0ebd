// The thread's last error, shared by the files of entry points (api.cpp holds
// it).
#pragma once

#include <hip/hip_runtime_api.h>

#include <string>

namespace ojbkq {

void clear_error();
int fail(int code, const std::string& msg);
int hip_fail(hipError_t e, const char* where);

}  // namespace ojbkq

#define OJBKQ_HIP(call, where)                              \
  do {                                                      \
    hipError_t e_ = (call);                                 \
    if (e_ != hipSuccess) return ojbkq::hip_fail(e_, where); \
  } while (0)
