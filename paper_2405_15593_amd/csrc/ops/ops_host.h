// Error reporting shared by the library's entry points (microadam_api.cpp
// holds the calling thread's message).
#pragma once
#include <hip/hip_runtime.h>

namespace microadam {

int report(int code, const char* msg);
int report_hip(hipError_t e, const char* what);
void clear_report();

}  // namespace microadam
