// Error reporting and argument checks shared by the C ABI's sources: each
// check returns LL_OK or records a message for ll_last_error and returns its
// code.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace lossy {

__attribute__((format(printf, 2, 3))) int fail(int code, const char* fmt, ...);
int ok();
int hip_check(hipError_t e, const char* what);
size_t elem_bytes(int32_t dtype);
bool aligned16(const void* p);
int check_rows(const char* name, const void* p, int64_t ld, int64_t d, size_t esize);
int check_vec(const char* name, const void* p, bool required);
int check_dtype(const char* name, int32_t t);

}  // namespace lossy
