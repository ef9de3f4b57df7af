// Host helpers that the checks of the sequence operators share.
#pragma once

#include "ops_kernels.h"

#include <cstdarg>
#include <cstdio>

namespace evk {

inline evconv_status refuse(evconv_status st, const char* format, ...) {
  char text[256];
  va_list args;
  va_start(args, format);
  vsnprintf(text, sizeof text, format, args);
  va_end(args);
  set_call_error(text);
  return st;
}

inline evconv_status launched(const char* what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? EVCONV_OK : refuse(EVCONV_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

inline bool float_type(int dtype) { return dtype == EVCONV_F32 || dtype == EVCONV_BF16; }
inline size_t type_size(int dtype) { return dtype == EVCONV_F32 ? 4 : 2; }
inline bool aligned(const void* p, size_t to) { return (uintptr_t)p % to == 0; }
// Whether rows of `dtype` at this address and these distances may be read 16 bytes at a time.
inline bool wide(int dtype, const void* p, int64_t stride) { return aligned(p, 16) && stride * (int64_t)type_size(dtype) % 16 == 0; }
inline bool wide(int dtype, const evconv_heads& h) { return wide(dtype, h.data, h.token_stride) && wide(dtype, h.data, h.head_stride); }

}  // namespace evk
