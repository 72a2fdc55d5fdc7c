// What the host sides of the operators without a handle share.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/rnnt_beam.h"

namespace rb {

struct AttendArgs;

void set_call_error(const char *msg);  // read by rnnt_beam_last_error(NULL)

inline int refuse(const char *msg) {
  set_call_error(msg);
  return RNNT_E_ARG;
}

// One kernel with one argument.  (The launch's own status: an error that other code left behind is not taken for this call's.)
template <typename Args>
inline int launch(void (*kernel)(Args), int64_t blocks, int blocks_y, int threads, const Args &args, hipStream_t stream) {
  if (blocks > 0x7fffffff) return refuse("more work than one launch takes");
  Args copy = args;
  void *params[] = {&copy};
  const hipError_t e = hipLaunchKernel(reinterpret_cast<const void *>(kernel), dim3((unsigned)blocks, (unsigned)blocks_y), dim3((unsigned)threads), params, 0, stream);
  if (e == hipSuccess) return RNNT_OK;
  (void)hipGetLastError();  // (reported here, not again by the next call of other code)
  set_call_error(hipGetErrorString(e));
  return RNNT_E_HIP;
}

// instantiated once per type and format (attend_kernels.hip); dp: the dims a kernel is compiled for, mt: tiles of 16 rows of a block
template <typename TT, int FMT>
int launch_attend(const AttendArgs &a, int dp, int mt, int64_t blocks, hipStream_t stream);

}  // namespace rb
