// rv_host.h -- what librv's host files share (not installed): errors, the device's context and the
// memory handle.
#pragma once

#include "rv_internal.h"
#include "rv_ops.h"

namespace rv {

// Records the description of a failure for rv_last_error and returns st.
rv_status fail(rv_status st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
rv_status hip_fail(hipError_t e, const char* what);
const char* error_text();

#define RV_HIP(call, what)                                 \
  do {                                                     \
    hipError_t e_ = (call);                                \
    if (e_ != hipSuccess) return ::rv::hip_fail(e_, what); \
  } while (0)

// The current device's limits and workspaces (rv_init must have run).
struct DeviceContext {
  int n_cus, n_queues, max_lds;
  float* part;         // the frame attention's partial slots, also scratch of other calls
  size_t part_floats;
  float* seq_part;     // rv_attend_seqs' partial slots
  size_t seq_floats;
};
rv_status device_context(DeviceContext* out);

// RV_ERR_INVALID unless `device` is the current one.
rv_status check_current(int device, const char* what);

// rv_init, and the partial slots of rv_attend_seqs.  No batch is refused for them: a launch that would need more
// takes half its sequences, then half of those (48 sequences of 200 tokens over 20,000 shared rows: seven launches,
// each of which reads the shared rows again, 1150 us; all apart in one, 1085).
constexpr int64_t kSeqPartSlots = 8192;
constexpr size_t kSeqPartFloats = (size_t)kSeqPartSlots * kSubFloats;
rv_status setup_sequences();

}  // namespace rv

struct rv_mem_s {
  int device = 0;
  int n_heads = 0;
  int64_t cap = 0, max_tokens = 0, len = 0;
  uint16_t* K = nullptr;
  uint16_t* V = nullptr;
  int32_t* prov = nullptr;
};
