// gts_host_only.cpp — stand-ins for the device side of libgts.so in a CPU-only
// build of the host library (gts_host.cpp), used to run its validation, image
// construction and argument checks under AddressSanitizer and UBSan without
// a GPU or device code.  Every kernel launch, and the no-allocation entry
// point (whose scratch is device memory), reports that there is no device.
#include <hip/hip_runtime.h>

#include "../../include/gts.h"
#include "gts_dev.h"
#include "gts_ops.h"

namespace gts {
hipError_t launch_sim(const Launch&, uint32_t, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_window(const Launch&, uint32_t, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_team(const Launch&, uint32_t, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_rotary(const gts_rotary_args&, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_rotary_table(float*, uint32_t, uint32_t, const TableFreqs&, double, hipStream_t) {
  return hipErrorNoDevice;
}
hipError_t launch_append(const gts_append_args&, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_attention(const gts_attention_args&, hipStream_t) { return hipErrorNoDevice; }
uint64_t attention_scratch(uint32_t, uint32_t, uint32_t, uint32_t, uint32_t) { return 0; }
hipError_t launch_norm(const gts_norm_args&, hipStream_t) { return hipErrorNoDevice; }
hipError_t launch_norm_grad(const gts_norm_grad_args&, hipStream_t) { return hipErrorNoDevice; }
uint64_t norm_grad_scratch(uint32_t, uint32_t) { return 0; }
hipError_t launch_matmul(const gts_matmul_args&, hipStream_t) { return hipErrorNoDevice; }
uint64_t matmul_scratch(uint32_t, uint32_t, uint32_t) { return 0; }
hipError_t launch_linear_grad(const gts_linear_grad_args&, hipStream_t) { return hipErrorNoDevice; }
uint64_t linear_grad_scratch(uint32_t, uint32_t) { return 0; }
hipError_t launch_prompt(const gts_prompt_args&, hipStream_t) { return hipErrorNoDevice; }
uint64_t prompt_groups(uint32_t, uint32_t, uint32_t) { return 0; }
hipError_t launch_prompt_grad(const gts_prompt_grad_args&, hipStream_t) { return hipErrorNoDevice; }
uint64_t prompt_grad_scratch(uint32_t, uint32_t, uint32_t, uint32_t, uint32_t) { return 0; }
}  // namespace gts

extern "C" int gts_simulate_hwset_noalloc(const gts_graph*, const gts_hwset*, uint32_t, uint32_t, uint32_t*,
                                          uint32_t*, int32_t*, uint64_t*, uint32_t, void*) {
  return GTS_E_HIP;
}
