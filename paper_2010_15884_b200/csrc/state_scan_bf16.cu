// State space scan, forward, tokens of type __nv_bfloat16.
#include "state_scan.cuh"

namespace sysconv {
cudaError_t launch_scan_bf16(const sysscan_args &a, cudaStream_t s, int *launches) { return launch_scan_t<__nv_bfloat16>(a, s, launches); }
}  // namespace sysconv
