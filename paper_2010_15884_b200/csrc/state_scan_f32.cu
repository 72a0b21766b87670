// State space scan, forward, tokens of type float.
#include "state_scan.cuh"

namespace sysconv {
cudaError_t launch_scan_f32(const sysscan_args &a, cudaStream_t s, int *launches) { return launch_scan_t<float>(a, s, launches); }
}  // namespace sysconv
