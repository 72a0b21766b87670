// State space scan, forward, tokens of type __half.
#include "state_scan.cuh"

namespace sysconv {
cudaError_t launch_scan_f16(const sysscan_args &a, cudaStream_t s, int *launches) { return launch_scan_t<__half>(a, s, launches); }
}  // namespace sysconv
