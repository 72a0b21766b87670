// State space scan, backward, tokens of type __half.
#include "state_scan_backward.cuh"

namespace sysconv {
cudaError_t launch_scan_backward_f16(const sysscan_args &a, cudaStream_t s, int *launches)
{
    return launch_scan_backward_t<__half>(a, s, launches);
}
}  // namespace sysconv
