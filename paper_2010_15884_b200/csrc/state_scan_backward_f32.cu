// State space scan, backward, tokens of type float.
#include "state_scan_backward.cuh"

namespace sysconv {
cudaError_t launch_scan_backward_f32(const sysscan_args &a, cudaStream_t s, int *launches)
{
    return launch_scan_backward_t<float>(a, s, launches);
}
}  // namespace sysconv
