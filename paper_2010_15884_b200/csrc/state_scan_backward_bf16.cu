// State space scan, backward, tokens of type __nv_bfloat16.
#include "state_scan_backward.cuh"

namespace sysconv {
cudaError_t launch_scan_backward_bf16(const sysscan_args &a, cudaStream_t s, int *launches)
{
    return launch_scan_backward_t<__nv_bfloat16>(a, s, launches);
}
}  // namespace sysconv
