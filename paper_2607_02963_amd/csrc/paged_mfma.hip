// Launches of the bfloat16 kernels of the attention over paged caches, compiled
// as the other matrix-core kernels are (see the build script): the IEEE mode bit
// clear and without NaN semantics.
#include <hip/hip_runtime.h>

#include "kernel_paged_rows.h"

namespace pdec {

void launch_paged_rows(const PagedArgs& a, int head_dim, int grid, hipStream_t s)
{
    const dim3 g((unsigned)grid), b(256);
    if (head_dim == 128) {
        if (a.rows == 256) hipLaunchKernelGGL((paged_rows_kernel<128, 2>), g, b, 0, s, a);
        else hipLaunchKernelGGL((paged_rows_kernel<128, 1>), g, b, 0, s, a);
    } else {
        if (a.rows == 256) hipLaunchKernelGGL((paged_rows_kernel<64, 2>), g, b, 0, s, a);
        else hipLaunchKernelGGL((paged_rows_kernel<64, 1>), g, b, 0, s, a);
    }
}

}  // namespace pdec
