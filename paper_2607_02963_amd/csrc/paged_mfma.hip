// Launches of the bfloat16 kernels of the attention over paged caches, a
// translation unit of their own for the compilation's time.  Compiled with NaN
// semantics, unlike the dense matrix-core kernels (see the build script): hidden
// rows hold anything, and a visible NaN is the result of the rows that see it.
#include <hip/hip_runtime.h>

#include "kernel_paged_few.h"
#include "kernel_paged_few4.h"
#include "kernel_paged_rows.h"
#include "pdec.h"

namespace pdec {

namespace {

template <int D, bool FP8, bool Q4 = false>
void launch_rows(const PagedArgs& a, hipStream_t s)
{
    if (a.rows == 256) hipLaunchKernelGGL((paged_rows_kernel<D, 2, FP8, Q4>), dim3((unsigned)a.blocks), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((paged_rows_kernel<D, 1, FP8, Q4>), dim3((unsigned)a.blocks), dim3(256), 0, s, a);
}

template <int D, bool FP8, int HW>
void launch_few(const PagedArgs& a, hipStream_t s)
{
    const dim3 grid((unsigned)a.blocks), block(64 * kFewWaves);
    if (a.rows == 16) hipLaunchKernelGGL((paged_few_kernel<D, 1, FP8, HW>), grid, block, 0, s, a);
    else if (a.rows == 32) hipLaunchKernelGGL((paged_few_kernel<D, 2, FP8, HW>), grid, block, 0, s, a);
    else if constexpr (D == 64) {
        if (a.rows == 48) hipLaunchKernelGGL((paged_few_kernel<D, 3, FP8, HW>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((paged_few_kernel<D, 4, FP8, HW>), grid, block, 0, s, a);
    }
}

template <int D, bool BIG, typename T>
void launch_few4(const PagedArgs& a, hipStream_t s)
{
    const dim3 grid((unsigned)a.blocks), block(64 * kFewWaves);
    if (a.rows == 16) hipLaunchKernelGGL((paged_few4_kernel<D, 1, BIG, T>), grid, block, 0, s, a);
    else if constexpr (D == 64 || sizeof(T) == 2) {
        if (a.rows == 32) hipLaunchKernelGGL((paged_few4_kernel<D, 2, BIG, T>), grid, block, 0, s, a);
        else if constexpr (sizeof(T) == 2) {
            if (a.rows == 48) hipLaunchKernelGGL((paged_few4_kernel<D, 3, BIG, T>), grid, block, 0, s, a);
            else if constexpr (D == 64) hipLaunchKernelGGL((paged_few4_kernel<D, 4, BIG, T>), grid, block, 0, s, a);
        }
    }
}

template <typename T>
void launch_few4(const PagedArgs& a, int head_dim, hipStream_t s)
{
    const bool big = a.page_shift >= 6;
    if (head_dim == 128) big ? launch_few4<128, true, T>(a, s) : launch_few4<128, false, T>(a, s);
    else big ? launch_few4<64, true, T>(a, s) : launch_few4<64, false, T>(a, s);
}

}  // namespace

void launch_paged_few4(const PagedArgs& a, int head_dim, bool f32, hipStream_t s)
{
    f32 ? launch_few4<float>(a, head_dim, s) : launch_few4<uint16_t>(a, head_dim, s);
}

void launch_paged_few(const PagedArgs& a, int head_dim, bool fp8, hipStream_t s)
{
    const bool two = a.heads == 2;
    if (head_dim == 128 && !fp8) launch_few<128, false, 1>(a, s);
    else if (head_dim == 128) two ? launch_few<128, true, 2>(a, s) : launch_few<128, true, 1>(a, s);
    else if (fp8) two ? launch_few<64, true, 2>(a, s) : launch_few<64, true, 1>(a, s);
    else two ? launch_few<64, false, 2>(a, s) : launch_few<64, false, 1>(a, s);
}

void launch_paged_rows(const PagedArgs& a, int head_dim, int cache_dtype, hipStream_t s)
{
    if (cache_dtype == PDEC_DTYPE_E2M1) {
        head_dim == 128 ? launch_rows<128, true, true>(a, s) : launch_rows<64, true, true>(a, s);
        return;
    }
    const bool fp8 = cache_dtype == PDEC_DTYPE_E4M3;
    if (head_dim == 128) fp8 ? launch_rows<128, true>(a, s) : launch_rows<128, false>(a, s);
    else fp8 ? launch_rows<64, true>(a, s) : launch_rows<64, false>(a, s);
}

}  // namespace pdec
