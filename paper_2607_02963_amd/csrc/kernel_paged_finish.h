// Finish pass of the attention over paged caches: joins the states of a pair
// that was cut over several work-groups (paged_common.h).
//
// A wave per row: the reference max over the states, then the sum of
// 2^(m - M) times each state, in the order of the work-groups.  What bounds it:
// a chain of two memory round trips, and where few pairs are cut into many the
// states' bytes, so that a pair's rows are spread over the work-groups.
#pragma once

#include "kernel_mfma.h"
#include "paged_common.h"

namespace pdec {

template <int D, typename T>
__global__ __launch_bounds__(64 * kPagedFinishRows) void paged_finish_kernel(PagedArgs a)
{
    constexpr int E = D / 64;  // elements per lane
    const int lane = threadIdx.x & 63;
    const int r = blockIdx.y * kPagedFinishRows + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int J = a.num_seqs * a.groups;
    // pairs that do not exist have no note
    if (a.by_pair && paged_units(a, blockIdx.x % J) == 0) return;
    const int4 cut = a.cut[blockIdx.x];
    if (cut.x < 0) return;
    const int s = cut.z / a.groups, row0 = (cut.z - s * a.groups) * a.rows;
    const PagedSeq sq = paged_seq(a, s);
    if (r >= min(a.rows, sq.n * a.G - row0)) return;
    const int count = cut.y - cut.x + 1;
    auto state = [&](int i) { return (long)(2 * (cut.x + i) + (i == 0 ? 1 : 0)) * a.rows + r; };
    float M = kMinRef;
    for (int i = lane; i < count; i += 64) M = fmaxf(M, a.part_ml[2 * state(i)]);
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) M = fmaxf(M, __shfl_xor(M, off));
    float L = 0.f, acc[E];
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.f;
    constexpr int B = 8;  // states in flight
    for (int i0 = 0; i0 < count; i0 += B) {
        float x[B][E];
        float2 ml[B];
#pragma unroll
        for (int b = 0; b < B; ++b) {
            const long at = state(min(i0 + b, count - 1));
            ml[b] = *reinterpret_cast<const float2*>(a.part_ml + 2 * at);
#pragma unroll
            for (int e = 0; e < E; ++e) x[b][e] = a.part_o[at * D + E * lane + e];
        }
#pragma unroll
        for (int b = 0; b < B; ++b) {
            if (i0 + b >= count) break;
            const float f = fast_exp2(ml[b].x - M);
            L += f * ml[b].y;
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] += f * x[b][e];
        }
    }
    const long qr = paged_qrow(a, sq, cut.w, row0 + r);
    const bool any = L > 0.f || L != L;
    const float inv = any ? 1.f / L : 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        if constexpr (sizeof(T) == 4) static_cast<float*>(a.out)[qr * D + E * lane + e] = acc[e] * inv;
        else static_cast<uint16_t*>(a.out)[qr * D + E * lane + e] = from_f32<uint16_t>(acc[e] * inv);
    }
    if (lane == 0 && a.lse) a.lse[qr] = any ? kLn2 * (M + log2f(L)) : kNegInf;
}

}  // namespace pdec
