// Finish pass of the attention over paged caches: joins the states of a pair
// that was cut over several work-groups (paged_common.h).
//
// W waves per row, wave w taking states w, w + W, ..: the reference max over all
// states, then the sum of 2^(m - M) times each state; the waves' sums meet in
// LDS, in order.  What bounds it: a chain of two memory round trips, and the
// states' bytes.  Where few pairs are cut into many states (one long axis) a
// single wave would take them in turn: 64 states of 896 rows took 21.7 us with
// W = 1, and take 9.2 with W = 4.
#pragma once

#include "kernel_mfma.h"
#include "paged_common.h"

namespace pdec {

constexpr int kPagedFinishRows = 4;  // rows per work-group with one wave per row

template <int D, typename T, int W>
__global__ __launch_bounds__(64 * (W > 1 ? W : kPagedFinishRows)) void paged_finish_kernel(PagedArgs a)
{
    constexpr int E = D / 64;  // elements per lane
    constexpr int RPB = W > 1 ? 1 : kPagedFinishRows;  // rows per work-group
    __shared__ float part[W > 1 ? W : 1][D + 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int y = blockIdx.y * RPB + wave / W, hs = y % a.heads, r = y / a.heads, w = wave % W;
    const int J = a.num_seqs * a.groups;
    // pairs that do not exist have no note
    if (a.by_pair && paged_units(a, blockIdx.x % J) == 0) return;
    const int4 cut = a.cut[blockIdx.x];
    // not cut; or (lengths outside the contract) a note that nobody wrote
    if (cut.x < 0 || cut.y < cut.x || cut.y >= a.workers || (uint32_t)cut.z >= (uint32_t)J || (uint32_t)cut.w >= (uint32_t)(a.H_kv / a.heads)) return;
    const int s = cut.z / a.groups, row0 = (cut.z - s * a.groups) * a.rows;
    const PagedSeq sq = paged_seq(a, s);
    if (r >= min(a.rows, sq.n * a.G - row0)) return;  // W > 1: the whole work-group, which has one row
    const int count = cut.y - cut.x + 1;
    auto state = [&](int i) { return ((long)(2 * (cut.x + i) + (i == 0 ? 1 : 0)) * a.heads + hs) * a.rows + r; };
    constexpr int B = 8;  // states in flight
    float L = 0.f, acc[E], x[B][E];
    float2 ml[B];
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.f;
    auto load = [&](int i0) {  // states past the last repeat it and are left out below
#pragma unroll
        for (int b = 0; b < B; ++b) {
            const long at = state(min(i0 + W * b, count - 1));
            ml[b] = *reinterpret_cast<const float2*>(a.part_ml + 2 * at);
#pragma unroll
            for (int e = 0; e < E; ++e) x[b][e] = a.part_o[at * D + E * lane + e];
        }
    };
    load(w);
    float M = kMinRef;
    for (int i = lane; i < count; i += 64) M = fmaxf(M, a.part_ml[2 * state(i)]);
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) M = fmaxf(M, __shfl_xor(M, off));
    for (int i0 = w; i0 < count; i0 += W * B) {
        if (i0 != w) load(i0);
#pragma unroll
        for (int b = 0; b < B; ++b) {
            if (i0 + W * b >= count) break;
            const float f = fast_exp2(ml[b].x - M);
            L += f * ml[b].y;
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] += f * x[b][e];
        }
    }
    if constexpr (W > 1) {
#pragma unroll
        for (int e = 0; e < E; ++e) part[w][E * lane + e] = acc[e];
        if (lane == 0) part[w][D] = L;
        __syncthreads();
        if (w > 0) return;
#pragma unroll
        for (int k = 1; k < W; ++k) {
            L += part[k][D];
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] += part[k][E * lane + e];
        }
    }
    const long qr = paged_qrow(a, sq, cut.w * a.heads + hs, row0 + r);
    const bool any = L > 0.f || L != L;
    const float inv = any ? 1.f / L : 0.f;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < E; ++e) static_cast<float*>(a.out)[qr * D + E * lane + e] = acc[e] * inv;
    } else if constexpr (E == 2) {
        *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(a.out) + qr * D + 2 * lane) = pack_bf16x2(acc[0] * inv, acc[1] * inv);
    } else {
        static_cast<uint16_t*>(a.out)[qr * D + lane] = from_f32<uint16_t>(acc[0] * inv);
    }
    if (lane == 0 && a.lse) a.lse[qr] = any ? kLn2 * (M + log2f(L)) : kNegInf;
}

}  // namespace pdec
