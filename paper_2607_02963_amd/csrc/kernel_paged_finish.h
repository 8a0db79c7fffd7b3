// Finish pass of the attention over paged caches: joins the states of a pair
// that was cut over several work-groups (paged_common.h).
//
// W waves per row, wave w taking states w, w + W, ..: the reference max over all
// states, then the sum of 2^(m - M) times each state; the waves' sums meet in
// LDS, in order.  With one wave to a row D / 4 lanes take the row, and the wave two
// rows (four at D = 64).  What bounds it: a chain of three memory round trips (the
// note, the states, out), and with many rows the states' bytes.  Where few pairs are
// cut into many states (one long axis) a single wave would take them in turn: 64
// states of 896 rows took 21.7 us with W = 1, and take 9.2 with W = 4.  57000 rows of
// two to four states (64 MB) took 45 us with a wave per row and eight states asked for
// whatever their number, and take 16.
#pragma once

#include "kernel_mfma.h"
#include "paged_common.h"

namespace pdec {

// Lanes and rows of a wave, and rows of a work-group (256 threads with one wave per row).
template <int D, int W>
struct FinishCfg {
    static constexpr int LPR = W > 1 ? 64 : D / 4, RPW = 64 / LPR, RPB = W > 1 ? 1 : 4 * RPW, THREADS = W > 1 ? 64 * W : 256;
};

template <int D, typename T, int W>
__global__ __launch_bounds__((FinishCfg<D, W>::THREADS)) void paged_finish_kernel(PagedArgs a)
{
    using C = FinishCfg<D, W>;
    constexpr int E = D / C::LPR;  // elements per lane
    typedef float vec_t __attribute__((ext_vector_type(E)));
    __shared__ float part[W > 1 ? W : 1][D + 1];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), w = wave % W;
    const int lane = threadIdx.x % C::LPR;  // of its row
    const int y = blockIdx.y * C::RPB + (W > 1 ? 0 : (int)threadIdx.x / C::LPR);
    const int hs = a.heads == 2 ? y & 1 : 0, r = a.heads == 2 ? y >> 1 : y;
    const int J = a.num_seqs * a.groups;
    // pairs that do not exist have no note
    if (a.by_pair && paged_units(a, blockIdx.x % J) == 0) return;
    const int4 cut = a.cut[blockIdx.x];
    // not cut; or (lengths outside the contract) a note that nobody wrote
    if (cut.x < 0 || cut.y < cut.x || cut.y >= a.workers || (uint32_t)cut.z >= (uint32_t)J || (uint32_t)cut.w >= (uint32_t)(a.H_kv / a.heads)) return;
    const int s = cut.z / a.groups, row0 = (cut.z - s * a.groups) * a.rows;
    const PagedSeq sq = paged_seq(a, s);
    if (r >= min(a.rows, sq.n * a.G - row0)) return;  // all of the row's lanes; W > 1: the whole work-group
    const int count = cut.y - cut.x + 1;
    auto state = [&](int i) { return ((long)(2 * (cut.x + i) + (i == 0 ? 1 : 0)) * a.heads + hs) * a.rows + r; };
    constexpr int B = 8;  // states in flight
    float L = 0.f;
    vec_t acc = 0.f, x[B];
    float2 ml[B];
    auto load = [&](int i0) {
#pragma unroll
        for (int b = 0; b < B; ++b) {
            if (i0 + W * b >= count) break;  // by a scalar: the loads before it stay under way
            const long at = state(i0 + W * b);
            ml[b] = *reinterpret_cast<const float2*>(a.part_ml + 2 * at);
            x[b] = *reinterpret_cast<const vec_t*>(a.part_o + at * D + E * lane);
        }
    };
    load(w);
    float M = kMinRef;
    for (int i = lane; i < count; i += C::LPR) M = fmaxf(M, a.part_ml[2 * state(i)]);
#pragma unroll
    for (int off = 1; off < C::LPR; off <<= 1) M = fmaxf(M, __shfl_xor(M, off));
    for (int i0 = w; i0 < count; i0 += W * B) {
        if (i0 != w) load(i0);
#pragma unroll
        for (int b = 0; b < B; ++b) {
            if (i0 + W * b >= count) break;
            const float f = fast_exp2(ml[b].x - M);
            L += f * ml[b].y;
            acc += f * x[b];
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
    acc *= inv;
    T* const out = static_cast<T*>(a.out) + qr * D + E * lane;
    if constexpr (sizeof(T) == 4) *reinterpret_cast<vec_t*>(out) = acc;
    else if constexpr (E == 4) *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf16x2(acc[0], acc[1]), pack_bf16x2(acc[2], acc[3]));
    else if constexpr (E == 2) *reinterpret_cast<uint32_t*>(out) = pack_bf16x2(acc[0], acc[1]);
    else *out = from_f32<uint16_t>(acc[0]);
    if (lane == 0 && a.lse) a.lse[qr] = any ? kLn2 * (M + log2f(L)) : kNegInf;
}

}  // namespace pdec
