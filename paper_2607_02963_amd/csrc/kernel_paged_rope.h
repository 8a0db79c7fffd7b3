// Rotary positions of a ragged batch's tokens: alone, forward or back (the gradient), and
// fused with the append to a paged cache.
//
// Pair i of a head's first R elements turns by pos f_i and is multiplied by `magnitude`.
// Going back it turns by -pos f_i: the transposed matrix, which takes a gradient of the
// turned row to one of the plain row.  f_i = theta^(-2i/R), for long contexts divided by
// the scaling's factor for all pairs (linear), theta raised so that the last pair's is
// divided by it (ntk; a larger theta is all there is to it), or divided the more the fewer
// turns the pair makes over the trained length (by parts); or from the caller's table.
//
// A wave takes a token (or, where tokens are few, some of its heads).  Lane i forms pair
// i's cosine and sine, the angle in double and in turns, so that far positions keep them;
// they pass through LDS to the lanes, 32 bytes of a head each, the same for every head: their
// pairs' cosines and sines stay in registers.  bfloat16 rows turn in float32 (2^-24 of
// a term), rounded once; float32 rows in double, whose rate is float32's here, rounded once.
//
// What bounds them: the bytes, each read and written once.  8001 float32 tokens, 28 and 4
// heads of 128 (262 MB) 56 us, 4.7 TB/s of the 5.2 of a large copy (87% of the wave cycles
// wait); the append of 15236 bfloat16 tokens with their queries (281 MB) 59 us, 4.7 TB/s.
// With few tokens it is the call on the host: 32 tokens 9.5 and 10.6 us, the kernels 3.6 and 4.5.
#pragma once

#include "kernel_paged_io.h"

namespace pdec {

struct RopeSpec {
    double log2_theta;
    double inv_factor;    // linear, by parts: 1 / factor
    double turns_per_f;   // by parts: original_len / 2 pi
    double slow, inv_range;
    double magnitude;
    const double* freqs;  // device, or null
    int R, interleaved, by_parts;
    int back;
};

// f_i in turns per position.
__device__ inline double rope_turns(const RopeSpec& r, int i)
{
    double f;
    if (r.freqs) f = r.freqs[i];
    else {
        f = exp2(-(2.0 * i / r.R) * r.log2_theta);
        double u = 0.0;  // the share of the plain frequency
        if (r.by_parts) u = fmin(fmax((r.turns_per_f * f - r.slow) * r.inv_range, 0.0), 1.0);
        f = u * f + (1.0 - u) * (f * r.inv_factor);
    }
    return f * 0.15915494309189533577;  // 1 / 2 pi
}

template <typename T> struct RopeReal { typedef float type; };
template <> struct RopeReal<float> { typedef double type; };

// Stores to global memory, where the compiler can not tell by itself that it is.
typedef __attribute__((address_space(1))) u32x4_t rope_global_t;
__device__ inline void rope_store(void* p, u32x4_t x) { *(rope_global_t*)(uintptr_t)p = x; }
// Past the caches' working set.  The append's rows (queries among them) of 4096 tokens of 36
// heads of 128 (75 MB) took 19.7 us kept in the caches and take 16.3, of 8192 39 and 35, of 16384
// 68 and 63; with a reader of the queries behind 29.7 and 29.2, 55.5 and 54.7, 109 and 105; up to
// 2048 the two are alike.  (Rows turned alone keep
// the caches, as who reads them next gains more: float32 gradients, 262 MB, past them and not: 52
// and 56 us into memory of their own, 52 and 48 into that of the call before, of which some is
// still cached, 99 and 87 with a reader of the turned queries behind; 131 MB 25 and 31, 25 and 26,
// 53 and 48.)
__device__ inline void rope_store_once(void* p, u32x4_t x) { __builtin_nontemporal_store(x, (rope_global_t*)(uintptr_t)p); }

// 16 bytes of a row, E elements.
template <typename T>
struct RopePiece {
    static constexpr int E = 16 / sizeof(T);
    u32x4_t x;
    __device__ inline float get(int i) const
    {
        if constexpr (E == 4) return __uint_as_float(x[i]);
        else return __uint_as_float((i & 1) ? x[i >> 1] & 0xffff0000u : x[i >> 1] << 16);
    }
    __device__ inline void set(const float (&v)[E])
    {
        if constexpr (E == 4) {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = __float_as_uint(v[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
        }
    }
};

// The lane's part of a head: two pieces of E elements, E pairs where it turns.  Of the turning
// elements piece u of each half, so that neighbouring lanes' pieces are neighbours: halves
// pair the one with the other, and interleaved pairs lie within each.  The rest the same way.
template <int D, typename T>
struct RopeLane {
    typedef typename RopeReal<T>::type real;
    static constexpr int E = RopePiece<T>::E, UNITS = D / (2 * E), HEADS = 64 / UNITS;  // parts of a head; heads of a wave at a time
    int unit, head;   // part of the head, and head of the wave's
    bool turns;
    int off[2], pair[2];  // the pieces, and the first pair of the first E / 2 and of the others
    real c[E], s[E];

    __device__ inline void init(const RopeSpec& r, int lane)
    {
        unit = lane % UNITS;
        head = lane / UNITS;
        turns = unit < r.R / (2 * E);
        const int u = turns ? unit : unit - r.R / (2 * E);
        off[0] = (turns ? 0 : r.R) + E * u;
        off[1] = off[0] + (turns ? r.R : D - r.R) / 2;
        pair[0] = r.interleaved ? E / 2 * u : E * u;
        pair[1] = pair[0] + (r.interleaved ? r.R / 4 : E / 2);
        if (!turns) pair[0] = pair[1] = 0;
    }
    // Cosines and sines at position pos, through the wave's part of LDS.
    __device__ inline void at(const RopeSpec& r, double turns_i, int lane, int pos, real (*cs)[64])
    {
        double t = pos * turns_i, sn, cn;
        t -= rint(t);
        sincospi(2.0 * t, &sn, &cn);
        cs[0][lane] = (real)(cn * r.magnitude);
        cs[1][lane] = (real)((r.back ? -sn : sn) * r.magnitude);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int e = 0; e < E; ++e) {
            c[e] = cs[0][pair[e / (E / 2)] + e % (E / 2)];
            s[e] = cs[1][pair[e / (E / 2)] + e % (E / 2)];
        }
    }
    __device__ inline void turn(const RopeSpec& r, RopePiece<T>& a, RopePiece<T>& b) const
    {
        if (!turns) return;
        float x[E], y[E];
        if (r.interleaved) {
#pragma unroll
            for (int e = 0; e < E; e += 2) {
                const real a0 = a.get(e), a1 = a.get(e + 1), b0 = b.get(e), b1 = b.get(e + 1);
                x[e] = (float)(a0 * c[e / 2] - a1 * s[e / 2]);
                x[e + 1] = (float)(a1 * c[e / 2] + a0 * s[e / 2]);
                y[e] = (float)(b0 * c[(E + e) / 2] - b1 * s[(E + e) / 2]);
                y[e + 1] = (float)(b1 * c[(E + e) / 2] + b0 * s[(E + e) / 2]);
            }
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const real a0 = a.get(e), b0 = b.get(e);
                x[e] = (float)(a0 * c[e] - b0 * s[e]);
                y[e] = (float)(b0 * c[e] + a0 * s[e]);
            }
        }
        a.set(x);
        b.set(y);
    }
};

struct RopeRowsArgs {
    RopeSpec spec;
    const int32_t* positions;
    const void* in[2];    // queries, keys
    void* out[2];
    long in_stride[2], out_stride[2];  // of a token, in elements
    int heads[2];
    int num_tokens;
    int split;            // waves that share a token's heads
    int wide;             // work-groups of the grid in x
};

// grid (a.wide, split, z), four tokens to a work-group.  An in-place call leaves what does not turn.
template <int D, typename T>
__global__ __launch_bounds__(256) void rope_rows_kernel(RopeRowsArgs a)
{
    typedef RopeLane<D, T> L;
    constexpr int BATCH = 4;  // heads' parts under way
    __shared__ __attribute__((aligned(16))) typename L::real cs[4][2][64];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    L me;
    me.init(a.spec, lane);
    const int its0 = (a.heads[0] + L::HEADS - 1) / L::HEADS, its = its0 + (a.heads[1] + L::HEADS - 1) / L::HEADS;
    const int t = (blockIdx.z * a.wide + blockIdx.x) * 4 + w;
    if (t >= a.num_tokens) return;
    const int pos = a.positions[t];
    const T* const in[2] = {static_cast<const T*>(a.in[0]) + t * a.in_stride[0], static_cast<const T*>(a.in[1]) + t * a.in_stride[1]};
    T* const out[2] = {static_cast<T*>(a.out[0]) + t * a.out_stride[0], static_cast<T*>(a.out[1]) + t * a.out_stride[1]};
    const bool copy[2] = {a.in[0] != a.out[0], a.in[1] != a.out[1]};
    for (int it0 = blockIdx.y; it0 < its; it0 += BATCH * a.split) {
        RopePiece<T> x[BATCH][2];
        bool here[BATCH];
        T* dst[BATCH];
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
            const int it = it0 + k * a.split;
            const bool keys = it >= its0;
            const int h = (keys ? it - its0 : it) * L::HEADS + me.head;
            here[k] = it < its && h < (keys ? a.heads[1] : a.heads[0]) && (me.turns || (keys ? copy[1] : copy[0]));
            if (!here[k]) continue;
            const T* src = (keys ? in[1] : in[0]) + (long)h * D;
            dst[k] = (keys ? out[1] : out[0]) + (long)h * D;
            x[k][0].x = *reinterpret_cast<const u32x4_t*>(src + me.off[0]);
            x[k][1].x = *reinterpret_cast<const u32x4_t*>(src + me.off[1]);
        }
        if (it0 == (int)blockIdx.y)
            me.at(a.spec, lane < a.spec.R / 2 ? rope_turns(a.spec, lane) : 0.0, lane, pos, cs[w]);  // under the loads
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
            if (!here[k]) continue;
            me.turn(a.spec, x[k][0], x[k][1]);
            rope_store(dst[k] + me.off[0], x[k][0].x);
            rope_store(dst[k] + me.off[1], x[k][1].x);
        }
    }
}

struct PagedRopeArgs {
    PagedIoArgs io;       // k_rows, v_rows: the new keys and values
    RopeSpec spec;
    const void* q;
    void* q_out;
    const int32_t* pos_base;  // [S] or null
    long q_stride, q_out_stride, k_stride, v_stride;
    int H_q;
    int split, wide;      // as for rope_rows_kernel
};

// The place of row r (uniform over the wave): page and row in it, page -1 for none; and its
// position.  False for a row behind the last sequence's.
__device__ inline bool paged_rope_place(const PagedRopeArgs& a, int r, int& page, int& slot, int& pos)
{
    const int s = paged_owner(a.io, r);
    if (s < 0) return false;
    const int first = a.io.cu[s], end = a.io.cu[s + 1], len = a.io.lens[s];
    page = -1;
    slot = 0;
    if (r < first || first < 0) return false;
    const int key = r - first + len;
    pos = (int)((uint32_t)key + (uint32_t)(a.pos_base ? a.pos_base[s] : 0));
    if (len >= 0 && len <= a.io.max_len - (min(end, a.io.num_tokens) - first)) {
        const int e = a.io.block_table[(long)s * a.io.max_pages + (key >> a.io.page_shift)];
        page = (uint32_t)e < (uint32_t)a.io.num_pages ? e : -1;
        slot = key & ((1 << a.io.page_shift) - 1);
    }
    return true;
}

// A wave takes a token, or every split-th of the steps over its heads: queries, then keys,
// then values.  grid (a.wide, split, z), at least tokens / 4 and sequences / 64 work-groups.  A key row is rounded to the
// rows' type before it is quantised: the cache holds what rope and then the append leave.
template <int D, typename T, PagedForm FORM>
__global__ __launch_bounds__(256) void paged_rope_append_kernel(PagedRopeArgs a)
{
    typedef RopeLane<D, T> L;
    constexpr int BATCH = 4;
    __shared__ __attribute__((aligned(16))) typename L::real cs[4][2][64];
    __shared__ __attribute__((aligned(16))) T rows_s[FORM == kPlainRows ? 1 : 4][FORM == kPlainRows ? 16 : L::HEADS * D];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const PagedIoArgs& io = a.io;
    const int wg = blockIdx.z * a.wide + blockIdx.x;
    // the counts after the append, 64 sequences to a work-group
    if (blockIdx.y == 0 && w == 0 && wg <= (io.num_seqs - 1) / 64) {
        const int s = 64 * wg + lane;
        if (s < io.num_seqs) {
            const int n = io.lens[s], m = min(max(io.cu[s + 1], 0), io.num_tokens) - min(max(io.cu[s], 0), io.num_tokens);
            io.lens_out[s] = n >= 0 && m > 0 && n <= io.max_len - m ? n + m : n;
        }
    }
    const int t = wg * 4 + w;
    if (t >= io.num_tokens) return;
    int page = -1, slot = 0, pos = 0;
    L me;
    me.init(a.spec, lane);
    const int its_q = (a.H_q + L::HEADS - 1) / L::HEADS, its_k = (io.H_kv + L::HEADS - 1) / L::HEADS;
    const int its = its_q + 2 * its_k;
    const T* const q_row = static_cast<const T*>(a.q) + t * a.q_stride;
    const T* const k_row = static_cast<const T*>(io.k_rows) + t * a.k_stride;
    const T* const v_row = static_cast<const T*>(io.v_rows) + t * a.v_stride;
    const int v0 = L::E * me.unit, v1 = D / 2 + v0;  // a value's pieces
    for (int it0 = blockIdx.y; it0 < its; it0 += BATCH * a.split) {
        RopePiece<T> x[BATCH][2];
        int kind[BATCH], head[BATCH];  // 0 queries, 1 keys, 2 values, 3 nothing
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
            const int it = it0 + k * a.split;
            kind[k] = it < its_q ? 0 : it < its_q + its_k ? 1 : it < its ? 2 : 3;
            const int h0 = (kind[k] == 0 ? it : kind[k] == 1 ? it - its_q : it - its_q - its_k) * L::HEADS;
            head[k] = h0 + me.head;
            if (kind[k] == 3 || head[k] >= (kind[k] == 0 ? a.H_q : io.H_kv)) continue;
            const T* src = kind[k] == 0 ? q_row : kind[k] == 1 ? k_row : v_row;
            src += (long)head[k] * D;
            x[k][0].x = *reinterpret_cast<const u32x4_t*>(src + (kind[k] == 2 ? v0 : me.off[0]));
            x[k][1].x = *reinterpret_cast<const u32x4_t*>(src + (kind[k] == 2 ? v1 : me.off[1]));
        }
        if (it0 == (int)blockIdx.y) {  // under the first loads
            const double turns_i = lane < a.spec.R / 2 ? rope_turns(a.spec, lane) : 0.0;
            if (!paged_rope_place(a, t, page, slot, pos)) return;
            me.at(a.spec, turns_i, lane, pos, cs[w]);
        }
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
            if (kind[k] == 3 || (kind[k] > 0 && page < 0)) continue;
            const bool here = head[k] < (kind[k] == 0 ? a.H_q : io.H_kv);
            if (kind[k] < 2 && here) me.turn(a.spec, x[k][0], x[k][1]);
            const int o0 = kind[k] == 2 ? v0 : me.off[0], o1 = kind[k] == 2 ? v1 : me.off[1];
            if (kind[k] == 0) {
                if (here && (me.turns || a.q_out != a.q)) {
                    T* dst = static_cast<T*>(a.q_out) + t * a.q_out_stride + (long)head[k] * D;
                    rope_store_once(dst + o0, x[k][0].x);
                    rope_store_once(dst + o1, x[k][1].x);
                }
                continue;
            }
            unsigned char* pages = static_cast<unsigned char*>(kind[k] == 1 ? io.k_pages : io.v_pages);
            if constexpr (FORM == kPlainRows) {
                if (here) {
                    T* dst = reinterpret_cast<T*>(pages) + ((((long)page << io.page_shift) + slot) * io.H_kv + head[k]) * D;
                    rope_store_once(dst + o0, x[k][0].x);
                    rope_store_once(dst + o1, x[k][1].x);
                }
            } else {
                // the heads' rows in order, eight consecutive elements to a lane
                T* lin = rows_s[w];
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                __builtin_amdgcn_wave_barrier();
                if (here) {
                    *reinterpret_cast<u32x4_t*>(lin + me.head * D + o0) = x[k][0].x;
                    *reinterpret_cast<u32x4_t*>(lin + me.head * D + o1) = x[k][1].x;
                }
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                __builtin_amdgcn_wave_barrier();
                uint8_t* scales = kind[k] == 1 ? io.k_scales : io.v_scales;
#pragma unroll
                for (int g = lane; g < L::HEADS * D / 8; g += 64) {
                    const int h = head[k] - me.head + g / (D / 8), e = 8 * (g % (D / 8));
                    if (h >= io.H_kv) continue;  // all of a row's lanes
                    Row8<T> y;
                    y.load(lin + 8 * g);
                    int byte;
                    if constexpr (FORM == kE2m1Rows) {
                        const long at = e2m1_row(page, h, io.H_kv, io.page_shift, slot);
                        float v[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) v[j] = y.get(j);
                        *reinterpret_cast<uint32_t*>(pages + at * (D / 2) + e / 2) = quantise4(v, byte);
                        if (e % kE2m1Block == 0) scales[at * (D / kE2m1Block) + e / kE2m1Block] = (uint8_t)byte;
                    } else {
                        const long at = (((long)page << io.page_shift) + slot) * io.H_kv + h;
                        *reinterpret_cast<uint2*>(pages + at * D + e) = quantise8<D>(y, byte);
                        if (e == 0) scales[(((long)page * io.H_kv + h) << io.page_shift) + slot] = (uint8_t)byte;
                    }
                }
            }
        }
    }
}

}  // namespace pdec
