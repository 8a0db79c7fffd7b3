// Writing rows to a paged cache and reading them back, and the join of two
// attention results.
//
// All three move memory: a row in, a row out, a few operations per element.
// 16-byte accesses; the sequence of a row is found once per wave by counting the
// offsets at or below it, 64 places at a time: one memory round trip for up to 64
// sequences, two for up to 4096.
//
// What bounds them: at serving sizes the call (the append of 32 tokens is 2.9 us on
// the device and 9 as a call), at large ones the bytes: 32768 rows of 4 heads of 128
// read from 8-bit pages (101 MB) 22 us, 4.6 TB/s; 16384 appended (67 MB) 12 us; 17472
// joined rows of 128 float32 (27 MB) 7.5 us, 3.6 TB/s.
#pragma once

#include "kernel_mfma.h"
#include "paged_common.h"

namespace pdec {

struct PagedIoArgs {
    const void* k_rows;  // append: k_new, v_new; read: k_out, v_out
    const void* v_rows;
    void* k_pages;
    void* v_pages;
    uint8_t* k_scales;
    uint8_t* v_scales;
    const int32_t* block_table;
    const int32_t* cu;
    const int32_t* lens;  // append: before; read: keys
    int32_t* lens_out;    // append
    int num_seqs, num_tokens, H_kv;
    int page_shift, num_pages, max_pages, max_len;
};

// Sequence of row t (uniform over the wave): as many whole sequences lie before it as
// ends cu[s + 1] at or below t; -1 for a row behind the last sequence's.
__device__ inline int paged_owner(const PagedIoArgs& a, int t)
{
    const int lane = paged_lane();
    int lo = 0, n = a.num_seqs;  // the number is in [lo, lo + n]
    while (n > 64) {
        const int step = (n + 63) / 64, i = lo + (lane + 1) * step;
        const int c = __builtin_popcountll(__ballot(i <= lo + n && a.cu[min(i, a.num_seqs)] <= t));
        lo += c * step;
        n = min(step, n - c * step);
    }
    const int below = lo + __builtin_popcountll(__ballot(lane < n && a.cu[min(lo + lane + 1, a.num_seqs)] <= t));
    return below < a.num_seqs ? below : -1;
}

// Eight consecutive elements of a row.
template <typename T>
struct Row8 {
    u32x4_t x[sizeof(T) / 2];
    __device__ inline void load(const void* p)
    {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) x[i] = static_cast<const u32x4_t*>(p)[i];
    }
    __device__ inline void store(void* p) const
    {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) static_cast<u32x4_t*>(p)[i] = x[i];
    }
    __device__ inline float get(int i) const
    {
        if constexpr (sizeof(T) == 4) return __uint_as_float(x[i >> 2][i & 3]);
        else return __uint_as_float((i & 1) ? x[0][i >> 1] & 0xffff0000u : x[0][i >> 1] << 16);
    }
    __device__ inline void set(const float (&v)[8])
    {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i >> 2][i & 3] = __float_as_uint(v[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[0][i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
        }
    }
};

// Eight elements of a row of D, D / 8 lanes to a row, as e4m3 with the row's
// power of two: its byte in `byte`, the same in all of the row's lanes.
// Infinities and NaNs are stored as NaN.  |x| 2^-k is at most 448, but for
// magnitudes beyond 448 * 2^119, which become that (a larger power of two would
// let a rounded-up value pass float32's range when read back).
template <int D, typename T>
__device__ inline uint2 quantise8(const Row8<T>& r, int& byte)
{
    uint32_t top = 0;  // |x| as its bits, which order as the values do
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t u = __float_as_uint(r.get(i)) & 0x7fffffffu;
        top = u < 0x7f800000u ? max(top, u) : top;
    }
#pragma unroll
    for (int off = 1; off < D / 8; off <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, off));
    // top = m 2^e, 1 <= m < 2, and 448 = 1.75 * 2^8: k = e - 8, one more where m > 1.75
    // (a top below 2^-126 has e <= -127 and gets the least k)
    int k = (int)(top >> 23) - 127 - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
    k = top ? min(max(k, -126), 119) : 0;
    byte = k + 127;
    const float inv = __uint_as_float((uint32_t)(127 - k) << 23);  // 2^-k, 2^-119 .. 2^126
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        const float x0 = r.get(i), x1 = r.get(i + 1);
        int v = 0;
        v = __builtin_amdgcn_cvt_pk_fp8_f32(fminf(fmaxf(x0 * inv, -448.f), 448.f), fminf(fmaxf(x1 * inv, -448.f), 448.f), v, false);
        if ((__float_as_uint(x0) & 0x7f800000u) == 0x7f800000u) v |= 0x7f;
        if ((__float_as_uint(x1) & 0x7f800000u) == 0x7f800000u) v |= 0x7f00;
        w[i / 4] |= ((uint32_t)v & 0xffffu) << (8 * (i & 2));
    }
    return make_uint2(w[0], w[1]);
}

// Where rows r0 .. r0 + N - 1 of the batch lie in the pool: page and row in it.
// page is -1 for a row without a place, -2 for one that exists but has no key
// (read).  A lane looks up a row, so that N rows take the round trips of one;
// the results are scalars.  `before`: lens counts the keys before the rows
// (append), else all keys (read).
template <int N>
struct PagedPlace {
    int page[N], slot[N];
};

template <int N>
__device__ inline void paged_place(const PagedIoArgs& a, int r0, bool before, PagedPlace<N>& p)
{
    const int r = r0 + min(paged_lane(), N - 1);
    int page = -1, slot = 0;
    int s = r0 < a.num_tokens ? paged_owner(a, r0) : -1;
    if (s >= 0 && r < a.num_tokens) {
        int first = a.cu[s], end = a.cu[s + 1], len = a.lens[s];
        if (r >= end) {  // a later sequence's: the first that ends behind r, mostly the next
            int hi = a.num_seqs;
            for (int step = 1; ++s < hi; step *= 2) {
                const int at = min(s + step - 1, hi - 1);
                if (a.cu[at + 1] > r) {
                    hi = at;
                    break;
                }
                s = at;
            }
            while (s < hi) {
                const int mid = s + (hi - s) / 2;
                if (a.cu[mid + 1] > r) hi = mid;
                else s = mid + 1;
            }
            if (s < a.num_seqs) {
                first = a.cu[s];
                end = a.cu[s + 1];
                len = a.lens[s];
            }
        }
        if (s < a.num_seqs && r >= first && first >= 0) {
            int key = r - first;
            bool ok;
            if (before) {
                ok = len >= 0 && len <= a.max_len - (min(end, a.num_tokens) - first);
                key += len;
            } else {
                ok = key < min(len, a.max_len);
                page = -2;
            }
            if (ok) {
                const int e = a.block_table[(long)s * a.max_pages + (key >> a.page_shift)];
                page = (uint32_t)e < (uint32_t)a.num_pages ? e : page;
                slot = key & ((1 << a.page_shift) - 1);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        p.page[i] = __builtin_amdgcn_readlane(page, i);
        p.slot[i] = __builtin_amdgcn_readlane(slot, i);
    }
}

// A wave takes N consecutive tokens of one tensor, eight elements a lane.
// grid (max(tokens / (4 N), sequences / 64), 2): few tokens a token per wave, for
// the latency; many four, with one look-up and all their loads under way.
template <int D, typename T, bool QUANT, int N>
__global__ __launch_bounds__(256) void paged_append_kernel(PagedIoArgs a)
{
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool is_v = blockIdx.y != 0;
    const int elems = a.H_kv * D, r0 = (blockIdx.x * 4 + w) * N;
    const T* src = static_cast<const T*>(is_v ? a.v_rows : a.k_rows) + (long)r0 * elems;
    Row8<T> row[N];
    auto load = [&](int e) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (r0 + i < a.num_tokens && e < elems) row[i].load(src + (long)i * elems + e);
    };
    load(8 * lane);  // under the look-ups
    // the counts after the append, 64 sequences to a work-group
    if (!is_v && w == 0) {
        const int s = 64 * blockIdx.x + lane;
        if (s < a.num_seqs) {
            const int n = a.lens[s], m = min(max(a.cu[s + 1], 0), a.num_tokens) - min(max(a.cu[s], 0), a.num_tokens);
            a.lens_out[s] = n >= 0 && m > 0 && n <= a.max_len - m ? n + m : n;
        }
    }
    PagedPlace<N> p;
    paged_place(a, r0, true, p);
    unsigned char* pages = static_cast<unsigned char*>(is_v ? a.v_pages : a.k_pages);
    uint8_t* scales = is_v ? a.v_scales : a.k_scales;
    for (int e = 8 * lane; e < elems; e += 512) {
        if (e >= 512) load(e);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (p.page[i] < 0) continue;
            const long at = ((long)p.page[i] << a.page_shift) + p.slot[i];
            unsigned char* dst = pages + (at * elems + e) * (QUANT ? 1 : (int)sizeof(T));
            if constexpr (QUANT) {
                int byte;
                *reinterpret_cast<uint2*>(dst) = quantise8<D>(row[i], byte);
                if (e % D == 0) scales[(((long)p.page[i] * a.H_kv + e / D) << a.page_shift) + p.slot[i]] = (uint8_t)byte;
            } else {
                row[i].store(dst);
            }
        }
    }
}

// A wave takes N consecutive rows of one tensor.  grid (rows / (4 N), 2).
template <int D, typename T, bool QUANT, int N>
__global__ __launch_bounds__(256) void paged_read_kernel(PagedIoArgs a)
{
    const int lane = threadIdx.x & 63;
    const bool is_v = blockIdx.y != 0;
    const int elems = a.H_kv * D;
    const int r0 = (blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * N;
    const unsigned char* pages = static_cast<const unsigned char*>(is_v ? a.v_pages : a.k_pages);
    const uint8_t* scales = is_v ? a.v_scales : a.k_scales;
    T* out = static_cast<T*>(const_cast<void*>(is_v ? a.v_rows : a.k_rows)) + (long)r0 * elems;
    PagedPlace<N> p;
    paged_place(a, r0, false, p);
    for (int e = 8 * lane; e < elems; e += 512) {
        Row8<T> row[N];
        uint2 x[N];
        uint32_t byte[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (p.page[i] < 0) continue;
            const long at = ((long)p.page[i] << a.page_shift) + p.slot[i];
            if constexpr (QUANT) {
                x[i] = *reinterpret_cast<const uint2*>(pages + at * elems + e);
                byte[i] = scales[(((long)p.page[i] * a.H_kv + e / D) << a.page_shift) + p.slot[i]];
            } else {
                row[i].load(pages + (at * elems + e) * (int)sizeof(T));
            }
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (p.page[i] == -1) continue;
            if (p.page[i] < 0) {
                const float z[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                row[i].set(z);
            } else if constexpr (QUANT) {
                const float sc = paged_scale(byte[i], 0);
                float v[8];
#pragma unroll
                for (int k = 0; k < 8; k += 4) {
                    const int word = (int)(k ? x[i].y : x[i].x);
                    const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8(word, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(word, true);
                    v[k] = lo.x * sc, v[k + 1] = lo.y * sc, v[k + 2] = hi.x * sc, v[k + 3] = hi.y * sc;
                }
                row[i].set(v);
            }
            row[i].store(out + (long)i * elems + e);
        }
    }
}

// Eight elements per lane; a row's lanes are in one work-group.
template <int D, typename T>
__global__ __launch_bounds__(256) void merge_states_kernel(long rows, const void* oa, const float* la, const void* ob,
                                                           const float* lb, void* out, float* lse)
{
    constexpr int PER = D / 8;
    const long i = (long)blockIdx.x * 256 + threadIdx.x, r = i / PER;
    float x = 0.f, y = 0.f;
    Row8<T> p, q;
    const bool in = r < rows;
    if (in) {
        p.load(static_cast<const T*>(oa) + 8 * i);
        q.load(static_cast<const T*>(ob) + 8 * i);
        x = la[r];
        y = lb[r];
    }
    __syncthreads();  // in place: one lane writes the lse that the row's other lanes read
    if (!in) return;
    const float m = fmaxf(x, y);
    const bool use_a = x != kNegInf, use_b = y != kNegInf;
    const float wa = use_a ? expf(x - m) : 0.f, wb = use_b ? expf(y - m) : 0.f;
    const float total = wa + wb;
    const float inv = (use_a | use_b) ? 1.f / total : 0.f;
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const float u = use_a ? wa * p.get(k) : 0.f;
        v[k] = (use_b ? fmaf(wb, q.get(k), u) : u) * inv;
    }
    p.set(v);
    p.store(static_cast<T*>(out) + 8 * i);
    if (lse && i == r * PER) lse[r] = (use_a | use_b) ? m + logf(total) : kNegInf;
}

}  // namespace pdec
