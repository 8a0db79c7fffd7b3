// Block tables on the GPU: pages from a pool's free list to the sequences that get new
// tokens, and back.
//
// The free list is a stack.  Reserving takes pages off its top in order (by sequence, then
// by place in the sequence), releasing puts them back in the opposite order, so that one
// undoes the other; both depend on nothing but their inputs.
//
// Two passes.  The first counts, a wave to a sequence's row of the table: the entries that
// lack a page, or whose page goes back.  In the second a work-group takes a few sequences,
// sums the counts of all sequences before them (1024 at a time, four to a lane: the sums
// are a few KB, and cheaper than a pass of their own), and then each wave deals a
// sequence's pages, each lane a token's position and row.  A batch of up to 64 sequences
// is one work-group's, in one launch.
//
// What bounds it: the chain of memory round trips (lengths, entries, the free list, the
// entries again).
#pragma once

#include "paged_common.h"

namespace pdec {

struct PagedTableArgs {
    const int32_t* first;  // reserve: new tokens; release: first keys kept, or null
    const int32_t* lens;   // reserve: keys before; release: keys kept
    int32_t* block_table;
    int32_t* free_pages;
    const int32_t* free_in;
    int32_t* free_out;
    int32_t* cu;           // reserve only, as the next two
    int32_t* positions;    // may be null
    int64_t* slots;        // may be null
    int2* counts;          // [S] pages and tokens, of the first pass
    int num_seqs, num_tokens, page_shift, num_pages, max_pages, max_len;
};

constexpr int kTableOne = 64;  // sequences that one work-group takes alone

__device__ inline bool table_there(const PagedTableArgs& a, int entry) { return (uint32_t)entry < (uint32_t)a.num_pages; }

// Sequence s: its new tokens (0 for a request that cannot be) and the entries [lo, hi) of
// its row that they need; or, releasing, the entries [lo, hi) that it keeps.
struct TableSeq {
    int n, len, lo, hi;
};

template <bool RESERVE>
__device__ inline TableSeq table_seq(const PagedTableArgs& a, int s)
{
    const int page = 1 << a.page_shift;
    TableSeq x = {0, a.lens[s], 0, 0};
    if constexpr (RESERVE) {
        x.n = a.first[s];
        if (x.n < 0 || x.len < 0 || x.len > a.max_len || x.n > a.max_len - x.len) x.n = 0;
        if (x.n > 0) {
            x.lo = x.len >> a.page_shift;
            x.hi = (x.len + x.n + page - 1) >> a.page_shift;
        }
    } else {
        const int from = a.first ? max(a.first[s], 0) : 0, len = min(max(x.len, 0), a.max_len);
        if (len > from) {
            x.lo = from >> a.page_shift;
            x.hi = (len + page - 1) >> a.page_shift;
        }
    }
    return x;
}

// Entries of a row that the wave looks at, 64 U from `at`, in order (reserve) or from the row's
// end (release): which of its U the lane's must be dealt with.
template <bool RESERVE, int U>
struct TableLook {
    int e[U], entry[U];
    uint64_t b[U];
    __device__ inline void look(const PagedTableArgs& a, const int32_t* row, const TableSeq& x, int at, int cols)
    {
        const int lane = paged_lane();
#pragma unroll
        for (int u = 0; u < U; ++u) {
            e[u] = RESERVE ? at + 64 * u + lane : cols - 1 - (at + 64 * u + lane);
            const bool in = RESERVE ? e[u] < x.hi : e[u] >= 0 && (e[u] < x.lo || e[u] >= x.hi);
            entry[u] = in ? row[e[u]] : RESERVE ? 0 : -1;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) b[u] = __ballot(table_there(a, entry[u]) != RESERVE);
    }
    __device__ inline int count() const
    {
        int n = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) n += __builtin_popcountll(b[u]);
        return n;
    }
};

// The wave's row: how many entries lack a page (reserve), or go back (release).
template <bool RESERVE>
__device__ inline int table_count(const PagedTableArgs& a, int s, const TableSeq& x, int cols)
{
    constexpr int U = 4;
    const int32_t* row = a.block_table + (long)s * a.max_pages;
    int n = 0;
    for (int at = RESERVE ? x.lo : 0; at < (RESERVE ? x.hi : cols); at += 64 * U) {
        TableLook<RESERVE, U> k;
        k.look(a, row, x, at, cols);
        n += k.count();
    }
    return n;
}

// Deals the wave's row its pages from free_pages[from], [from - 1], .. (reserve), or puts
// them to free_pages[from], [from + 1], ..
template <bool RESERVE>
__device__ inline void table_deal(const PagedTableArgs& a, int s, const TableSeq& x, int cols, int from)
{
    constexpr int U = 4;
    int32_t* row = a.block_table + (long)s * a.max_pages;
    const uint64_t below = (1ull << paged_lane()) - 1;
    for (int at = RESERVE ? x.lo : 0; at < (RESERVE ? x.hi : cols); at += 64 * U) {
        TableLook<RESERVE, U> k;
        k.look(a, row, x, at, cols);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = __builtin_popcountll(k.b[u] & below);
            if (k.b[u] >> paged_lane() & 1) {
                if constexpr (RESERVE) row[k.e[u]] = a.free_pages[from - i];
                else {
                    // (a page that is released twice would pass the list's end)
                    if (from + i < a.num_pages) a.free_pages[from + i] = k.entry[u];
                    row[k.e[u]] = -1;
                }
            }
            from += (RESERVE ? -1 : 1) * __builtin_popcountll(k.b[u]);
        }
    }
}

template <bool RESERVE>
__global__ __launch_bounds__(256) void paged_table_count_kernel(PagedTableArgs a)
{
    const int s = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (s >= a.num_seqs) return;
    const TableSeq x = table_seq<RESERVE>(a, s);
    const int n = table_count<RESERVE>(a, s, x, (a.max_len + (1 << a.page_shift) - 1) >> a.page_shift);
    if (paged_lane() == 0) a.counts[s] = make_int2(n, x.n);
}

// A work-group's sequences: all (ONE), or `WAVES` of them.  Releasing, the sequences are
// numbered from the last, so that the sums are of those behind.
template <bool RESERVE, bool ONE>
struct TableShape {
    static constexpr int THREADS = ONE ? 1024 : 256, WAVES = THREADS / 64, SEQS = ONE ? kTableOne : WAVES, CHUNK = 4 * THREADS;
};

template <bool RESERVE, bool ONE>
__global__ __launch_bounds__((TableShape<RESERVE, ONE>::THREADS)) void paged_table_kernel(PagedTableArgs a)
{
    typedef TableShape<RESERVE, ONE> C;
    __shared__ uint64_t wave_s[2][C::WAVES];
    __shared__ unsigned long long most_s[2];  // pages and tokens of the sequences that are served
    __shared__ int2 counts_s[ONE ? C::SEQS : 1];
    __shared__ int from_s[C::SEQS], token_s[C::SEQS];  // of each of the group's sequences; from -1: not served
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int cols = (a.max_len + (1 << a.page_shift) - 1) >> a.page_shift;
    const int top = min(max(a.free_in[0], 0), a.num_pages);
    const int s0 = blockIdx.x * C::SEQS, s1 = min(s0 + C::SEQS, a.num_seqs);  // the group's, by their numbers
    auto seq = [&](int i) { return RESERVE ? i : a.num_seqs - 1 - i; };
    TableSeq own[C::SEQS / C::WAVES];  // the wave's: s0 + w, s0 + w + WAVES, ..
#pragma unroll
    for (int k = 0; k < C::SEQS / C::WAVES; ++k) {
        const int i = s0 + w + k * C::WAVES;
        if (i < s1) own[k] = table_seq<RESERVE>(a, seq(i));
    }
    if constexpr (ONE) {
#pragma unroll
        for (int k = 0; k < C::SEQS / C::WAVES; ++k) {
            const int i = w + k * C::WAVES;
            if (i >= s1) break;
            const int n = table_count<RESERVE>(a, seq(i), own[k], cols);
            if (lane == 0) counts_s[i] = make_int2(n, own[k].n);
        }
    }
    if (tid < 2) most_s[tid] = 0;
    __syncthreads();

    uint64_t sum[2] = {0, 0};  // of the chunks before
    for (int c0 = 0; c0 < s1; c0 += C::CHUNK) {
        uint64_t x[2][4];  // inclusive sums over the lane's four
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = c0 + 4 * tid + j;
            int2 n = make_int2(0, 0);
            if (i < s1) n = ONE ? counts_s[ONE ? i : 0] : a.counts[seq(i)];
            x[0][j] = (uint32_t)n.x + (j ? x[0][j - 1] : 0);
            x[1][j] = (uint32_t)n.y + (j ? x[1][j - 1] : 0);
        }
        uint64_t total[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            uint64_t y = x[k][3];
#pragma unroll
            for (int off = 1; off < 64; off <<= 1) {
                const uint64_t z = __shfl_up(y, off);
                if (lane >= off) y += z;
            }
            if (lane == 63) wave_s[k][w] = y;
            total[k] = y - x[k][3];  // of the wave's lanes before
        }
        __syncthreads();
        uint64_t before[2], all[2] = {0, 0};
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            before[k] = sum[k] + total[k];
#pragma unroll
            for (int i = 0; i < C::WAVES; ++i) {
                if (i < w) before[k] += wave_s[k][i];
                all[k] += wave_s[k][i];
            }
            sum[k] += all[k];
        }
        uint64_t p = 0, t = 0;  // of the last that is served
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = c0 + 4 * tid + j;
            const uint64_t pj = before[0] + x[0][j], tj = before[1] + x[1][j];
            const bool served = i < s1 && (!RESERVE || (pj <= (uint64_t)top && tj <= (uint64_t)a.num_tokens));
            if (served) p = pj, t = tj;
            if (i >= s0 && i < s1) {
                const uint64_t p0 = before[0] + (j ? x[0][j - 1] : 0), t0 = before[1] + (j ? x[1][j - 1] : 0);
                from_s[i - s0] = !served ? -1 : RESERVE ? top - (int)p0 : (int)min((uint64_t)top + p0, (uint64_t)a.num_pages);
                token_s[i - s0] = (int)t0;
            }
        }
        if (p > 0) atomicMax(&most_s[0], (unsigned long long)p);
        if (t > 0) atomicMax(&most_s[1], (unsigned long long)t);
        __syncthreads();
    }

    if (tid == 0 && s1 == a.num_seqs)
        a.free_out[0] = RESERVE ? top - (int)most_s[0] : (int)min((uint64_t)top + sum[0], (uint64_t)a.num_pages);
#pragma unroll
    for (int k = 0; k < C::SEQS / C::WAVES; ++k) {
        const int i = s0 + w + k * C::WAVES;
        if (i >= s1) break;
        const int from = __builtin_amdgcn_readfirstlane(from_s[i - s0]);
        if (from >= 0) table_deal<RESERVE>(a, seq(i), own[k], cols, RESERVE ? from - 1 : from);
        if constexpr (RESERVE)
            if (lane == 0) a.cu[i + 1] = from >= 0 ? token_s[i - s0] + own[k].n : (int)most_s[1];
    }
    if constexpr (RESERVE) {
        if (tid == 0 && s0 == 0) a.cu[0] = 0;
        if (!a.positions && !a.slots) return;
        __syncthreads();  // the entries are written
        for (int i = s0; i < s1; ++i) {
            if (from_s[i - s0] < 0) break;  // nor are the later ones
            const TableSeq x = table_seq<RESERVE>(a, i);
            const int32_t* row = a.block_table + (long)i * a.max_pages;
            const int t0 = token_s[i - s0];
            for (int j = tid; j < x.n; j += C::THREADS) {
                const int key = x.len + j;
                if (a.positions) a.positions[t0 + j] = key;
                if (a.slots) a.slots[t0 + j] = ((int64_t)row[key >> a.page_shift] << a.page_shift) + (key & ((1 << a.page_shift) - 1));
            }
        }
    }
}

}  // namespace pdec
