// Block tables on the GPU: pages from a pool's free list to the sequences that get new
// tokens, and back.
//
// The free list is a stack.  Reserving takes pages off its top in order (by sequence, then
// by place in the sequence), releasing puts them back in the opposite order, so that one
// undoes the other; both depend on nothing but their inputs.
//
// Two passes.  The first counts, a wave to a sequence's row of the table: the entries that
// lack a page, or whose page goes back.  In the second a work-group takes a few sequences,
// sums the counts of all sequences before them (2048 at a time, eight to a lane: the counts
// are a few KB, and summing them cheaper than a pass of its own), and then each wave deals a
// sequence's pages, each lane a token's position and row.  A batch of up to 64 sequences
// is one work-group's, in one launch.  Of many sequences a pass between the two sums each
// 2048, and a work-group sums those sums and one 2048.
//
// What bounds it: the chain of memory round trips: lengths, entries, the sums, the free
// list, the entries again.  32 sequences a token each: 5.8 us on the device, 7.6 as a call.
// 1500 sequences of up to 511 new tokens and 9000 keys (300000 tokens served), reserved and released:
// 27.5 us for the two calls; the kernels 3.3 and 14.9, 3.3 and 7.9, of which positions and
// slots are 3.7.  Few sequences of many tokens keep their one work-group at positions and slots:
// 64 of 512 tokens 41 us the pair of calls, of 4096 212 (65, by two passes: 21 and 47).
#pragma once

#include "kernel_mfma.h"
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
    int2* counts;          // [S, even] pages and tokens, of the first pass; releasing, from the last sequence
    ulonglong2* totals;    // [S / kTableChunk] theirs of kTableChunk sequences each, if asked for
    int num_seqs, num_tokens, page_shift, num_pages, max_pages, max_len;
};

constexpr int kTableOne = 64;  // sequences that one work-group takes alone
constexpr int kTableChunk = 2048;  // sequences whose counts a work-group sums at a time

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
    int at, cols, entry[U];
    __device__ inline int place(int u) const  // the lane's u-th entry
    {
        const int i = at + 64 * u + paged_lane();
        return RESERVE ? i : cols - 1 - i;
    }
    __device__ inline void load(const int32_t* row, const TableSeq& x, int first, int columns)
    {
        at = first;
        cols = columns;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int e = place(u);
            entry[u] = row[RESERVE ? max(min(e, x.hi - 1), 0) : max(e, 0)];  // no branch: all under way at once
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int e = place(u);
            const bool in = RESERVE ? e < x.hi : e >= 0 && (e < x.lo || e >= x.hi);
            entry[u] = in ? entry[u] : RESERVE ? 0 : -1;
        }
    }
    __device__ inline uint64_t found(const PagedTableArgs& a, int u) const { return __ballot(table_there(a, entry[u]) != RESERVE); }
    __device__ inline int count(const PagedTableArgs& a) const
    {
        int n = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) n += table_there(a, entry[u]) != RESERVE ? 1 : 0;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) n += __shfl_xor(n, off);
        return __builtin_amdgcn_readfirstlane(n);
    }
    // give(entry's place, entry, number among those found) for each entry found
    template <typename F>
    __device__ inline void each(const PagedTableArgs& a, F give) const
    {
        int n = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint64_t b = found(a, u);
            if (b) give((b >> paged_lane() & 1) != 0, place(u), entry[u], n + __builtin_popcountll(b & ((1ull << paged_lane()) - 1)));
            n += __builtin_popcountll(b);
        }
    }
    // Deals the entries found pages from free_pages[from], [from - 1], .. (reserve), or puts
    // theirs to free_pages[from], [from + 1], ..
    __device__ inline void deal(const PagedTableArgs& a, int32_t* row, int from) const
    {
        each(a, [&](bool mine, int e, int page, int i) {
            if (!mine) return;
            if constexpr (RESERVE) row[e] = a.free_pages[from - i];
            else {
                // (a page that is released twice would pass the list's end)
                if (from + i < a.num_pages) a.free_pages[from + i] = page;
                row[e] = -1;
            }
        });
    }
};

// A row's looks, U entries to a lane at a time: one memory round trip for most rows.
template <bool RESERVE> constexpr int kTableLook = RESERVE ? 4 : 16;
template <bool RESERVE>
__device__ inline int table_begin(const TableSeq& x) { return RESERVE ? x.lo : 0; }
template <bool RESERVE>
__device__ inline int table_end(const TableSeq& x, int cols) { return RESERVE ? x.hi : cols; }

// The wave's row: how many entries lack a page (reserve), or go back (release).
template <bool RESERVE>
__device__ inline int table_count(const PagedTableArgs& a, int s, const TableSeq& x, int cols)
{
    constexpr int U = kTableLook<RESERVE>;
    int n = 0;
    for (int at = table_begin<RESERVE>(x); at < table_end<RESERVE>(x, cols); at += 64 * U) {
        TableLook<RESERVE, U> k;
        k.load(a.block_table + (long)s * a.max_pages, x, at, cols);
        n += k.count(a);
    }
    return n;
}

template <bool RESERVE>
__device__ inline void table_deal(const PagedTableArgs& a, int s, const TableSeq& x, int cols, int from)
{
    constexpr int U = kTableLook<RESERVE>;
    int32_t* row = a.block_table + (long)s * a.max_pages;
    for (int at = table_begin<RESERVE>(x); at < table_end<RESERVE>(x, cols); at += 64 * U) {
        TableLook<RESERVE, U> k;
        k.load(row, x, at, cols);
        k.deal(a, row, from);
        from += (RESERVE ? -1 : 1) * k.count(a);
    }
}

template <bool RESERVE>
__global__ __launch_bounds__(256) void paged_table_count_kernel(PagedTableArgs a)
{
    const int s = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (s >= a.num_seqs) return;
    const TableSeq x = table_seq<RESERVE>(a, s);
    const int n = table_count<RESERVE>(a, s, x, (a.max_len + (1 << a.page_shift) - 1) >> a.page_shift);
    if (paged_lane() == 0) a.counts[RESERVE ? s : a.num_seqs - 1 - s] = make_int2(n, x.n);
}

// Sums of pages and tokens, in 64 bits: a batch outside the contract may ask for anything.
struct TableSum {
    uint64_t p, t;
    __device__ inline TableSum operator+(const TableSum& y) const { return TableSum{p + y.p, t + y.t}; }
};

__device__ inline TableSum table_scan(TableSum x)  // inclusive, over the wave
{
    const int lane = paged_lane();
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const TableSum y = {__shfl_up(x.p, off), __shfl_up(x.t, off)};
        if (lane >= off) x = x + y;
    }
    return x;
}

// The work-group's tokens: positions and rows of the pool.  token[i], i < count: the first
// token of its sequence i; len[i] its keys before; end: behind its last; page_of(i, entry):
// what the table holds.
template <int THREADS, typename F>
__device__ inline void table_tokens(const PagedTableArgs& a, int count, const int* token, const int* len, int first, int end, F page_of)
{
    constexpr int U = 4;
    for (int t0 = first + (int)threadIdx.x; t0 < end; t0 += U * THREADS) {
        int key[U], entry[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int t = t0 + u * THREADS;
            int lo = 0, n = count - 1;  // the last sequence that begins at or before t
            while (n > 0) {
                const int half = (n + 1) / 2;
                if (token[lo + half] <= t) lo += half, n -= half;
                else n = half - 1;
            }
            key[u] = len[lo] + t - token[lo];
            entry[u] = t < end ? page_of(lo, key[u] >> a.page_shift) : 0;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int t = t0 + u * THREADS;
            if (t >= end) break;
            if (a.positions) a.positions[t] = key[u];
            if (a.slots) a.slots[t] = ((int64_t)entry[u] << a.page_shift) + (key[u] & ((1 << a.page_shift) - 1));
        }
    }
}

// Up to kTableOne sequences: one work-group, their sums a wave's scan.
// Releasing, the sequences are numbered from the last, so that the sums are of those behind.
// PER: sequences of a wave, up to four.
constexpr int kTableWaves = 16;
template <bool RESERVE, int PER>
__global__ __launch_bounds__(64 * kTableWaves) void paged_table_one_kernel(PagedTableArgs a)
{
    constexpr int U = RESERVE ? 4 : 32 / PER;  // a lane's entries of a row at first: as many as the registers hold
    __shared__ int2 counts_s[kTableOne];
    __shared__ int token_s[kTableOne], len_s[kTableOne];
    const int lane = paged_lane(), w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), S = a.num_seqs;
    const int cols = (a.max_len + (1 << a.page_shift) - 1) >> a.page_shift;
    const int top = min(max(a.free_in[0], 0), a.num_pages);
    auto seq = [&](int i) { return RESERVE ? i : S - 1 - i; };
    TableSeq x[PER];
    TableLook<RESERVE, U> look[PER];  // the rows' first entries, all asked for at once
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int i = w + k * kTableWaves;
        x[k] = i < S ? table_seq<RESERVE>(a, seq(i)) : TableSeq{0, 0, 0, 0};
    }
    // a reservation's first pages, in case
    const int ahead = RESERVE && lane < top ? a.free_pages[top - 1 - lane] : 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int i = w + k * kTableWaves;
        look[k].load(a.block_table + (long)seq(min(i, S - 1)) * a.max_pages, x[k], table_begin<RESERVE>(x[k]), i < S ? cols : 0);
    }
    int n[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int i = w + k * kTableWaves;
        n[k] = look[k].count(a);
        const int next = table_begin<RESERVE>(x[k]) + 64 * U;
        if (i < S && next < table_end<RESERVE>(x[k], cols)) n[k] = table_count<RESERVE>(a, seq(i), x[k], cols);  // a longer row
        if (lane == 0 && i < S) {
            counts_s[i] = make_int2(n[k], x[k].n);
            len_s[i] = x[k].len;
        }
    }
    __syncthreads();
    // every wave forms the sums
    const int2 mine = lane < S ? counts_s[lane] : make_int2(0, 0);
    const TableSum own = {(uint32_t)mine.x, (uint32_t)mine.y}, sum = table_scan(own);
    const bool served = lane < S && (!RESERVE || (sum.p <= (uint64_t)top && sum.t <= (uint64_t)a.num_tokens));
    const int count = __builtin_popcountll(__ballot(served));  // the first so many
    const int pages = count > 0 ? __builtin_amdgcn_readlane((int)min(sum.p, (uint64_t)INT32_MAX), count - 1) : 0;
    const int tokens = count > 0 ? __builtin_amdgcn_readlane((int)sum.t, count - 1) : 0;
    const int p0 = (int)min(sum.p - own.p, (uint64_t)a.num_pages), t0 = (int)(sum.t - own.t);
    if (w == 0) {
        if (lane == 0) a.free_out[0] = RESERVE ? top - pages : (int)min((long)top + pages, (long)a.num_pages);
        if constexpr (RESERVE) {
            if (lane == 0) a.cu[0] = 0;
            if (lane < S) a.cu[lane + 1] = lane < count ? t0 + mine.y : tokens;
            if (lane < S) token_s[lane] = t0;
        }
    }
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int i = w + k * kTableWaves;
        if (i >= count || n[k] == 0) continue;
        const int at = __builtin_amdgcn_readlane(p0, i);
        int32_t* row = a.block_table + (long)seq(i) * a.max_pages;
        if (table_begin<RESERVE>(x[k]) + 64 * U < table_end<RESERVE>(x[k], cols))
            table_deal<RESERVE>(a, seq(i), x[k], cols, RESERVE ? top - 1 - at : min(top + at, a.num_pages));
        else if (RESERVE && at + n[k] <= 64) {
            // from the pages that were asked for ahead
            look[k].each(a, [&](bool mine, int e, int, int j) {
                const int page = __shfl(ahead, at + j);
                if (mine) row[e] = page;
            });
        } else {
            look[k].deal(a, row, RESERVE ? top - 1 - at : min(top + at, a.num_pages));
        }
    }
    if constexpr (RESERVE) {
        if (!a.positions && !a.slots) return;
        __syncthreads();  // the entries are written
        table_tokens<64 * kTableWaves>(a, count, token_s, len_s, 0, tokens,
                                       [&](int i, int e) { return a.block_table[(long)i * a.max_pages + e]; });
    }
}

// A work-group sums the counts of kTableChunk sequences.
__global__ __launch_bounds__(256) void paged_table_totals_kernel(PagedTableArgs a)
{
    constexpr int WAVES = 4, PER = kTableChunk / 256;
    __shared__ TableSum wave_s[WAVES];
    const int first = blockIdx.x * kTableChunk + PER * (int)threadIdx.x;
    TableSum x = {0, 0};
#pragma unroll
    for (int j = 0; j < PER; j += 2) {
        if (first + j >= a.num_seqs) break;
        const int4 n = *reinterpret_cast<const int4*>(a.counts + first + j);
        x = x + TableSum{(uint32_t)n.x, (uint32_t)n.y};
        if (first + j + 1 < a.num_seqs) x = x + TableSum{(uint32_t)n.z, (uint32_t)n.w};
    }
    x = table_scan(x);
    if (paged_lane() == 63) wave_s[threadIdx.x >> 6] = x;
    __syncthreads();
    if (threadIdx.x > 0) return;
    x = wave_s[0];
    for (int i = 1; i < WAVES; ++i) x = x + wave_s[i];
    a.totals[blockIdx.x] = make_ulonglong2(x.p, x.t);
}

// More sequences: four to a work-group, the counts of the first pass summed up to them, whole
// chunks by their totals.
template <bool RESERVE, bool TOTALS>
__global__ __launch_bounds__(256) void paged_table_kernel(PagedTableArgs a)
{
    constexpr int WAVES = 4, PER = 8, CHUNK = 64 * WAVES * PER;
    static_assert(CHUNK == kTableChunk && CHUNK % WAVES == 0, "a work-group's sequences are of one chunk");
    __shared__ TableSum wave_s[WAVES];
    __shared__ int fit_s;
    __shared__ unsigned long long most_s[2];  // pages and tokens of the sequences that are served
    __shared__ int from_s[WAVES], need_s[WAVES], token_s[WAVES], len_s[WAVES];  // from -1: not served
    constexpr int LOOK = 64 * kTableLook<RESERVE>;
    __shared__ int page_s[RESERVE ? WAVES : 1][RESERVE ? LOOK : 1], long_s[WAVES];  // a row's pages, unless they are more
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int cols = (a.max_len + (1 << a.page_shift) - 1) >> a.page_shift;
    const int top = min(max(a.free_in[0], 0), a.num_pages);
    const int s0 = blockIdx.x * WAVES, s1 = min(s0 + WAVES, a.num_seqs);  // the group's, by their numbers
    auto seq = [&](int i) { return RESERVE ? i : a.num_seqs - 1 - i; };
    TableSeq own = {0, 0, 0, 0};
    if (s0 + w < s1) own = table_seq<RESERVE>(a, seq(s0 + w));
    int32_t* const row = a.block_table + (long)seq(min(s0 + w, s1 - 1)) * a.max_pages;
    TableLook<RESERVE, kTableLook<RESERVE>> look;  // the row's first entries, under the sums
    look.load(row, own, table_begin<RESERVE>(own), cols);
    const bool is_long = table_begin<RESERVE>(own) + LOOK < table_end<RESERVE>(own, cols);
    if (lane == 0) {
        len_s[w] = own.len;
        long_s[w] = is_long;
    }
    if (tid < 2) most_s[tid] = 0;

    TableSum sum = {0, 0};  // of the chunks before
    int chunk = 0, last_chunk = s0 / CHUNK;
    if constexpr (TOTALS) {
        // whole chunks that are served, in front of the group's; the first that is not is the last to look at
        if (tid == 0) fit_s = 0;
        __syncthreads();
        for (int i0 = 0; i0 < last_chunk; i0 += 256) {
            const int i = i0 + tid;
            const ulonglong2 n = i < last_chunk ? a.totals[i] : make_ulonglong2(0, 0);
            const TableSum y = table_scan(TableSum{n.x, n.y});
            if (lane == 63) wave_s[w] = y;
            __syncthreads();
            TableSum in = sum + y;
#pragma unroll
            for (int k = 0; k < WAVES; ++k) {
                if (k < w) in = in + wave_s[k];
                sum = sum + wave_s[k];
            }
            const bool fits = i < last_chunk && (!RESERVE || (in.p <= (uint64_t)top && in.t <= (uint64_t)a.num_tokens));
            const int n_fit = __builtin_popcountll(__ballot(fits));
            if (fits && lane == n_fit - 1) {  // the sums grow, so the wave's first n_fit
                atomicMax(&most_s[0], (unsigned long long)in.p);
                atomicMax(&most_s[1], (unsigned long long)in.t);
                atomicAdd(&fit_s, n_fit);
            }
            __syncthreads();
        }
        chunk = fit_s;
        sum = TableSum{most_s[0], most_s[1]};
        if (chunk < last_chunk) {
            if (tid < WAVES) from_s[tid] = -1;
            last_chunk = chunk;
        }
        __syncthreads();
    }
    for (; chunk <= last_chunk; ++chunk) {
        const int c0 = chunk * CHUNK;
        int4 n[PER / 2];
#pragma unroll
        for (int j = 0; j < PER / 2; ++j) {
            const int i = c0 + PER * tid + 2 * j;
            n[j] = i < s1 ? *reinterpret_cast<const int4*>(a.counts + i) : make_int4(0, 0, 0, 0);
            if (i + 1 >= s1) n[j].z = n[j].w = 0;
        }
        TableSum x[PER];  // inclusive sums over the lane's
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            x[j] = j & 1 ? TableSum{(uint32_t)n[j / 2].z, (uint32_t)n[j / 2].w} : TableSum{(uint32_t)n[j / 2].x, (uint32_t)n[j / 2].y};
            if (j) x[j] = x[j] + x[j - 1];
        }
        const TableSum y = table_scan(x[PER - 1]);
        if (lane == 63) wave_s[w] = y;
        __syncthreads();
        TableSum before = {sum.p + y.p - x[PER - 1].p, sum.t + y.t - x[PER - 1].t};
#pragma unroll
        for (int i = 0; i < WAVES; ++i) {
            if (i < w) before = before + wave_s[i];
            sum = sum + wave_s[i];
        }
        TableSum last = {0, 0};  // of the last that is served
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int i = c0 + PER * tid + j;
            const TableSum in = before + x[j], ex = j ? before + x[j - 1] : before;
            const bool served = i < s1 && (!RESERVE || (in.p <= (uint64_t)top && in.t <= (uint64_t)a.num_tokens));
            if (served) last = in;
            if (i >= s0 && i < s1) {
                from_s[i - s0] = !served ? -1 : RESERVE ? top - (int)ex.p : (int)min((uint64_t)top + ex.p, (uint64_t)a.num_pages);
                need_s[i - s0] = (int)(in.p - ex.p);
                token_s[i - s0] = (int)ex.t;
            }
        }
        if (last.p > 0) atomicMax(&most_s[0], (unsigned long long)last.p);
        if (last.t > 0) atomicMax(&most_s[1], (unsigned long long)last.t);
        __syncthreads();
    }

    if (tid == 0 && s1 == a.num_seqs)
        a.free_out[0] = RESERVE ? top - (int)most_s[0] : (int)min((uint64_t)top + sum.p, (uint64_t)a.num_pages);
    if (s0 + w < s1) {
        const int from = __builtin_amdgcn_readfirstlane(from_s[w]);
        if constexpr (RESERVE) {
#pragma unroll
            for (int u = 0; u < kTableLook<RESERVE>; ++u)
                if (look.place(u) < own.hi) page_s[w][64 * u + lane] = look.entry[u];
        }
        if (from >= 0 && need_s[w] > 0) {
            if (is_long) table_deal<RESERVE>(a, seq(s0 + w), own, cols, RESERVE ? from - 1 : from);
            else if constexpr (RESERVE)
                look.each(a, [&](bool mine, int e, int, int i) {
                    if (mine) page_s[w][e - own.lo] = row[e] = a.free_pages[from - 1 - i];
                });
            else look.deal(a, row, from);
        }
        if constexpr (RESERVE)
            if (lane == 0) a.cu[s0 + w + 1] = from >= 0 ? token_s[w] + own.n : (int)most_s[1];
    }
    if constexpr (RESERVE) {
        if (tid == 0 && s0 == 0) a.cu[0] = 0;
        if (!a.positions && !a.slots) return;
        bool any = false;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) any |= long_s[i] != 0;
        if (any) __syncthreads();  // the entries are written
        else lds_barrier();
        int count = 0;
        while (count < s1 - s0 && from_s[count] >= 0) ++count;  // none behind one that is not served
        if (count == 0) return;
        const int first = token_s[0], end = count < s1 - s0 ? (int)most_s[1] : (int)sum.t;
        table_tokens<256>(a, count, token_s, len_s, first, end, [&](int i, int e) {
            return any ? a.block_table[(long)(s0 + i) * a.max_pages + e] : page_s[i][e - (len_s[i] >> a.page_shift)];
        });
    }
}

}  // namespace pdec
