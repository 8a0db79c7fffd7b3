// Attention over paged caches: arguments, the division of the work, and what
// its kernels share.
//
// A sequence's new tokens have R = n G query rows per kv head (r = token * G +
// head of the group), all against the same keys.  They are cut into groups of
// `rows` rows; a (kv head, sequence, row group) is a pair of rows and keys that
// one work-group can take, in 64-key units up to the last key that the group's
// last row sees.  The units of all pairs, one after another (by head, then
// sequence, then row group), are dealt in equal runs to `workers` work-groups.
// Heads come first so that neighbours, which share an XCD's cache, read the same
// keys (by head last, 2048 tokens over 32768 keys took 1140 us for 1084 at 8 kv
// heads, 992 for 981 at 4).
// Lengths are known on the device only, and differ: a sequence of 100 keys and
// one of 30000 in one batch, or the row groups of a causal chunk, still give
// every work-group the same number of units.  A run is a few whole pairs and
// at most one cut pair at each end; a work-group writes whole pairs to the
// output and a cut pair's state (reference max, normaliser, unnormalised
// output, all float32) to one of its two slots, and a finish pass joins a cut
// pair's slots in the order of the work-groups.  So the workspace depends on
// the number of work-groups only, and repeated calls agree bit for bit.
// A pair's start has a price beside its units (`pad` units: its queries, an
// empty ring, the plain loop at its end), which counts in the deal.
#pragma once

#include "pdec_common.h"

namespace pdec {

// One launch's arguments.
struct PagedArgs {
    const void* q;
    const void* k_pages;
    const void* v_pages;
    const uint8_t* k_scales;
    const uint8_t* v_scales;
    const int32_t* block_table;
    const int32_t* cu_tokens;
    const int32_t* seq_lens;
    void* out;
    float* lse;       // may be null
    float* part_o;    // [2 workers, heads, rows, D]
    float* part_ml;   // [2 workers, heads, rows, 2]
    int4* cut;        // a cut pair's (first work-group, last, pair of its head, head); first = -1: not cut
    int num_seqs, num_tokens, H_q, H_kv, G;
    int page_shift, num_pages, max_pages, max_chunk, max_len, causal;
    float qscale;     // softmax scale * log2(e)
    int rows;         // query rows per item and head
    int heads;        // kv heads of a pair (kernel_paged_few.h), 1 elsewhere
    int groups;       // row groups per (kv head, sequence), at most
    int rows_from;    // this launch serves the sequences with rows_from <= R <= rows_to
    int rows_to;
    int workers;      // work-groups that share the units, a multiple of 8
    int least;        // units per work-group, at least
    int pad;          // price of a pair's start, in units
    int blocks;       // work-groups of the launch, a multiple of 8
    int whole;        // 1: work-group i takes pair i whole, nothing is cut
    int by_pair;      // 1: cut[] is indexed by pair, 0: by the work-group a pair begins in
};

struct PagedSeq {
    int t0, n, L;  // first new token, their number, keys
};

__device__ inline PagedSeq paged_seq(const PagedArgs& a, int s)
{
    PagedSeq x;
    x.t0 = min(max(a.cu_tokens[s], 0), a.num_tokens);
    const int t1 = min(max(a.cu_tokens[s + 1], 0), a.num_tokens);
    x.n = min(max(t1 - x.t0, 0), a.max_chunk);
    x.L = min(max(a.seq_lens[s], 0), a.max_len);
    return x;
}

// Keys that new token i sees: the first so many.
__device__ inline int paged_seen(const PagedArgs& a, const PagedSeq& x, int i)
{
    return a.causal ? min(max(x.L - x.n + i + 1, 0), x.L) : x.L;
}

// A work-group's place in its run.  Positions count every pair's pad and units,
// the pad first.  Uniform over the work-group.
struct PagedRun {
    int w;          // its number
    int head, s, group;  // the pair at hand: kv head (or `heads` of them), sequence, row group
    PagedSeq seq;
    int u, units;   // next position in it, and its units
    int left;       // positions left of the run
    int pos;        // next position in the list of all
    int per, more;  // positions per work-group, the first `more` one more
};

// What to do next: units [u0, u1) of a pair.
struct PagedPart {
    int head, s, group, u0, u1;
    PagedSeq seq;
    bool whole;     // all of the pair
    int slot;       // where its state goes if not
    int end;        // position behind the pair
};

__device__ inline int paged_lane() { return (int)__builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0)); }

__device__ inline int paged_units_of(const PagedArgs& a, const PagedSeq& x, int group)
{
    const int R = x.n * a.G, row0 = group * a.rows;
    if (row0 >= R || R < a.rows_from || R > a.rows_to) return 0;
    const int last = min(R, row0 + a.rows) - 1;
    return max(1, (paged_seen(a, x, last / a.G) + kUnit - 1) / kUnit);
}

// Units of pair j = sequence * groups + row group (the same for every head);
// 0 where there are no such rows, at least 1 where there are.
__device__ inline int paged_units(const PagedArgs& a, int j)
{
    const int s = j / a.groups;
    return paged_units_of(a, paged_seq(a, s), j - s * a.groups);
}

// False if the work-group has nothing to do.  Every wave computes the same; one
// lane of the work-group (the caller says which) notes for the finish pass what is cut.
__device__ inline bool paged_begin(const PagedArgs& a, int w, PagedRun& r, bool note)
{
    const int J = a.num_seqs * a.groups, lane = paged_lane(), sets = a.H_kv / a.heads;
    if (note && !a.whole && !a.by_pair) a.cut[w] = make_int4(-1, 0, 0, 0);  // unless a pair is cut below
    int j;
    r.w = w;
    r.u = 0;
    if (a.whole) {
        if (w >= J * sets) return false;
        r.head = w / J;
        j = w - r.head * J;
        r.pos = 0;
    } else {
        // Inclusive, over the lanes.  Sums saturate: a head's positions and those of all
        // heads fit 30 bits by the host's bounds on the sizes, but offsets outside the
        // contract (each of many sequences with all of the tokens) pass 32 bits.
        auto scan = [&](uint32_t x) {
#pragma unroll
            for (int off = 1; off < 64; off <<= 1) {
                const uint32_t y = __shfl_up(x, off);
                if (lane >= off) x = __builtin_elementwise_add_sat(x, y);
            }
            return x;
        };
        // A lane's pair, or where there are many its sequence with all its groups: most of
        // a mixed batch's sequences have one group of as many as the longest chunk's bound
        // allows (200 sequences, one of 2048 new tokens: 335 us by pairs, 228 by sequences;
        // 64, one of 1024: 128 and 107).  Few sequences of many groups each would keep a
        // lane counting (one chunk of 32768 tokens, 896 groups: 7.67 and 7.80 ms; 64 chunks
        // of 14 groups 544 and 561 us).
        const bool by_seq = J > 1024 && a.num_seqs > 16;
        const int items = by_seq ? a.num_seqs : J;
        PagedSeq x = {0, 0, 0};
        auto cost = [&](int k) {
            if (k >= items) return 0;
            if (!by_seq) {
                const int s = k / a.groups;
                x = paged_seq(a, s);
                const int n = paged_units_of(a, x, k - s * a.groups);
                return n > 0 ? n + a.pad : 0;
            }
            x = paged_seq(a, k);
            int n = 0;
            for (int g = 0; g < a.groups; ++g) {
                const int u = paged_units_of(a, x, g);
                if (u == 0) break;
                n += u + a.pad;
            }
            return n;
        };
        auto last = [](uint32_t x) { return (uint32_t)__builtin_amdgcn_readlane((int)x, 63); };
        int n = cost(lane);
        uint32_t incl = scan(n), sum = last(incl);
        for (int j0 = 64; j0 < items; j0 += 64) sum = __builtin_elementwise_add_sat(sum, last(scan(cost(j0 + lane))));
        if ((uint64_t)sum * (uint32_t)sets > INT32_MAX / 2) return false;  // lengths outside the contract
        const int total = (int)sum;
        const int workers = min(a.workers, max(total * sets / a.least, 1));
        if (w >= workers || total == 0) return false;
        r.per = total * sets / workers;
        r.more = total * sets - r.per * workers;
        r.pos = w * r.per + min(w, r.more);
        r.left = r.per + (w < r.more ? 1 : 0);
        r.head = r.pos / total;
        int rest = r.pos - r.head * total, j0 = 0;
        if (items > 64) incl = scan(n = cost(lane));
        while (true) {
            const uint32_t all = last(incl);  // scalar, as everything that leaves the loop
            if ((uint32_t)rest < all) break;
            rest -= (int)all;
            j0 += 64;
            if (j0 >= items) return false;  // lengths that changed under the call
            incl = scan(n = cost(j0 + lane));
        }
        int at = __builtin_ctzll(__ballot(incl > (uint32_t)rest));
        rest -= __builtin_amdgcn_readlane((int)incl - n, at);
        r.seq.t0 = __builtin_amdgcn_readlane(x.t0, at);
        r.seq.n = __builtin_amdgcn_readlane(x.n, at);
        r.seq.L = __builtin_amdgcn_readlane(x.L, at);
        if (!by_seq) {
            j = j0 + at;
            r.s = j / a.groups;
            r.group = j - r.s * a.groups;
            r.u = rest;
            r.units = __builtin_amdgcn_readlane(n, at) - a.pad;
            return true;
        }
        r.s = j0 + at;
        for (int g0 = 0; g0 < a.groups; g0 += 64) {  // a lane per group
            const int u = g0 + lane < a.groups ? paged_units_of(a, r.seq, g0 + lane) : 0, c = u > 0 ? u + a.pad : 0;
            const int upto = (int)scan(c), all = __builtin_amdgcn_readlane(upto, 63);
            if (rest >= all) {
                rest -= all;
                continue;
            }
            at = __builtin_ctzll(__ballot(upto > rest));
            r.group = g0 + at;
            r.u = rest - __builtin_amdgcn_readlane(upto - c, at);
            r.units = __builtin_amdgcn_readlane(u, at);
            return true;
        }
        return false;
    }
    r.s = j / a.groups;
    r.group = j - r.s * a.groups;
    r.seq = paged_seq(a, r.s);
    r.units = paged_units_of(a, r.seq, r.group);
    r.left = r.units;
    return r.units > 0;
}

// The next part of the run; false at its end.  (All that leaves the loop is scalar
// and no store is by the lane: one inside the loop would make everything that
// leaves it a vector value.)
__device__ inline bool paged_next(const PagedArgs& a, PagedRun& r, PagedPart& p)
{
    const int pad = a.whole ? 0 : a.pad, sets = a.H_kv / a.heads;
    while (r.left > 0) {
        while (r.u >= r.units + pad || r.units == 0) {  // positions are left, so another pair follows
            r.u = 0;
            ++r.group;
            if (r.group >= a.groups || (r.units = paged_units_of(a, r.seq, r.group)) == 0) {
                // the next sequence's first group; behind one that has none, 64 sequences at a time
                r.group = 0;
                if (++r.s >= a.num_seqs) {
                    r.s = 0;
                    if (++r.head >= sets) return false;  // lengths that changed under the call
                }
                r.seq = paged_seq(a, r.s);
                r.units = paged_units_of(a, r.seq, 0);
                if (r.units == 0) {
                    const int k = r.s + paged_lane();
                    const uint64_t b = __ballot(k < a.num_seqs && paged_units_of(a, paged_seq(a, min(k, a.num_seqs - 1)), 0) > 0);
                    r.s += b ? __builtin_ctzll(b) - 1 : 63;  // the one before it
                }
            }
        }
        const int take = min(r.left, r.units + pad - r.u);
        p.u0 = max(r.u - pad, 0);
        p.u1 = max(r.u + take - pad, 0);
        p.head = r.head;
        p.s = r.s;
        p.group = r.group;
        p.seq = r.seq;
        p.whole = p.u0 == 0 && p.u1 == r.units;
        p.slot = 2 * r.w + (p.u0 == 0 ? 1 : 0);
        p.end = r.pos - r.u + r.units + pad;
        r.pos += take;
        r.left -= take;
        r.u += take;
        if (p.u1 > p.u0) return true;  // else of the pair's price only
    }
    return false;
}

// One lane of the work-group notes for the finish pass whether a pair that begins
// with this part is cut.
__device__ inline void paged_note(const PagedArgs& a, const PagedRun& r, const PagedPart& p)
{
    if (a.whole || p.u0 > 0) return;
    const int j = p.s * a.groups + p.group;
    const int at = p.end - 1, first = r.more * (r.per + 1);  // the work-group of the pair's last position
    const int last = min(at < first ? at / (r.per + 1) : r.more + (at - first) / r.per, a.workers - 1);
    const int4 cut = make_int4(p.whole ? -1 : r.w, last, j, p.head);
    if (a.by_pair) a.cut[p.head * a.num_seqs * a.groups + j] = cut;
    else if (!p.whole) a.cut[r.w] = cut;
}

// Number of a work-group: block b runs on XCD b % 8, and neighbours in the
// list, which read the same keys, share an XCD's cache.  (The number of blocks
// is an argument: the grid's size stands in the dispatch packet, in host memory,
// and 256 work-groups that read it start over 13 us.)
__device__ inline int paged_worker(const PagedArgs& a, int block) { return (block % 8) * (a.blocks / 8) + block / 8; }

// Row of q / out / lse of row r of a pair.
__device__ inline long paged_qrow(const PagedArgs& a, const PagedSeq& x, int head, int r)
{
    const int i = r / a.G;
    return (long)(x.t0 + i) * a.H_q + head * a.G + (r - i * a.G);
}

// Entry i (uniform) of a row of the block table, through the scalar cache.
__device__ inline int paged_entry(const int32_t* row, int i)
{
    typedef __attribute__((address_space(4))) const int32_t const_i32_t;
    return ((const_i32_t*)(uintptr_t)row)[i];
}

// Page of key t of a sequence, -1 if absent.
__device__ inline int paged_page(const PagedArgs& a, int s, int t)
{
    const int p = a.block_table[(long)s * a.max_pages + min(t >> a.page_shift, a.max_pages - 1)];
    return (uint32_t)p < (uint32_t)a.num_pages ? p : -1;
}

// 2^(byte - 127) of byte i of a word; 0 for a byte of 0
__device__ inline float paged_scale(uint32_t word, int i) { return __uint_as_float(((word >> (8 * i)) & 255u) << 23); }

void launch_paged_f32(const PagedArgs& a, int head_dim, bool fp8, hipStream_t stream);
void launch_paged_few(const PagedArgs& a, int head_dim, bool fp8, hipStream_t stream);
void launch_paged_rows(const PagedArgs& a, int head_dim, bool fp8, hipStream_t stream);
void launch_paged_finish(const PagedArgs& a, int head_dim, int dtype, hipStream_t stream);

}  // namespace pdec
