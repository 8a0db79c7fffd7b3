// Attention over paged caches, few query rows per kv head (single tokens,
// drafted tokens, short chunks), bfloat16, on v_mfma_f32_16x16x32_bf16.
//
// What bounds it: the bytes of the pages.  A key meets 16 NT rows at most, so
// nothing is shared between waves: each of a work-group's eight waves takes every
// eighth 32-key block of the part (of its head's waves' blocks) through a ring of
// its own in LDS (16 KB, filled by global_load_lds_dwordx4), with a softmax state
// of its own, and never waits for another wave until the states are joined at the
// part's end.  A block's 16-key halves are each on one page: a scalar base and
// fixed lane offsets per half, the pages of the block after the ring's read one
// block ahead.  A ring holds two blocks (four of 8-bit rows of 64), but one of
// bfloat16 rows of 128: there a wave asks for its next block behind this one's
// products and has nothing under way meanwhile, and only the other wave of its SIMD
// covers for it.  One token of each of 32 sequences over 8-bit pages (291 MB): 62 us,
// 4.7 TB/s with the finish pass; one over 32768 bfloat16 keys (67 MB) 20.4 us,
// 3.3 TB/s: two blocks to a wave, half of the wave cycles waiting, and the passes'
// starts and ends about 8.
//
// Up to 32 rows at D = 128 and 64 at D = 64: above, 64 rows' accumulators leave a
// SIMD one wave at D = 128, and the kernel for many rows, which shares its keys over
// its waves, is as fast or faster from there (13 sequences of 35 rows of 128 47.7
// against 39.9 us, of 56 rows 53.8 against 41.7; 64 rows of 64 48.4 against 51.7).
// Not over 8-bit pages where memory bounds the call: 32 sequences of 35 rows took
// 112 us in a form for 64 rows, and take 120 in the kernel for many rows.
//
// Per block, products and layouts as in the decode step (kernel_mfma.h):
//   S^T  = K  Q^T    A = 16 keys x 32 d from LDS, B = Q^T (registers)
//   O^T += V^T P^T   A = V^T by a transposing LDS read, B = P^T (registers)
// Rows are permuted 16 bytes at a time in LDS so that the reads of one phase
// meet different banks.
//
// HW kv heads to a work-group, its waves dealt to the heads in turn: two where a
// head's row is a cache line (128 bytes) or half of one, so that neighbouring rows
// are asked for at about the same time.  32 tokens over 8 heads of 64: 104 against
// 77 us over 8-bit pages (half a line, whose other half was fetched twice), 120
// against 108 over bfloat16; over 4 heads of 128 in 8 bits 65.3 against 62.8.
//
// 8-bit pages stay 8 bits in LDS, and their operands are widened in registers:
// each is used by one wave only, so once each.  A lane's 16 bytes of a key row
// are the operands of two steps (the contraction over d is taken in that order,
// Q's too); ds_read_b64_tr_b8 gives 8 keys of one d.  A key's power of two
// multiplies its scores, a value's its probability before that is rounded.
#pragma once

#include "kernel_paged_rows.h"

namespace pdec {

// 16-byte chunk permutations of the rows in LDS: chunk ch of key k sits at ch ^ swizzle(k).
template <int D, bool FP8>
__device__ inline int few_kswz(int key)
{
    if constexpr (FP8) return D == 128 ? (key & 7) : ((key >> 1) & 3);
    return key & (D / 8 - 1);
}
template <int D, bool FP8>
__device__ inline int few_vswz(int key)
{
    // 8-bit: a phase of the transposing read is keys 4 q .. + 3 and 16 + 4 q .. + 3
    if constexpr (FP8) return D == 128 ? ((key & 3) | ((key >> 2) & 4)) : (((key >> 1) & 1) | ((key >> 3) & 2));
    return (2 * key) & (D == 128 ? 14 : 6);
}

// Eight e4m3 values as bf16
__device__ inline u32x4_t widen8(uint32_t lo, uint32_t hi)
{
    u32x4_t r;
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true));
    return r;
}

// One wave-wide DMA of N KB, N instructions of 16 bytes per lane from one scalar base
// to consecutive places in LDS.  An instruction's immediate offset counts for its LDS
// address and for its memory address: off[i] has it taken out (i KB, which the i-th
// KB of a tensor is at least away from its first, a KB being whole rows).
template <int N>
__device__ inline void dma_rows(uint64_t base, const uint32_t (&off)[N], uint32_t lds_base, uint64_t lanes)
{
    const uint64_t sb = sgpr_base(reinterpret_cast<const void*>(base)), ln = sgpr_base(reinterpret_cast<const void*>(lanes));
    const uint32_t m = __builtin_amdgcn_readfirstlane(lds_base);
    if constexpr (N == 1)
        asm volatile("s_mov_b32 m0, %0\n\ts_mov_b64 exec, %1\n\ts_nop 2\n\tglobal_load_lds_dwordx4 %3, %2\n\ts_mov_b64 exec, -1" :
                     : "s"(m), "s"(ln), "s"(sb), "v"(off[0]) : "memory");
    else if constexpr (N == 2)
        asm volatile("s_mov_b32 m0, %0\n\ts_mov_b64 exec, %1\n\ts_nop 2\n\tglobal_load_lds_dwordx4 %3, %2\n\t"
                     "global_load_lds_dwordx4 %4, %2 offset:1024\n\ts_mov_b64 exec, -1" :
                     : "s"(m), "s"(ln), "s"(sb), "v"(off[0]), "v"(off[1]) : "memory");
    else {
        static_assert(N == 4, "instructions of a half");
        asm volatile("s_mov_b32 m0, %0\n\ts_mov_b64 exec, %1\n\ts_nop 2\n\tglobal_load_lds_dwordx4 %3, %2\n\t"
                     "global_load_lds_dwordx4 %4, %2 offset:1024\n\tglobal_load_lds_dwordx4 %5, %2 offset:2048\n\t"
                     "global_load_lds_dwordx4 %6, %2 offset:0xc00\n\ts_mov_b64 exec, -1" :
                     : "s"(m), "s"(ln), "s"(sb), "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]) : "memory");
    }
}

constexpr int kFewWaves = 8;  // of a work-group

template <int D, int NT, bool FP8, int HW>
__global__ __launch_bounds__(64 * kFewWaves) void paged_few_kernel(PagedArgs a)
{
    constexpr int NW = kFewWaves;
    constexpr int RT = 16 * NT;
    constexpr int NK = NW / HW;                  // waves that share a head's keys
    constexpr int RING = 131072 / NW;            // bytes of a wave's ring
    constexpr int ESZ = FP8 ? 1 : 2, ROWB = D * ESZ;
    constexpr int KB = 32;                       // keys per block
    constexpr int TENSOR = KB * ROWB, SLOT = 2 * TENSOR;
    constexpr int NS = RING / SLOT;              // ring slots of a wave
    constexpr int CPK = ROWB / 16;               // 16-byte chunks per key
    constexpr int KPI = 64 / CPK;                // keys per DMA instruction
    constexpr int PPH = 16 / KPI;                // instructions per half of a tensor
    constexpr int PB = 4 * PPH + (FP8 ? 1 : 0);  // and per block, its scales with them
    constexpr int KS = D / 32, DT = D / 16;
    constexpr int OROW = D + 4;                  // row pitch of the merge buffer, in floats
    static_assert((NS - 1) * PB < 64, "the wait counts them");
    static_assert(16 * OROW * 4 <= RING, "merge buffer");
    __shared__ __attribute__((aligned(1024))) unsigned char lds[NW * RING + (FP8 ? NW * NS * 64 : 0)];
    __shared__ float m_s[NW][16], l_s[NW][16];

    const int w = __builtin_amdgcn_readfirstlane(wi_id() >> 6);
    const int wk = w / HW, wh = w % HW;  // the wave's blocks, and its head of the pair's
    const int lane = paged_lane(), l16 = lane & 15, lg = lane >> 4;
    PagedRun run;
    PagedPart part;
    if (!paged_begin(a, paged_worker(a, wg_id()), run, wi_id() == 0)) return;

    const float c = a.qscale;
    const uint32_t strideB = (uint32_t)a.H_kv * ROWB, pageB = strideB << a.page_shift;  // bytes of a token, a page
    const uint32_t ring = lds_u32(lds) + w * RING, sc_ring = lds_u32(lds) + NW * RING + w * NS * 64;
    // byte offset of the lane's chunk in instruction i of half h of a tensor, less 1024 i (dma_rows)
    uint32_t koffs[2][PPH], voffs[2][PPH];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < PPH; ++i) {
            const int k = i * KPI + lane / CPK, key = 16 * h + k;
            koffs[h][i] = (uint32_t)k * strideB + 16 * ((lane % CPK) ^ few_kswz<D, FP8>(key)) - 1024 * i;
            voffs[h][i] = (uint32_t)k * strideB + 16 * ((lane % CPK) ^ few_vswz<D, FP8>(key)) - 1024 * i;
        }
    // operand reads, relative to a slot
    uint32_t kread[FP8 ? KS / 2 : KS], vread[DT];
#pragma unroll
    for (int t = 0; t < (FP8 ? KS / 2 : KS); ++t) kread[t] = l16 * ROWB + 16 * ((4 * t + lg) ^ few_kswz<D, FP8>(l16));
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
        if constexpr (FP8) {
            const int j = l16 >> 1, key = (j < 4 ? 0 : 12) + 4 * lg + j;
            vread[dt] = TENSOR + key * ROWB + 16 * (dt ^ few_vswz<D, FP8>(key)) + 8 * (l16 & 1);
        } else {
            const int key = 4 * lg + (l16 >> 2);
            vread[dt] = TENSOR + key * ROWB + 16 * ((2 * dt + ((l16 & 3) >> 1)) ^ few_vswz<D, FP8>(key)) + 8 * (l16 & 1);
        }
    }
    typedef __attribute__((address_space(3))) const u32x4_t lds_u32x4_t;
    typedef __attribute__((address_space(3))) const uint32_t lds_u32_t;
    const uint64_t sc_lane = FP8 ? reinterpret_cast<uint64_t>(lane & 8 ? a.v_scales : a.k_scales) + 4 * (lane & 3) : 0;

    while (paged_next(a, run, part)) {
        if (w == 0 && lane == 0) paged_note(a, run, part);
        const PagedSeq sq = part.seq;
        const int R = sq.n * a.G, row0 = part.group * RT, nrows = min(RT, R - row0);
        const int tiles = (nrows + 15) / 16;
        const int nb = 2 * (part.u1 - part.u0), mine = nb > wk ? (nb - wk + NK - 1) / NK : 0;  // blocks: of the part, of the wave
        const int t0 = part.u0 * kUnit;
        const int32_t* table = a.block_table + (long)part.s * a.max_pages;
        const int head = part.head * HW + wh;
        const uint64_t kbase = sgpr_base(a.k_pages) + (uint64_t)head * ROWB, vbase = sgpr_base(a.v_pages) + (uint64_t)head * ROWB;

        // the wave's block b: its first key, and its halves' pages
        auto first = [&](int b) __attribute__((always_inline)) { return t0 + KB * (wk + NK * b); };
        struct Pages { int half[2]; };
        auto pages = [&](int b) __attribute__((always_inline)) {
            Pages x;
#pragma unroll
            for (int h = 0; h < 2; ++h)
                x.half[h] = h > 0 && a.page_shift > 4 ? x.half[0] : paged_entry(table, min((first(b) + 16 * h) >> a.page_shift, a.max_pages - 1));
            return x;
        };
        auto there = [&](const Pages& x, int h) __attribute__((always_inline)) { return (uint32_t)x.half[h] < (uint32_t)a.num_pages; };
        // blocks past the last are pieces of one lane, so that every wait counts the same
        // (ring.h); an absent page is read as page 0, and its keys masked
        auto issue = [&](int b, const Pages& x) __attribute__((always_inline)) {
            const uint64_t lanes = b < mine ? ~0ull : 1ull;
            const uint32_t dst = ring + (b % NS) * SLOT;
            const int row = first(b) & ((1 << a.page_shift) - 1);  // of the first half
            uint64_t at[2], sc[2];
            const int page0 = there(x, 0) && b < mine ? x.half[0] : 0;
            at[0] = (uint64_t)(uint32_t)page0 * pageB + (uint32_t)row * strideB;
            if constexpr (FP8) sc[0] = (((uint64_t)(uint32_t)page0 * a.H_kv + head) << a.page_shift) + (uint32_t)row;
            if (a.page_shift > 4) {  // both halves on one page
                at[1] = at[0] + 16 * strideB;
                if constexpr (FP8) sc[1] = sc[0] + 16;
            } else {
                const int page1 = there(x, 1) && b < mine ? x.half[1] : 0;
                at[1] = (uint64_t)(uint32_t)page1 * pageB;
                if constexpr (FP8) sc[1] = ((uint64_t)(uint32_t)page1 * a.H_kv + head) << a.page_shift;
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                dma_rows(kbase + at[h], koffs[h], dst + 1024 * h * PPH, lanes);
                dma_rows(vbase + at[h], voffs[h], dst + TENSOR + 1024 * h * PPH, lanes);
            }
            if constexpr (FP8) {  // 16 bytes each of K's halves, then of V's, four lanes to a half
                const uint64_t from = (lane & 4 ? sc[1] : sc[0]) + sc_lane;
                dma_4B_lanes(from, sc_ring + (b % NS) * 64, lanes & 0xffffu);
            }
        };

        // ---- this lane's rows: 16 nt + l % 16; those past the last see nothing ----
        int seen[NT];
        u32x4_t qf[NT][KS];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int r = 16 * nt + l16, rr = row0 + min(r, nrows - 1);
            seen[nt] = r < nrows ? paged_seen(a, sq, rr / a.G) : 0;
            const uint16_t* q = static_cast<const uint16_t*>(a.q) + paged_qrow(a, sq, head, rr) * D;
#pragma unroll
            for (int t = 0; t < KS; ++t)
                qf[nt][t] = *reinterpret_cast<const u32x4_t*>(q + (FP8 ? 64 * (t / 2) + 16 * lg + 8 * (t & 1) : 32 * t + 8 * lg));
        }
        // keys that every row sees (rows past the last are masked or not, their results are not stored)
        const int least = __builtin_amdgcn_readfirstlane(paged_seen(a, sq, row0 / a.G));
        const int most = __builtin_amdgcn_readfirstlane(paged_seen(a, sq, (row0 + nrows - 1) / a.G));
#pragma unroll
        for (int b = 0; b < NS; ++b)
            if (mine > 0) issue(b, pages(min(b, mine - 1)));
        Pages ahead = pages(min(NS, max(mine - 1, 0)));
        Pages now = pages(0);

        f32x4_t o[NT][DT];
        float m_ref[NT], lsum[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            m_ref[nt] = kMinRef;
            lsum[nt] = 0.f;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) o[nt][dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        }
        // the query loads and the DMA complete in no order relative to each other
        wait_vmcnt<0>();

        for (int b = 0; b < mine; ++b) {
            wave_wait_vmcnt<(NS - 1) * PB>();  // block b has landed
            const uint32_t slot = ring + (b % NS) * SLOT;
            const int t = first(b);
            const bool there0 = there(now, 0), there1 = there(now, 1);
            if ((there0 | there1) && t < most) {
                u32x4_t kf[2][KS], vf[DT];
                uint32_t ks[2], vs[2];
#pragma unroll
                for (int kt = 0; kt < 2; ++kt) {
                    if constexpr (FP8) {
#pragma unroll
                        for (int u = 0; u < KS / 2; ++u) {
                            const u32x4_t x = *(lds_u32x4_t*)(uintptr_t)(slot + kread[u] + 16 * kt * ROWB);
                            kf[kt][2 * u] = widen8(x[0], x[1]);
                            kf[kt][2 * u + 1] = widen8(x[2], x[3]);
                        }
                        ks[kt] = *(lds_u32_t*)(uintptr_t)(sc_ring + (b % NS) * 64 + 16 * kt + 4 * lg);
                        vs[kt] = *(lds_u32_t*)(uintptr_t)(sc_ring + (b % NS) * 64 + 32 + 16 * kt + 4 * lg);
                    } else {
#pragma unroll
                        for (int s = 0; s < KS; ++s) kf[kt][s] = *(lds_u32x4_t*)(uintptr_t)(slot + kread[s] + 16 * kt * ROWB);
                    }
                }
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    if constexpr (FP8) {
                        typedef __attribute__((ext_vector_type(2))) int i32x2_t;
                        const i32x2_t x = __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) i32x2_t*)(uintptr_t)(slot + vread[dt]));
                        vf[dt] = widen8((uint32_t)x.x, (uint32_t)x.y);
                    } else {
                        typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;
                        const u32x2_t x0 = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(uintptr_t)(slot + vread[dt])));
                        const u32x2_t x1 = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t*)(uintptr_t)(slot + vread[dt] + 16 * ROWB)));
                        vf[dt] = u32x4_t{x0.x, x0.y, x1.x, x1.y};
                    }
                }
                const bool full = t + KB <= least && there0 && there1;
                // 0 times an infinite or NaN value is NaN: where a key is hidden from a row,
                // such values are left out of the products, then added key by key to the rows
                // that see the key
                bool apart = false;
                if (!full) {
                    typedef __attribute__((ext_vector_type(2))) uint16_t u16x2_t;
                    u16x2_t top = {0, 0};  // the largest magnitudes, as their bits
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2_t, vf[dt][e] & 0x7fff7fffu));
                    apart = __any(max(top.x, top.y) >= 0x7f80);
                }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    if (nt >= tiles) break;
                    f32x4_t s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
                    for (int i = 0; i < KS; ++i)
#pragma unroll
                        for (int kt = 0; kt < 2; ++kt) s[kt] = mfma_16x16x32(as_bf16x8(kf[kt][i]), as_bf16x8(qf[nt][i]), s[kt]);
                    float p[8], vp[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        p[i] = s[i >> 2][i & 3];
                        if constexpr (FP8) p[i] *= paged_scale(ks[i >> 2], i & 3);
                    }
                    if (!full) {
                        const int lim = seen[nt] - t - 4 * lg;
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            p[i] = ((16 * (i >> 2) + (i & 3) >= lim) | !(i < 4 ? there0 : there1)) ? kNegInf : p[i];
                    }
                    float mx = p[0];
#pragma unroll
                    for (int i = 1; i < 8; ++i) mx = paged_top(mx, p[i]);
                    if (__any(mx * c > m_ref[nt] + 8.f)) {  // rare after a row's first keys
                        const float mt = max_over_groups(mx) * c;
                        const bool up = mt > m_ref[nt] + 8.f;
                        const float alpha = up ? fast_exp2(m_ref[nt] - mt) : 1.f;
                        m_ref[nt] = up ? mt : m_ref[nt];
                        lsum[nt] *= alpha;
#pragma unroll
                        for (int dt = 0; dt < DT; ++dt) o[nt][dt] *= alpha;
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        p[i] = fast_exp2(fmaf(p[i], c, -m_ref[nt]));  // 0 for a hidden key
                        vp[i] = p[i];
                        // (a hidden key's scale may be anything, 0 times infinity among it)
                        if constexpr (FP8) vp[i] = full || p[i] > 0.f ? p[i] * paged_scale(vs[i >> 2], i & 3) : p[i];
                    }
                    // the row sums take P unrounded; the product's operands are bf16, so P is
                    // rounded by half a step (2^-8) of each term, as out is.  A value's power of
                    // two takes no bits
                    lsum[nt] += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
                    const bf16x8_t pf = as_bf16x8(u32x4_t{pack_bf16x2(vp[0], vp[1]), pack_bf16x2(vp[2], vp[3]),
                                                          pack_bf16x2(vp[4], vp[5]), pack_bf16x2(vp[6], vp[7])});
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) {
                        u32x4_t v = vf[dt];
                        if (apart) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) v[e] &= ~strange_bf16x2(v[e]);
                        }
                        o[nt][dt] = mfma_16x16x32(as_bf16x8(v), pf, o[nt][dt]);
                    }
                    if (!apart) continue;
#pragma unroll 1
                    for (int key = 0; key < KB; ++key) {
                        const int x = key & 15;
                        const bool sees = (t + key < seen[nt]) & (key < 16 ? there0 : there1);
                        const bool mine_k = lg == (x >> 2);
                        const int word = 2 * (key >> 4) + ((x & 3) >> 1);
                        const uint32_t half = (x & 1) ? 0xffff0000u : 0xffffu;
#pragma unroll
                        for (int dt = 0; dt < DT; ++dt) {
                            u32x4_t v = vf[dt];
                            asm volatile("" : "+v"(v));  // nothing of this rare loop before it
#pragma unroll
                            for (int e = 0; e < 4; ++e) v[e] &= strange_bf16x2(v[e]) & ((mine_k & (e == word)) ? half : 0u);
                            const f32x4_t y = mfma_16x16x32(as_bf16x8(v), pf, o[nt][dt]);
#pragma unroll
                            for (int i = 0; i < 4; ++i) o[nt][dt][i] = sees ? y[i] : o[nt][dt][i];
                        }
                    }
                }
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the slot has been read
            issue(b + NS, ahead);
            ahead = pages(min(b + NS + 1, mine - 1));
            now = pages(min(b + 1, mine - 1));
        }

        // ---- the waves' states joined, tile by tile; lane: row l % 16 of tile nt, d = 16 dt + 4 (l / 16) + i ----
        wait_vmcnt<0>();  // no DMA into the ring outlives the part
        float* const o_s = reinterpret_cast<float*>(lds);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            if (nt >= tiles) break;
            lds_barrier();  // the ring, or the tiles before, have been read
            float l = lsum[nt];
            l += __shfl_xor(l, 16);
            l += __shfl_xor(l, 32);
            if (lg == 0) {
                m_s[w][l16] = m_ref[nt];
                l_s[w][l16] = l;
            }
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
                *reinterpret_cast<f32x4_t*>(o_s + (w * 16 + l16) * OROW + 16 * dt + 4 * lg) = o[nt][dt];
            lds_barrier();
            const int rows = min(nrows - 16 * nt, 16);
            for (int i = 64 * w + lane; i < HW * rows * (D / 4); i += 64 * NW) {
                const int r = i / (D / 4) % rows, d4 = i % (D / 4), hs = i / (D / 4) / rows;
                float M = m_s[hs][r];
#pragma unroll
                for (int x = 1; x < NK; ++x) M = paged_top(M, m_s[HW * x + hs][r]);
                float L = 0.f;
                f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int x = 0; x < NK; ++x) {
                    const int y = HW * x + hs;
                    const float f = fast_exp2(m_s[y][r] - M);  // 0 for a wave that saw none of the row's keys
                    L += f * l_s[y][r];
                    acc += f * *reinterpret_cast<const f32x4_t*>(o_s + (y * 16 + r) * OROW + 4 * d4);
                }
                const int row = 16 * nt + r;
                if (!part.whole) {
                    const long at = ((long)part.slot * HW + hs) * RT + row;
                    *reinterpret_cast<f32x4_t*>(a.part_o + at * D + 4 * d4) = acc;
                    if (d4 == 0) *reinterpret_cast<float2*>(a.part_ml + 2 * at) = make_float2(M, L);
                    continue;
                }
                const long qr = paged_qrow(a, sq, part.head * HW + hs, row0 + row);
                const bool any = __float_as_uint(L) != 0;  // L is 0, positive or NaN
                const float inv = any ? 1.f / L : 0.f;
                acc *= inv;
                *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + qr * D + 4 * d4) =
                    make_uint2(pack_bf16x2(acc[0], acc[1]), pack_bf16x2(acc[2], acc[3]));
                if (d4 == 0 && a.lse) a.lse[qr] = any ? kLn2 * (M + __log2f(L)) : kNegInf;
            }
        }
        lds_barrier();  // the states have been read: the next part's DMA may come
    }
}

}  // namespace pdec
