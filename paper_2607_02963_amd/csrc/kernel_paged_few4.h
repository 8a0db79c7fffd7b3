// Attention over 4-bit paged caches, few query rows per kv head (bfloat16) or any (float32),
// on v_mfma_f32_16x16x32_bf16.
//
// The division of the work is that of the other caches' few-row kernel
// (kernel_paged_few.h): eight waves, each with a ring of its own in LDS, a softmax state
// of its own, joined at the part's end.  A wave's block is 64 keys, four quarters of 16,
// each on one page; a quarter of K or V is one DMA instruction (two are, at D = 64: an
// instruction takes the time of its lanes, used or not; drafted tokens, see below, took
// 25.7 us by quarters), the scales of a block's keys and values one more.
//
// Products and layouts, for 64 keys t + 16 q + j of quarters q:
//   S^T  = K  Q^T    four tiles of 16 keys; tile kt holds the keys 16 q + 4 kt + i, so
//                    that a lane's 16 scores are the keys of one quarter, in order
//   O^T += V^T P^T   two steps of 32 keys: ds_read_b64_tr_b4 gives a lane 16 keys of one
//                    d, the first eight for one step, the others for the second
// A lane's 16 bytes of a key row (8 at D = 64) have one scale, which the widening
// v_cvt_scalef32_pk_bf16_fp4 takes with it.  A lane's 16 values have a scale each, so
// that those multiply the probabilities, once for each block of 32 d, before they are
// rounded: a power of two takes no bits.  Where every row sees the block and all its scales
// are of 2^-63 .. 2^64, that is an addition to the exponents of two rounded probabilities at
// a time, of scales that the wave has spread in LDS as bfloat16 exponents.  A probability of
// 0 has no exponent: with the sign bit set in all others the addition is a subtraction of
// 2^15 less the exponent that stops at 0, which keeps it and clears the bit.
//
// float32 queries and probabilities are taken as the sums of three bfloat16 numbers, eight
// of their 24 bits each: exact, and 4-bit keys and values are exact in bfloat16, so that
// three products are the float32 product, at the rate of the bfloat16 ones (a third of
// 1200 TFLOP/s against 154 on the float32 matrix product): 512 tokens over 4000 keys,
// 28 heads of 128, took 389 us on the float32 product and take 124; 32 tokens of one sequence
// over 3000 keys 51 and 19.5, one of each of 32 sequences 27.3 (53 MB).
//
// What bounds it: the bytes and the parts' starts and ends.  One token of each of 32
// sequences of 1200 to 16384 keys, 28 heads of 128 over 4 (153.5 MB): 40 us as a call;
// the same with the DMA alone, without products and softmax, 35; each further byte moves at
// 5.7 TB/s, and about 14 us are fixed: the call's start, the parts' starts, the joins of
// eight waves' states and the finish pass.  2 to 9 drafted tokens of 13 sequences, 32
// heads of 64 over 8 (35 MB): 24 us, with the DMA alone 19.  The multiplying path alone took
// 46.3 and 37.5 before exponents were added, parts priced and units weighed by their tiles.
//
// Up to three tiles of 16 rows at D = 128, four at D = 64 (one and two in float32): one more
// and the state leaves the registers.  So many are worked on one (D = 128) or two (D = 64)
// after the other, keys and values widened anew, with the queries in LDS: 5 tokens of 32
// sequences, 35 rows of 128, 72 us (all tiles at once, spilling, 133; the kernel for many
// rows 109), 13 of 20 sequences, 52 rows of 64, 48 (60; 66).  With four tiles at D = 128, 64
// rows of 16 sequences took 32.6 us, of the kernel for many rows 26.6.  bfloat16 batches of
// more rows take that, float32 ones more items of these.
#pragma once

#include "kernel_paged_few.h"
#include "paged_e2m1.h"

namespace pdec {

// 16-byte chunk permutations of the rows in LDS: chunk ch of key k sits at ch ^ swizzle(k).
template <int D>
__device__ inline int few4_kswz(int key) { return D == 128 ? ((key >> 4) & 3) : ((key >> 4) & 1); }
template <int D>
__device__ inline int few4_vswz(int key) { return D == 128 ? ((key >> 2) & 3) : ((key >> 3) & 1); }

// One wave-wide DMA of 16 bytes per lane from the lanes' own addresses.
__device__ inline void dma_16B_lanes(uint64_t addr, uint32_t lds_base, uint64_t lanes)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_mov_b64 exec, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off\n\ts_mov_b64 exec, -1" :
                 : "s"(__builtin_amdgcn_readfirstlane(lds_base)), "v"(addr), "s"(sgpr_base(reinterpret_cast<const void*>(lanes)))
                 : "memory");
}

// x y, 0 if one is 0, whatever the other (v_mul_legacy_f32, which has no builtin; as
// inline assembly the compiler would not keep it apart from a v_exp_f32 before it).
__device__ float mul_zero(float x, float y) __asm("llvm.amdgcn.fmul.legacy");

// Two numbers of 15 bits, with bit 15 set in each that is not 0 (which the compiler would do
// by comparisons, one by one).
__device__ inline uint32_t mark_not_0(uint32_t x)
{
    uint32_t some, y;
    asm("v_pk_min_u16 %0, %1, %2" : "=v"(some) : "v"(x), "s"(0x00010001u));
    asm("v_pk_mad_u16 %0, %1, %2, %3" : "=v"(y) : "v"(some), "s"(0x80008000u), "v"(x));
    return y;
}

// x as the sum of three bfloat16 numbers of its sign, the first 16 bits of x and of what
// each leaves; two at a time.
__device__ inline void three_bf16(float x0, float x1, uint32_t (&y)[3])
{
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        const uint32_t u0 = __float_as_uint(x0), u1 = __float_as_uint(x1);
        y[i] = (u0 >> 16) | (u1 & 0xffff0000u);
        x0 -= __uint_as_float(u0 & 0xffff0000u);
        x1 -= __uint_as_float(u1 & 0xffff0000u);
    }
}

// BIG: pages of 64 keys or more, a block to a page.  T: an element of q and out.
template <int D, int NT, bool BIG, typename T>
__global__ __launch_bounds__(64 * kFewWaves) void paged_few4_kernel(PagedArgs a)
{
    constexpr int NW = kFewWaves;
    constexpr int RT = 16 * NT;
    constexpr int RING = 131072 / NW;            // bytes of a wave's ring
    constexpr int ROWB = D / 2;
    constexpr int KB = kUnit;                    // keys per block
    constexpr int TENSOR = KB * ROWB, SLOT = 2 * TENSOR;
    constexpr int NS = RING / SLOT;              // ring slots of a wave
    constexpr int CPK = ROWB / 16;               // 16-byte chunks per key
    constexpr int QB = 16 * ROWB;                // bytes of a quarter
    constexpr bool TWO = !BIG && QB < 1024;      // a DMA instruction takes two quarters, half of the lanes each
    constexpr int SPK = D / kE2m1Block;          // scales per key
    constexpr int SC = 2 * KB * SPK;             // bytes of a block's scales
    constexpr int PT = TENSOR / 1024;            // DMA instructions of K or V per block
    constexpr int PB = 2 * PT + 1;               // and of a block, its scales with them
    constexpr int KS = D / 32, DT = D / 16;
    constexpr int TERMS = sizeof(T) == 4 ? 3 : 1;  // bfloat16 numbers to a query element or probability
    constexpr int OROW = D + 4;                  // row pitch of the merge buffer, in floats
    constexpr uint64_t SLANES = (1ull << (SC / 16)) - 1;
    static_assert(KB == 64 && QB <= 1024 && (NS - 1) * PB < 64, "a block's instructions, and the wait that counts them");
    static_assert(16 * OROW * 4 <= RING, "merge buffer");
    constexpr int EXPS = 2 * KB * SPK;           // bytes of a wave's exponents: SPK times KB keys
    // the queries' operands in LDS, a KB for each tile's step of 32 d, read once a block, where the
    // registers do not hold them beside the state
    constexpr bool QLDS = TERMS == 1 && NT * D >= 256;
    constexpr int TURN_T = D == 128 && NT > 2 ? 1 : D == 64 && NT > 3 ? 2 : NT;  // tiles at a time
    constexpr int QS = QLDS ? NT * KS * 1024 : 0;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[NW * RING + NW * NS * SC + NW * EXPS + QS];
    __shared__ float m_s[NW][16], l_s[NW][16];

    const int w = __builtin_amdgcn_readfirstlane(wi_id() >> 6);
    const int lane = paged_lane(), l16 = lane & 15, lg = lane >> 4;
    PagedRun run;
    PagedPart part;
    constexpr bool WEIGHED = NT > 1;  // the pairs' blocks differ in price
    if (!paged_begin<WEIGHED>(a, paged_worker(a, wg_id()), run, wi_id() == 0)) return;

    const float c = a.qscale;
    const uint32_t ring = lds_u32(lds) + w * RING, sc_ring = lds_u32(lds) + NW * RING + w * NS * SC;
    const uint32_t exps = lds_u32(lds) + NW * RING + NW * NS * SC + w * EXPS;
    // byte offset of the lane's chunk in instruction i (of a quarter, or 1 KB: dma_rows): of V the
    // same for all, of K with the bits flipped that the quarter's number permutes
    constexpr int KPI = TWO ? 16 : 1024 / ROWB;  // keys of an instruction, on one page
    const int ikey = lane / CPK % KPI, lkey = lane / CPK;
    const uint32_t koff = (uint32_t)ikey * ROWB + 16 * ((lane % CPK) ^ few4_kswz<D>(lkey));
    const uint32_t voff = (uint32_t)ikey * ROWB + 16 * ((lane % CPK) ^ few4_vswz<D>(ikey & 15));
    // operand reads, relative to a slot: key 16 (l16 / 4) + l16 % 4 + 4 kt of K, the lane's elements;
    // key 16 lg + l16 of V, eight bytes of tile dt (of which dt / 2 flips bits of the address that
    // nothing else sets)
    uint32_t kread;
    const int kkey = 16 * (l16 >> 2) + (l16 & 3), vkey = 16 * lg + l16;
    if constexpr (D == 128) kread = kkey * ROWB + 16 * (lg ^ few4_kswz<D>(kkey));
    else kread = kkey * ROWB + 16 * ((lg >> 1) ^ few4_kswz<D>(kkey)) + 8 * (lg & 1);
    const uint32_t vread = TENSOR + vkey * ROWB + 16 * few4_vswz<D>(l16);
    const uint32_t ksread = kkey * SPK + (D == 128 ? lg : lg >> 1), vsread = KB * SPK + 16 * lg * SPK;
    const uint32_t qs = lds_u32(lds) + NW * RING + NW * NS * SC + NW * EXPS;
    typedef __attribute__((address_space(3))) const u32x4_t lds_u32x4_t;
    typedef __attribute__((address_space(3))) u32x4_t lds_u32x4w_t;
    typedef __attribute__((address_space(3))) const u32x2_t lds_u32x2_t;
    typedef __attribute__((address_space(3))) const uint8_t lds_u8_t;
    typedef __attribute__((ext_vector_type(2))) int i32x2_t;
    typedef __attribute__((address_space(3))) i32x2_t lds_i32x2_t;
    // the scales: lanes 0 .. 4 SPK - 1 K's, SPK to a quarter, then V's
    const int sq_lane = lane / SPK & 3;
    const uint64_t sc_lane = reinterpret_cast<uint64_t>(lane & (4 * SPK) ? a.v_scales : a.k_scales) + 16 * (lane % SPK);

    while (paged_next<WEIGHED>(a, run, part)) {
        if (w == 0 && lane == 0) paged_note(a, run, part);
        const PagedSeq sq = part.seq;
        const int R = sq.n * a.G, row0 = part.group * RT, nrows = min(RT, R - row0);
        const int tiles = (nrows + 15) / 16;
        const int nb = part.u1 - part.u0, mine = nb > w ? (nb - w + NW - 1) / NW : 0;  // blocks: of the part, of the wave
        const int t0 = part.u0 * kUnit;
        const int32_t* table = a.block_table + (long)part.s * a.max_pages;
        const int head = part.head;
        const uint64_t kbase = sgpr_base(a.k_pages), vbase = sgpr_base(a.v_pages);

        // The wave's block b: its first key; and its quarters' rows of the pool, looked up 64 quarters
        // (BIG: blocks) at a time, a lane to each, and read back from the lanes: scalar loads in the
        // loop would be waited for with every read of the LDS.  An absent page is read as page 0, and
        // its keys masked.
        auto first = [&](int b) __attribute__((always_inline)) { return t0 + KB * (w + NW * b); };
        constexpr int Q = BIG ? 1 : 4, TURN = 64 / Q;  // look-ups of a block; blocks of a look-up
        uint32_t row_lo = 0, row_hi = 0;
        uint64_t there = 0, last_there = 0;  // of the turn at hand, and of the one before
        auto look_up = [&](int b0) __attribute__((always_inline)) {
            const int t = first(min(b0 + lane / Q, mine - 1)) + 16 * (lane % Q);
            const int page = table[min(t >> a.page_shift, a.max_pages - 1)];
            const bool ok = (uint32_t)page < (uint32_t)a.num_pages;
            const uint64_t row = (((uint64_t)(uint32_t)(ok ? page : 0) * a.H_kv + head) << a.page_shift) + (uint32_t)(t & ((1 << a.page_shift) - 1));
            last_there = there;
            row_lo = (uint32_t)row;
            row_hi = (uint32_t)(row >> 32);
            there = __ballot(ok);
        };
        // blocks past the last are pieces of one lane, so that every wait counts the same (ring.h)
        auto issue = [&](int b) __attribute__((always_inline)) {
            const uint64_t real = b < mine ? ~0ull : 1ull;
            const uint32_t dst = ring + (b % NS) * SLOT;
            uint32_t ko = koff;
            asm volatile("" : "+v"(ko));  // one register, not one for every instruction
            uint32_t koffs[PT], voffs[PT];
#pragma unroll
            for (int i = 0; i < PT; ++i) {
                koffs[i] = ko ^ (16 * few4_kswz<D>(1024 / ROWB * i));
                voffs[i] = voff;
            }
            const int at = min(b, mine - 1) % TURN * Q;
            auto row_of = [&](int q) {
                return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)row_hi, at + q) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)row_lo, at + q);
            };
            if constexpr (BIG) {
                const uint64_t row = row_of(0);
                dma_rows(kbase + row * ROWB, koffs, dst, real);
                dma_rows(vbase + row * ROWB, voffs, dst + TENSOR, real);
                dma_16B_lanes(sc_lane + (row + 16 * sq_lane) * SPK, sc_ring + (b % NS) * SC, real & SLANES);
            } else {
                uint64_t row[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) row[q] = row_of(q);
#pragma unroll
                for (int i = 0; i < PT; ++i) {
                    if constexpr (TWO) {
                        const uint64_t at2 = (lane < 32 ? row[2 * i] : row[2 * i + 1]) * ROWB;
                        dma_16B_lanes(kbase + at2 + koffs[i], dst + 1024 * i, real);
                        dma_16B_lanes(vbase + at2 + voffs[i], dst + TENSOR + 1024 * i, real);
                    } else {
                        const uint32_t off[2][1] = {{koffs[i]}, {voffs[i]}};
                        dma_rows(kbase + row[i] * ROWB, off[0], dst + 1024 * i, real);
                        dma_rows(vbase + row[i] * ROWB, off[1], dst + TENSOR + 1024 * i, real);
                    }
                }
                const uint64_t lo = sq_lane & 1 ? row[1] : row[0], hi = sq_lane & 1 ? row[3] : row[2];
                dma_16B_lanes(sc_lane + (sq_lane & 2 ? hi : lo) * SPK, sc_ring + (b % NS) * SC, real & SLANES);
            }
        };

        // ---- this lane's rows: 16 nt + l % 16; those past the last see nothing ----
        int seen[NT];
        u32x4_t qf[QLDS ? 1 : NT][KS][TERMS];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int r = 16 * nt + l16, rr = row0 + min(r, nrows - 1);
            seen[nt] = r < nrows ? paged_seen(a, sq, rr / a.G) : 0;
            const T* q = static_cast<const T*>(a.q) + paged_qrow(a, sq, head, rr) * D + 8 * KS * lg;
            if constexpr (QLDS) {  // a step to a wave
                static_assert(NW % KS == 0, "a wave's steps are of one place in the rows");
                if (nt % (NW / KS) == w / KS) *(lds_u32x4w_t*)(uintptr_t)(qs + 1024 * (nt * KS + w % KS) + 16 * lane) = *reinterpret_cast<const u32x4_t*>(q + 8 * (w % KS));
                continue;
            }
#pragma unroll
            for (int i = 0; i < KS; ++i) {
                const u32x4_t x = *reinterpret_cast<const u32x4_t*>(q + 8 * i);
                if constexpr (TERMS == 1) qf[nt][i][0] = x;
                else {
                    const u32x4_t y = *reinterpret_cast<const u32x4_t*>(q + 8 * i + 4);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t z[3];
                        if (j < 2) three_bf16(__uint_as_float(x[2 * j]), __uint_as_float(x[2 * j + 1]), z);
                        else three_bf16(__uint_as_float(y[2 * j - 4]), __uint_as_float(y[2 * j - 3]), z);
#pragma unroll
                        for (int e = 0; e < TERMS; ++e) qf[nt][i][e][j] = z[e];
                    }
                }
            }
        }
        // keys that every row sees (rows past the last are masked or not, their results are not stored)
        const int least = __builtin_amdgcn_readfirstlane(paged_seen(a, sq, row0 / a.G));
        const int most = __builtin_amdgcn_readfirstlane(paged_seen(a, sq, (row0 + nrows - 1) / a.G));
        if (mine > 0) look_up(0);
        // the query loads and the DMA complete in no order relative to each other: those first, so that the
        // first block is waited for alone; the compiler sees a use of them here, or it might wait for them,
        // and so for all of the DMA, in the loop (2 to 8 tokens of 32 sequences, heads of 64, 50.5 and 54 us)
        wait_vmcnt<0>();
        if constexpr (!QLDS) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < KS; ++i)
#pragma unroll
                    for (int e = 0; e < TERMS; ++e) asm volatile("" : "+v"(qf[nt][i][e]));
        }
        if (mine > 0) {
#pragma unroll
            for (int b = 0; b < NS; ++b) issue(b);
        }

        f32x4_t o[NT][DT];
        float m_ref[NT], lsum[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            m_ref[nt] = kMinRef;
            lsum[nt] = 0.f;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) o[nt][dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        }
        if constexpr (QLDS) lds_barrier();  // all steps are there
        for (int b = 0; b < mine; ++b) {
            wave_wait_vmcnt<(NS - 1) * PB>();  // block b has landed
            const uint32_t slot = ring + (b % NS) * SLOT, scs = sc_ring + (b % NS) * SC;
            const int t = first(b);
            // the look-up may be a turn ahead of the block at hand
            const bool behind = b / TURN < (min(b + NS - 1, mine - 1)) / TURN;
            const uint32_t have = (uint32_t)((behind ? last_there : there) >> (b % TURN * Q)) & ((1u << Q) - 1);  // its quarters'
            if (have && t < most) {
                const bool full = t + KB <= least && have == (1u << Q) - 1;
                const bool mine_there = BIG || (have >> lg & 1);
                // the values' scales of key t + lane, spread by blocks of d: 2^15 less k where bfloat16 has its exponent
                bool odd;  // one of them is beyond 2^-63 .. 2^64: its byte's first two bits are alike
                constexpr uint32_t FIRST = SPK == 4 ? 0x80808080u : 0x8080u;  // bytes' first bits
                auto value_scales = [&](uint32_t base) __attribute__((always_inline)) -> uint32_t {  // of key t + lane
                    typedef __attribute__((address_space(3))) const uint16_t lds_u16c_t;
                    typedef __attribute__((address_space(3))) const uint32_t lds_u32c_t;
                    if constexpr (SPK == 4) return *(lds_u32c_t*)(uintptr_t)(base + KB * SPK + SPK * lane);
                    else return *(lds_u16c_t*)(uintptr_t)(base + KB * SPK + SPK * lane);
                };
                {
                    typedef __attribute__((address_space(3))) uint16_t lds_u16_t;
                    const uint32_t x = value_scales(scs);
                    odd = __any(((x ^ (x << 1)) & FIRST) != FIRST);
#pragma unroll
                    for (int i = 0; i < SPK; ++i) *(lds_u16_t*)(uintptr_t)(exps + 2 * KB * i + 2 * lane) = (uint16_t)(0x8000u + (127 << 7) - ((x >> (8 * i) & 255u) << 7));
                }
                // the tiles that have rows; a row past the last sees nothing, or its result is not stored
                auto block = [&](auto count, auto from) __attribute__((always_inline)) {
                    constexpr int N = count, F = from;  // tiles F .. F + N - 1
                    // registers: one tile's operands at a time (and where they are there, not: drafted tokens, heads
                    // of 64, 25.0 and 24.3 us, 1 to 8 of 32 sequences 54.9 and 53.3, 9 to 12 of 20 38.4 and 37.7)
                    constexpr bool TIGHT = N > 1 && (D == 128 || TERMS > 1);
                    i32x2_t vraw[DT];
                    uint32_t vat = slot + vread, eat = exps + 32 * lg;
                    asm volatile("" : "+v"(vat), "+v"(eat));  // one register each, not one for every read
                    auto read_v = [&](int dt) __attribute__((always_inline)) {
                        return __builtin_amdgcn_ds_read_tr4_b64_v2i32((lds_i32x2_t*)(uintptr_t)((vat ^ (16 * (dt >> 1))) + 8 * (dt & 1)));
                    };
                    float p[N][16];  // scores, then probabilities, of keys t + 16 lg + j
                    {
                        f32x4_t s[N][4];
                        if constexpr (QLDS) {
                            uint32_t x[4][KS];
                            float ks[4];
#pragma unroll
                            for (int kt = 0; kt < 4; ++kt) {
                                ks[kt] = e2m1_scale(*(lds_u8_t*)(uintptr_t)(scs + ksread + 4 * kt * SPK));
                                if constexpr (D == 128) {
                                    const u32x4_t y = *(lds_u32x4_t*)(uintptr_t)(slot + kread + 4 * kt * ROWB);
#pragma unroll
                                    for (int i = 0; i < KS; ++i) x[kt][i] = y[i];
                                } else {
                                    const u32x2_t y = *(lds_u32x2_t*)(uintptr_t)(slot + kread + 4 * kt * ROWB);
#pragma unroll
                                    for (int i = 0; i < KS; ++i) x[kt][i] = y[i];
                                }
#pragma unroll
                                for (int nt = 0; nt < N; ++nt) s[nt][kt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
                            }
#pragma unroll
                            for (int i = 0; i < KS; ++i) {
                                if (TIGHT) __builtin_amdgcn_sched_barrier(0);
                                u32x4_t qv[N];
#pragma unroll
                                for (int nt = 0; nt < N; ++nt) qv[nt] = *(lds_u32x4_t*)(uintptr_t)(qs + 1024 * ((F + nt) * KS + i) + 16 * lane);
#pragma unroll
                                for (int kt = 0; kt < 4; ++kt) {
                                    const bf16x8_t kf = as_bf16x8(e2m1_bf16(x[kt][i], ks[kt]));
#pragma unroll
                                    for (int nt = 0; nt < N; ++nt) s[nt][kt] = mfma_16x16x32(kf, as_bf16x8(qv[nt]), s[nt][kt]);
                                }
                            }
                        } else
#pragma unroll
                        for (int kt = 0; kt < 4; ++kt) {
                            if (TIGHT) __builtin_amdgcn_sched_barrier(0);
                            const float ks = e2m1_scale(*(lds_u8_t*)(uintptr_t)(scs + ksread + 4 * kt * SPK));
                            uint32_t x[KS];
                            if constexpr (D == 128) {
                                const u32x4_t y = *(lds_u32x4_t*)(uintptr_t)(slot + kread + 4 * kt * ROWB);
#pragma unroll
                                for (int i = 0; i < KS; ++i) x[i] = y[i];
                            } else {
                                const u32x2_t y = *(lds_u32x2_t*)(uintptr_t)(slot + kread + 4 * kt * ROWB);
#pragma unroll
                                for (int i = 0; i < KS; ++i) x[i] = y[i];
                            }
#pragma unroll
                            for (int nt = 0; nt < N; ++nt) s[nt][kt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                            for (int i = 0; i < KS; ++i) {
                                const bf16x8_t kf = as_bf16x8(e2m1_bf16(x[i], ks));
#pragma unroll
                                for (int nt = 0; nt < N; ++nt)
#pragma unroll
                                    for (int e = TERMS - 1; e >= 0; --e) s[nt][kt] = mfma_16x16x32(kf, as_bf16x8(qf[F + nt][i][e]), s[nt][kt]);
                            }
                        }
#pragma unroll
                        for (int nt = 0; nt < N; ++nt)
#pragma unroll
                            for (int j = 0; j < 16; ++j) p[nt][j] = s[nt][j >> 2][j & 3];
                    }
                    // the values, asked for under the softmax
                    if (!TIGHT) {
#pragma unroll
                        for (int dt = 0; dt < DT; ++dt) vraw[dt] = read_v(dt);
                    }
#pragma unroll
                    for (int nt = 0; nt < N; ++nt) {
                        if (!full) {
                            int lim = mine_there ? seen[F + nt] - t - 16 * lg : 0;
                            asm volatile("" : "+v"(lim));  // stays a branch
#pragma unroll
                            for (int j = 0; j < 16; ++j) p[nt][j] = j >= lim ? kNegInf : p[nt][j];
                        }
                        float mx = p[nt][0];
#pragma unroll
                        for (int j = 1; j < 16; ++j) mx = paged_top(mx, p[nt][j]);
                        if (__any(mx * c > m_ref[F + nt] + 8.f)) {  // rare after a row's first keys
                            const float mt = max_over_groups(mx) * c;
                            const bool up = mt > m_ref[F + nt] + 8.f;
                            const float alpha = up ? fast_exp2(m_ref[F + nt] - mt) : 1.f;
                            m_ref[F + nt] = up ? mt : m_ref[F + nt];
                            lsum[F + nt] *= alpha;
#pragma unroll
                            for (int dt = 0; dt < DT; ++dt) o[F + nt][dt] *= alpha;
                        }
                        float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            p[nt][j] = fast_exp2(fmaf(p[nt][j], c, -m_ref[F + nt]));  // 0 for a hidden key
                            sum[j & 3] += p[nt][j];
                        }
                        // the row sums take P unrounded; the product's operands are bf16, so with bf16
                        // queries P is rounded by half a step (2^-8) of each term, as out is
                        lsum[F + nt] += (sum[0] + sum[1]) + (sum[2] + sum[3]);
                    }
                    // O += V P of keys 16 lg + 8 h .. + 7, blk's 32 elements
                    auto products = [&](int blk, int h, const u32x4_t (&pf)[N][TERMS], float scale, auto fast) __attribute__((always_inline)) {
#pragma unroll
                        for (int dt = 2 * blk; dt < 2 * blk + 2; ++dt) {
                            if (TIGHT) vraw[dt] = read_v(dt);
                            uint32_t x = (uint32_t)(h ? vraw[dt].y : vraw[dt].x);
                            if (!fast) asm volatile("" : "+v"(x));  // else both paths' widening comes before the branch
                            const bf16x8_t vf = as_bf16x8(e2m1_bf16(x, scale));
#pragma unroll
                            for (int nt = 0; nt < N; ++nt)
#pragma unroll
                                for (int e = TERMS - 1; e >= 0; --e) o[F + nt][dt] = mfma_16x16x32(vf, as_bf16x8(pf[nt][e]), o[F + nt][dt]);
                        }
                    };
                    if (full && !odd) {
                        // P times 2^k: k added to its exponent, of what is not 0.  A product below 2^-126 comes out
                        // smaller, or 0; a float32 P's term below 2^-126 larger, by 2^-127 of a P at most
                        typedef __attribute__((ext_vector_type(2))) uint16_t u16x2_t;
                        u16x2_t pe[N][8][TERMS];
#pragma unroll
                        for (int nt = 0; nt < N; ++nt)
#pragma unroll
                            for (int j = 0; j < 8; ++j) {
                                uint32_t y[3];
                                if constexpr (TERMS == 1) y[0] = pack_bf16x2(p[nt][2 * j], p[nt][2 * j + 1]);
                                else three_bf16(p[nt][2 * j], p[nt][2 * j + 1], y);
#pragma unroll
                                for (int e = 0; e < TERMS; ++e) pe[nt][j][e] = __builtin_bit_cast(u16x2_t, mark_not_0(y[e]));
                            }
#pragma unroll
                        for (int blk = 0; blk < SPK; ++blk)
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                if (TIGHT) __builtin_amdgcn_sched_barrier(0);
                                const u32x4_t e = *(lds_u32x4_t*)(uintptr_t)(eat + 2 * KB * blk + 16 * h);
                                u32x4_t pf[N][TERMS];
#pragma unroll
                                for (int j = 0; j < 4; ++j) {
                                    const uint32_t ej = e[j];
#pragma unroll
                                    for (int nt = 0; nt < N; ++nt)
#pragma unroll
                                        for (int i = 0; i < TERMS; ++i) {
                                            pf[nt][i][j] = __builtin_bit_cast(uint32_t, __builtin_elementwise_sub_sat(pe[nt][4 * h + j][i], __builtin_bit_cast(u16x2_t, ej)));
                                        }
                                }
                                products(blk, h, pf, 1.f, std::true_type{});
                            }
                    } else {
                        // P times the scale, of a hidden value 0 whatever its scale.  P is 2^8 at most, and a scale 2^-127 ..
                        // 2^127: a product of 2^128 and up, whose value is 0 or its sum beyond float32's range, becomes the
                        // largest number; and where the row sees a scale below 2^-95 and none beyond 2^32, P is multiplied
                        // by 2^64 more, and the values are widened times 2^-64.  What sees a NaN value is NaN, whatever its P
                        uint32_t again = scs;
                        asm volatile("" : "+v"(again));  // else the word read above is kept
                        const uint32_t x = mine_there && t + lane < most ? value_scales(again) : 0x7f7f7f7fu;  // of what a row sees
                        const bool tiny = __any((~(x | x << 1 | x << 2) & FIRST) != 0) && !__any((x & (x << 1 | x << 2) & FIRST) != 0);
                        const float up = tiny ? 0x1p-64f : 1.f;
                        const uint32_t shift = tiny ? 64u << 23 : 0;
                        auto scaled = [&](float prob, uint32_t word, int i) __attribute__((always_inline)) {
                            const float y = mul_zero(prob, __uint_as_float(__float_as_uint(paged_scale(word, i)) + shift));
                            return fminf(y, TERMS == 1 ? 0x1.fep127f : 0x1.fffffep127f);
                        };
                        if (__any((x & x << 1 & x << 2 & x << 3 & FIRST) != 0)) {  // 240 and up
#pragma unroll
                            for (int blk = 0; blk < SPK; ++blk) {
                                const uint64_t nan = __ballot((x >> (8 * blk) & 255u) == 255u);  // key t + lane
                                if (nan == 0) continue;
#pragma unroll
                                for (int nt = 0; nt < N; ++nt) {
                                    const int n = min(max(seen[F + nt] - t, 0), 64);
                                    if (n > 0 && (nan << (64 - n)) != 0) o[F + nt][2 * blk] = o[F + nt][2 * blk + 1] = f32x4_t(__builtin_nanf(""));
                                }
                            }
                        }
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            uint32_t vs[2 * SPK];  // the scales of the lane's values 8 h .. 8 h + 7
#pragma unroll
                            for (int i = 0; i < SPK / 2; ++i) {
                                const u32x4_t x = *(lds_u32x4_t*)(uintptr_t)(scs + vsread + 8 * SPK * h + 16 * i);
#pragma unroll
                                for (int e = 0; e < 4; ++e) vs[4 * i + e] = x[e];
                            }
#pragma unroll
                            for (int blk = 0; blk < SPK; ++blk) {
                                if (TIGHT) __builtin_amdgcn_sched_barrier(0);
                                u32x4_t pf[N][TERMS];
#pragma unroll
                                for (int j = 0; j < 8; j += 2) {
#pragma unroll
                                    for (int nt = 0; nt < N; ++nt) {
                                        const float x0 = scaled(p[nt][8 * h + j], SPK == 4 ? vs[j] : vs[j / 2], blk);
                                        const float x1 = scaled(p[nt][8 * h + j + 1], SPK == 4 ? vs[j + 1] : vs[j / 2], SPK == 4 ? blk : 2 + blk);
                                        if constexpr (TERMS == 1) pf[nt][0][j >> 1] = pack_bf16x2(x0, x1);
                                        else {
                                            uint32_t y[3];
                                            three_bf16(x0, x1, y);
#pragma unroll
                                            for (int e = 0; e < TERMS; ++e) pf[nt][e][j >> 1] = y[e];
                                        }
                                    }
                                }
                                products(blk, h, pf, up, std::false_type{});
                            }
                        }
                    }
                };
                typedef std::integral_constant<int, 0> first_t;
                if constexpr (TURN_T < NT) {  // some tiles after the others, which widen the keys and values again
                    typedef std::integral_constant<int, TURN_T> turn_t;
                    block(turn_t{}, first_t{});
                    if (tiles > TURN_T) block(turn_t{}, turn_t{});
                    if constexpr (2 * TURN_T < NT)
                        if (tiles > 2 * TURN_T) block(turn_t{}, std::integral_constant<int, 2 * TURN_T>{});
                } else if (NT > 2 && tiles > 2) block(std::integral_constant<int, NT>{}, first_t{});
                else if (NT > 1 && tiles > 1) block(std::integral_constant<int, NT < 2 ? NT : 2>{}, first_t{});
                else block(std::integral_constant<int, 1>{}, first_t{});
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the slot has been read
            if ((b + NS) % TURN == 0 && b + NS < mine) look_up(b + NS);
            issue(b + NS);
        }

        // ---- the waves' states joined, tile by tile; lane: row l % 16 of tile nt, d = 16 dt + 4 (l / 16) + i ----
        wait_vmcnt<0>();  // no DMA into the ring outlives the part
        float* const o_s = reinterpret_cast<float*>(lds);
        constexpr int OW = 16 * OROW;  // a wave's rows, in floats
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
            for (int dt = 0; dt < DT; ++dt) *reinterpret_cast<f32x4_t*>(o_s + w * OW + l16 * OROW + 16 * dt + 4 * lg) = o[nt][dt];
            lds_barrier();
            const int rows = min(nrows - 16 * nt, 16);
            for (int i = 64 * w + lane; i < rows * (D / 4); i += 64 * NW) {
                const int r = i / (D / 4), d4 = i % (D / 4);
                float M = m_s[0][r];
#pragma unroll
                for (int x = 1; x < NW; ++x) M = paged_top(M, m_s[x][r]);
                float L = 0.f;
                f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int x = 0; x < NW; ++x) {
                    const float f = fast_exp2(m_s[x][r] - M);  // 0 for a wave that saw none of the row's keys
                    L += f * l_s[x][r];
                    acc += f * *reinterpret_cast<const f32x4_t*>(o_s + x * OW + r * OROW + 4 * d4);
                }
                const int row = 16 * nt + r;
                if (!part.whole) {
                    const long at = (long)part.slot * RT + row;
                    *reinterpret_cast<f32x4_t*>(a.part_o + at * D + 4 * d4) = acc;
                    if (d4 == 0) *reinterpret_cast<float2*>(a.part_ml + 2 * at) = make_float2(M, L);
                    continue;
                }
                const long qr = paged_qrow(a, sq, head, row0 + row);
                const bool any = __float_as_uint(L) != 0;  // L is 0, positive or NaN
                const float inv = any ? 1.f / L : 0.f;
                acc *= inv;
                if constexpr (TERMS == 3) *reinterpret_cast<f32x4_t*>(static_cast<float*>(a.out) + qr * D + 4 * d4) = acc;
                else
                    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + qr * D + 4 * d4) =
                        make_uint2(pack_bf16x2(acc[0], acc[1]), pack_bf16x2(acc[2], acc[3]));
                if (d4 == 0 && a.lse) a.lse[qr] = any ? kLn2 * (M + __log2f(L)) : kNegInf;
            }
        }
        lds_barrier();  // the states have been read: the next part's DMA may come
    }
}

}  // namespace pdec
