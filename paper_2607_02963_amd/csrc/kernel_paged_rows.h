// Attention over paged caches, many query rows per kv head (chunks of new
// tokens; the event streams' queries against a shared prefix), bfloat16, on
// v_mfma_f32_32x32x16_bf16.
//
// An item is 128 NT consecutive rows of a (kv head, sequence), NT 32-row tiles
// in each of four waves, against a run of 64-key units (paged_common.h).  Each
// unit is one stage of a four-slot LDS ring filled by global_load_lds_dwordx4:
// a wave moves 32 keys of K or of V, two halves of 16 keys, which are always
// on one page, so a half has one scalar base and the lanes fixed offsets from
// it.  The products and their operand layouts are those of whole branches
// (kernel_branch.h): per 32-key block S^T = K Q^T and O^T += V^T P^T, the
// scores of block b + 1 multiplied under the exponentials of block b and the
// P V products of block b under the maxima of block b + 1.
//
// 8-bit pages: a wave moves its 32 keys as they are into three raw slots of its
// own, and between two barriers turns those of stage st + 2 into a bfloat16 slot
// of the ring (one v_cvt_scalef32_pk_bf16_fp8 per pair, the key's power of two
// with it: exact), spread over the steps of the P V phases, whose vector work is
// light.  Turning them where they are read would do it once per wave, four times
// in all.  The products and all that follows are the same.
//
// Units that all rows of a wave see whole take that pipelined loop.  Units
// with hidden keys (the chunk's own tokens, the sequence's end, absent pages)
// take a plain one, tile by tile, where a value that is not finite meets only
// the rows that see it.
//
// What bounds it: the matrix cores, with the softmax beside them, as for whole
// branches: 2048 tokens over 32768 keys, 28 heads of 128 over 4 (932 GFLOP) take
// 920 us, 1010 TFLOP/s of the 1241 that a large library product reaches; six chunks
// of 301 to 1023 tokens over 8-bit pages 431 us, 835 TFLOP/s, the difference being
// the widening and the pairs' starts and ends.  lse is exact to float32 here, so
// the row sums are of the unrounded P, on the vector units.
#pragma once

#include "kernel_branch.h"
#include "paged_common.h"

namespace pdec {

// The larger of two scores, NaN if one is.  A NaN raises no row's reference, and its
// probability is NaN whatever that is.  (v_maximum3_f32: fmaxf would quiet each operand
// with a v_max(x, x) first.)
__device__ inline float paged_top(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// The halves of a bf16 pair that are infinite or NaN, as a mask: an exponent of
// all ones carries into its half's top bit.
__device__ inline uint32_t strange_bf16x2(uint32_t w)
{
    const uint32_t m = (((w & 0x7f807f80u) + 0x00800080u) & 0x80008000u) >> 15;
    return (m << 16) - m;
}

// dma_16B_m0 with the wait states for a base that a v_readfirstlane wrote right
// before: pages come from the block table, and the compiler forms some of their
// addresses in vector registers.
__device__ inline void dma_16B_page(uint64_t base, uint32_t off, uint32_t lds_base, uint64_t lanes)
{
    const uint64_t sb = sgpr_base(reinterpret_cast<const void*>(base));
    asm volatile("s_mov_b32 m0, %0\n\ts_mov_b64 exec, %3\n\ts_nop 2\n\tglobal_load_lds_dwordx4 %1, %2\n\ts_mov_b64 exec, -1" :
                 : "s"(__builtin_amdgcn_readfirstlane(lds_base)), "v"(off), "s"(sb), "s"(sgpr_base(reinterpret_cast<const void*>(lanes)))
                 : "memory");
}

// The same for the scales: one dword per lane from the lane's own address.
__device__ inline void dma_4B_lanes(uint64_t addr, uint32_t lds_base, uint64_t lanes)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_mov_b64 exec, %2\n\ts_nop 0\n\tglobal_load_lds_dword %1, off\n\ts_mov_b64 exec, -1" :
                 : "s"(__builtin_amdgcn_readfirstlane(lds_base)), "v"(addr), "s"(sgpr_base(reinterpret_cast<const void*>(lanes)))
                 : "memory");
}

template <int D, int NT, bool FP8>
__global__ __launch_bounds__(256) void paged_rows_kernel(PagedArgs a)
{
    constexpr int NW = 4;
    using C = BranchCfg<D, NT, NW>;
    constexpr int NB = FP8 ? 3 : C::NSTAGE;       // bfloat16 slots of the ring
    constexpr int NRAW = 3, RAW = FP8 ? 32 * D : 0;  // raw slots of a wave, and their bytes
    constexpr int ESZ = FP8 ? 1 : 2;
    constexpr int CPK = D * ESZ / 16;             // 16-byte chunks per key in memory
    constexpr int KPI = 64 / CPK;                 // keys per piece of a DMA instruction
    constexpr int PPW = 32 / KPI;                 // pieces of a wave per stage, a half's one after the other's
    constexpr int AHEAD = FP8 ? 5 : 3;            // stage moved behind the barrier of stage st: st + AHEAD
    constexpr int FLIGHT = FP8 ? 2 * (PPW + 1) : PPW;  // pieces that may be under way at a barrier
    constexpr int SCALES = FP8 ? 64 : 0;          // bytes for the 32 scales of a raw slot
    __shared__ __attribute__((aligned(1024))) unsigned char lds[NB * C::STAGE + NW * NRAW * (RAW + SCALES)];

    const int w = __builtin_amdgcn_readfirstlane(wi_id() >> 6);
    PagedRun run;
    PagedPart part;
    if (!paged_begin(a, paged_worker(a, wg_id()), run, wi_id() == 0)) return;
    __shared__ int find_s[2][2][NW];  // see below; two sets, used in turn
    int turn_s = 0;

    while (paged_next(a, run, part)) {
        if (w == 0 && paged_lane() == 0) paged_note(a, run, part);
        // The lane's offsets belong to the part: kept over the loop they would take
        // the registers that the pipelined loop needs (the compiler hoists what it can,
        // and spills).
        int lane = paged_lane();
        asm volatile("" : "+v"(lane));
        const int l32 = lane & 31, hi = lane >> 5;
        const float c = a.qscale;

        // ---- DMA: this wave moves keys 32 (w % 2) .. + 31 of a unit, of K (w < 2) or V ----
        const bool w_is_v = w >= NW / 2;
        const uint32_t strideB = (uint32_t)a.H_kv * D * ESZ;
        const int pkey = lane / CPK;  // key of the lane within a piece
        uint32_t off[4];  // byte offset of the lane's chunk in piece i, of period 4 in i
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int key = 32 * (w % 2) + pkey + i * KPI;
            // bfloat16 pieces land in the ring's permuted places, raw ones in a row
            const int ch = FP8 ? lane % CPK : (lane % CPK) ^ (w_is_v ? branch_vswz<D>(key) : branch_kswz<D>(key));
            off[i] = (uint32_t)(pkey + (i % (PPW / 2)) * KPI) * strideB + 16u * ch;
        }
        static_assert(16 % KPI == 0 && PPW * KPI == 32 && (PPW / 2 <= 4), "a wave's pieces are two halves of 16 keys");
        unsigned char* const ring_w = lds + (w_is_v ? C::STAGE_K : 0) + 32 * (w % 2) * C::ROWB;  // its keys of slot 0
        unsigned char* const raw_w = lds + NB * C::STAGE + w * NRAW * RAW;                       // its raw slots
        const uint32_t m_base = lds_u32(FP8 ? raw_w : ring_w);
        // 8-bit pages: the lane's first chunk, of key pkey, in raw slot 0 and in slot 0 of
        // the ring; the keys of every second piece have bit 3, which permutes K chunks
        const uint32_t raw0 = lds_u32(raw_w) + 16 * lane;
        const uint32_t ring0 = lds_u32(ring_w) + pkey * C::ROWB + 16 * ((2 * (lane % CPK)) ^ (w_is_v ? branch_vswz<D>(pkey) : branch_kswz<D>(pkey)));
        const uint32_t kflip = w_is_v ? 0 : 128;
        const uint32_t sc_base = lds_u32(lds) + NB * C::STAGE + NW * NRAW * RAW + w * NRAW * SCALES;
        static_assert(!FP8 || D == 64 || KPI == 8, "branch_kswz takes bits 0 to 3 of a key at D = 128, 1 to 3 at D = 64");
        const uint64_t pool = sgpr_base(w_is_v ? a.v_pages : a.k_pages);
        const uint64_t scales = FP8 ? sgpr_base(w_is_v ? a.v_scales : a.k_scales) : 0;

        // operand reads, as for whole branches.  A K step t, and a V tile dt, flip bits
        // of the address that nothing else sets: an address is its slot's and the
        // lane's sum, formed once a stage, with those bits flipped.
        const uint32_t koff = lds_u32(lds) + l32 * C::ROWB + 16 * (hi ^ branch_kswz<D>(l32));
        const int vq = lane >> 4, vi = lane & 15, vkey = 4 * (vq >> 1) + (vi >> 2);
        const uint32_t voff = lds_u32(lds) + C::STAGE_K + vkey * C::ROWB +
                              16 * ((2 * (vq & 1) + ((vi & 3) >> 1)) ^ branch_vswz<D>(vkey)) + 8 * (vi & 1);
        auto slot = [&](int st) __attribute__((always_inline)) { return (uint32_t)((st % NB) * C::STAGE); };
        auto read_k = [&](u32x4_t (&kf)[C::KS], uint32_t kbuf, int kb, int t) __attribute__((always_inline)) {
            typedef __attribute__((address_space(3))) const u32x4_t lds_u32x4_t;
            kf[t] = *(lds_u32x4_t*)(uintptr_t)((kbuf ^ (32 * t)) + kb * C::ROWB);
        };
        // half r (8 keys) of V operand (s, dt), index j = 2 (DT s + dt) + r: lane's keys 16 s + 8 r + 4 (l / 32) .. + 3
        auto read_v = [&](u32x2_t (&vf)[4 * C::DT], uint32_t vbuf, int kb, int j) __attribute__((always_inline)) {
            const int s = j / (2 * C::DT), dt = (j / 2) % C::DT;
            vf[j] = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                                    (__attribute__((address_space(3))) s16x4_t*)(uintptr_t)(
                                                        (vbuf ^ (64 * dt)) + (kb + 16 * s + 8 * (j & 1)) * C::ROWB)));
        };
        auto v_op = [&](const u32x2_t (&vf)[4 * C::DT], int s, int dt) __attribute__((always_inline)) {
            const u32x2_t x0 = vf[2 * (C::DT * s + dt)], x1 = vf[2 * (C::DT * s + dt) + 1];
            return u32x4_t{x0.x, x0.y, x1.x, x1.y};
        };

        const PagedSeq sq = part.seq;
        const int R = sq.n * a.G, row0 = part.group * C::RT, nrows = min(C::RT, R - row0);
        const int32_t* table = a.block_table + (long)part.s * a.max_pages;
        // The first page that is there, and the first that is not, among the part's
        // table entries; every lane looks at every 256th.
        auto find = [&](int e0, int e1, int& there, int& absent) __attribute__((always_inline)) {
            int first[2] = {e1, e1};
            for (int e = e0 + 64 * w; e < e1; e += 64 * NW) {
                const bool in = e + lane < e1;
                const bool ok = in && (uint32_t)table[min(e + lane, e1 - 1)] < (uint32_t)a.num_pages;
                const uint64_t b[2] = {__ballot(ok), __ballot(in && !ok)};
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    if (b[k] && first[k] == e1) first[k] = e + __builtin_ctzll(b[k]);
            }
            if (lane < 2) find_s[turn_s][lane][w] = lane ? first[1] : first[0];
            lds_barrier();  // also: no wave reads the ring for the part before any more
            there = absent = e1;
#pragma unroll
            for (int k = 0; k < NW; ++k) {
                there = min(there, __builtin_amdgcn_readfirstlane(find_s[turn_s][0][k]));
                absent = min(absent, __builtin_amdgcn_readfirstlane(find_s[turn_s][1][k]));
            }
            turn_s ^= 1;
        };
        const int e1 = min((part.u1 * kUnit - 1) >> a.page_shift, a.max_pages - 1) + 1;
        int there0, absent0;
        find(min((part.u0 * kUnit) >> a.page_shift, e1 - 1), e1, there0, absent0);
        // units at the front without a page (a cache that drops its oldest pages) are left out
        const int u0 = there0 == e1 ? part.u1 : max(part.u0, (there0 << a.page_shift) / kUnit);
        if (absent0 < there0 && u0 < part.u1) {
            find(there0, e1, there0, absent0);
            // the first page may begin inside its unit
            if ((there0 << a.page_shift) > u0 * kUnit) absent0 = (u0 * kUnit) >> a.page_shift;
        }
        const int nst = __builtin_amdgcn_readfirstlane(part.u1 - u0), t0 = __builtin_amdgcn_readfirstlane(u0 * kUnit);
        const int wrow0 = C::WROWS * w;
        const bool active = wrow0 < nrows;
        const uint64_t base0 = pool + (uint64_t)part.head * D * ESZ;

        // Pages of stage st's two halves that this wave moves.  Stages past the last repeat it.
        struct Pages { int half[2]; };
        auto pages = [&](int st) __attribute__((always_inline)) {
            const int t = t0 + max(min(st, nst - 1), 0) * kUnit + 32 * (w & 1);
            Pages x;
#pragma unroll
            for (int h = 0; h < 2; ++h) x.half[h] = paged_entry(table, min((t + 16 * h) >> a.page_shift, a.max_pages - 1));
            return x;
        };
        // An absent page is read as page 0; its keys are masked.
        struct Pending { uint64_t base[2]; uint32_t dst; uint64_t lanes; uint64_t scale; uint32_t scale_dst; };
        auto pending = [&](int st, const Pages& x) __attribute__((always_inline)) {
            const int t = t0 + min(st, nst - 1) * kUnit + 32 * (w & 1);
            Pending p;
            uint64_t sc[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int page = (uint32_t)x.half[h] < (uint32_t)a.num_pages ? x.half[h] : 0;
                const int row = (t + 16 * h) & ((1 << a.page_shift) - 1);
                p.base[h] = base0 + (((uint64_t)(uint32_t)page << a.page_shift) + (uint32_t)row) * strideB;
                sc[h] = scales + ((((uint64_t)(uint32_t)page * a.H_kv + part.head) << a.page_shift) + (uint32_t)row);
            }
            p.dst = m_base + (FP8 ? (st % NRAW) * RAW : (st % NB) * C::STAGE);
            p.lanes = ring_lanes(st, nst);
            if constexpr (FP8) {  // lanes 0 .. 3 the first half's 16 bytes, 4 .. 7 the second's
                p.scale = (lane & 4 ? sc[1] : sc[0]) + 4 * (lane & 3);
                p.scale_dst = sc_base + (st % NRAW) * SCALES;
            }
            return p;
        };
        auto issue_piece = [&](const Pending& pd, int i) __attribute__((always_inline)) {
            dma_16B_page(pd.base[i / (PPW / 2)], off[i & 3], pd.dst + 1024 * i, pd.lanes);
        };
        auto issue_stage = [&](const Pending& pd) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < PPW; ++i) issue_piece(pd, i);
            if constexpr (FP8) dma_4B_lanes(pd.scale, pd.scale_dst, pd.lanes & 255u);
        };

        // 8-bit pages, the turning of a raw stage: item m of 4 PPW is word m % 4 of
        // chunk m / 4.  from: the lane's 16 bytes of chunk 0 in the raw slot; sc: its
        // key's scale byte; to: the place of the first half of its first key's chunk in
        // the ring.  The second half is beside it, and chunk i's key i KPI rows on, its
        // K chunks permuted by one bit more.  A chunk is read while the one before it is
        // turned.
        typedef __attribute__((address_space(3))) u32x4_t lds_u32x4_t;
        typedef __attribute__((address_space(3))) uint8_t lds_u8_t;
        u32x4_t raw[2], wide;
        float scale[2];
        struct Turn { uint32_t from, sc, to; };
        auto turn_of = [&](int st) __attribute__((always_inline)) {
            return Turn{raw0 + (st % NRAW) * RAW, sc_base + (st % NRAW) * SCALES + pkey, ring0 + (st % NB) * C::STAGE};
        };
        auto read_raw = [&](const Turn& u, int i) __attribute__((always_inline)) {
            raw[i & 1] = *reinterpret_cast<const lds_u32x4_t*>((uintptr_t)(u.from + 1024 * i));
            scale[i & 1] = paged_scale(*reinterpret_cast<const lds_u8_t*>((uintptr_t)(u.sc + KPI * i)), 0);
        };
        auto turn = [&](const Turn& u, int m) __attribute__((always_inline)) {
            const int i = m / 4, j = m % 4;
            if (j == 0 && i + 1 < PPW) read_raw(u, i + 1);
            const uint32_t word = raw[i & 1][j];
            wide[2 * (j & 1)] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(word, scale[i & 1], false));
            wide[2 * (j & 1) + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(word, scale[i & 1], true));
            if (j & 1) {
                const uint32_t flip = (D == 128 && (i & 1) ? kflip : 0) + 16 * (j >> 1);
                *reinterpret_cast<lds_u32x4_t*>((uintptr_t)((u.to ^ flip) + i * KPI * C::ROWB)) = wide;
            }
        };
        constexpr int ITEMS = 4 * PPW;
        auto turn_stage = [&](int st) __attribute__((always_inline)) {
            const Turn u = turn_of(st);
            read_raw(u, 0);
#pragma unroll
            for (int m = 0; m < ITEMS; ++m) turn(u, m);
        };

        // ---- this lane's rows: 32 nt + l % 32 of the wave ----
        u32x4_t qf[NT][C::KS];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            // rows past the item's last repeat it; their results are not stored
            const int r = row0 + min(wrow0 + 32 * nt + l32, nrows - 1);
            const uint16_t* q = static_cast<const uint16_t*>(a.q) + paged_qrow(a, sq, part.head, r) * D + 8 * hi;
#pragma unroll
            for (int t = 0; t < C::KS; ++t) qf[nt][t] = *reinterpret_cast<const u32x4_t*>(q + 16 * t);
        }
        const int least = __builtin_amdgcn_readfirstlane(paged_seen(a, sq, (row0 + min(wrow0, nrows - 1)) / a.G));
        // The wave's first nd stages are seen whole by all of its rows.
        const bool holes = absent0 < e1;
        const int nd = __builtin_amdgcn_readfirstlane(
            !active ? 0 : max(min(min(least / kUnit, part.u1), holes ? (absent0 << a.page_shift) / kUnit : part.u1) - u0, 0));
        // Pages of stage st + AHEAD before the barrier of stage st, read one stage ago.
        Pages ahead;
        if (nst > 0) {
#pragma unroll
            for (int st = 0; st < 3; ++st) issue_stage(pending(st, pages(st)));
        }
        // the query loads and the DMA complete in no order relative to each other
        wait_vmcnt<0>();
        if constexpr (FP8) {
            // a wave reads only its own raw slots: no barrier
#pragma unroll
            for (int st = 0; st < 2; ++st)
                if (nst > 0) {
                    turn_stage(st);
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                    issue_stage(pending(st + 3, pages(st + 3)));
                }
        }
        ahead = pages(AHEAD);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int t = 0; t < C::KS; ++t) asm volatile("" : "+a"(qf[nt][t]));

        bf32x16_t o[NT][C::DT];
        float lsum[NT], m_ref[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            m_ref[nt] = kMinRef;
            lsum[nt] = 0.f;
#pragma unroll
            for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[nt][dt][i] = 0.f;
        }

        auto score_step = [&](bf32x16_t (&s)[NT], const u32x4_t (&kf)[C::KS], int i) __attribute__((always_inline)) {
            const int t = i / NT, nt = i % NT;
            if (t == 0) {
#pragma unroll
                for (int k = 0; k < 16; ++k) s[nt][k] = 0.f;
            }
            s[nt] = branch_mfma(kf[t], qf[nt][t], s[nt]);
        };
        auto pv_step = [&](const u32x4_t (&pk)[NT][2], const u32x2_t (&vf)[4 * C::DT], int i) __attribute__((always_inline)) {
            const int s = i / (C::DT * NT), dt = (i / NT) % C::DT, nt = i % NT;
            o[nt][dt] = branch_mfma(v_op(vf, s, dt), pk[nt][s], o[nt][dt]);
        };
        // max of element pair i (0 .. 8 NT - 1) into mx
        auto max_step = [&](float (&mx)[NT], const bf32x16_t (&s)[NT], int i) __attribute__((always_inline)) {
            const int nt = i / 8, k = 2 * (i % 8);
            mx[nt] = k == 0 ? paged_top(s[nt][0], s[nt][1]) : paged_top(paged_top(mx[nt], s[nt][k]), s[nt][k + 1]);
        };
        // a row's reference max moves only when its block max exceeds it by more than 8
        auto rescale_tile = [&](float mx, int nt) __attribute__((always_inline)) {
            const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
            const float mt = paged_top(__uint_as_float(b[0]), __uint_as_float(b[1])) * c;
            const bool up = mt > m_ref[nt] + 8.f;
            const float alpha = up ? fast_exp2(m_ref[nt] - mt) : 1.f;
            m_ref[nt] = up ? mt : m_ref[nt];
            lsum[nt] *= alpha;
#pragma unroll
            for (int dt = 0; dt < C::DT; ++dt) o[nt][dt] *= alpha;
        };
        auto rescale = [&](const float (&mx)[NT]) __attribute__((always_inline)) {
            bool need = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) need |= mx[nt] * c > m_ref[nt] + 8.f;
            if (__any(need)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) rescale_tile(mx[nt], nt);
            }
        };
        // P of element pair i (0 .. 8 NT - 1), rounded to bf16, the product's operand type, by half
        // a step (2^-8) of each term, as out is; the row sums take it unrounded
        auto prob_step = [&](u32x4_t (&pk)[NT][2], const bf32x16_t (&s)[NT], int i) __attribute__((always_inline)) {
            const int nt = i / 8, k = i % 8;
            const float p0 = fast_exp2(fmaf(s[nt][2 * k], c, -m_ref[nt])), p1 = fast_exp2(fmaf(s[nt][2 * k + 1], c, -m_ref[nt]));
            lsum[nt] += p0 + p1;
            pk[nt][k >> 2][k & 3] = pack_bf16x2(p0, p1);
            // keeps P in the phase that computes it
            if ((k & 3) == 3) asm volatile("" : "+v"(pk[nt][k >> 2]));
        };

        // The two phases of a block (kernel_branch.h).
        // A: the next block's scores sn under this block's exponentials.
        auto phase_a = [&](bf32x16_t (&sn)[NT], const bf32x16_t (&sc)[NT], u32x4_t (&pk)[NT][2],
                           const u32x4_t (&kf)[C::KS], u32x2_t (&vf)[4 * C::DT], uint32_t vbuf,
                           int kb) __attribute__((always_inline)) {
            constexpr int STEPS = NT * C::KS;
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                score_step(sn, kf, i);
#pragma unroll
                for (int j = i * 4 * C::DT / STEPS; j < (i + 1) * 4 * C::DT / STEPS; ++j) read_v(vf, vbuf, kb, j);
#pragma unroll
                for (int j = i * 8 * NT / STEPS; j < (i + 1) * 8 * NT / STEPS; ++j) prob_step(pk, sc, j);
            }
        };
        // B: this block's P V products under the next block's maxima, the K
        // operands of the block after it, and extra(i, steps) at step i.
        auto phase_b = [&](auto extra, const u32x4_t (&pk)[NT][2], const u32x2_t (&vf)[4 * C::DT],
                           const bf32x16_t (&sn)[NT], float (&mx)[NT], u32x4_t (&kf)[C::KS], uint32_t kbuf,
                           int nkb) __attribute__((always_inline)) {
            constexpr int STEPS = 2 * C::DT * NT;
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                pv_step(pk, vf, i);
#pragma unroll
                for (int j = i * C::KS / STEPS; j < (i + 1) * C::KS / STEPS; ++j) read_k(kf, kbuf, nkb, j);
                extra(i, STEPS);
#pragma unroll
                for (int j = i * 8 * NT / STEPS; j < (i + 1) * 8 * NT / STEPS; ++j) max_step(mx, sn, j);
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) asm volatile("" : "+v"(mx[nt]));
        };
        // Every wave passes one barrier per stage, in either loop; behind the one of
        // stage st, stage st + 1 is in the ring and stage st - 1 been consumed for all
        // of them.  bfloat16 pages: the slot of the latter takes stage st + 3.  8-bit
        // pages: stage st + 2 has landed in the wave's raw slot; it goes to the slot of
        // stage st - 1, and its raw slot then takes stage st + 5.
        if (nst > 0) lds_barrier();  // stages 0 and 1 are in the ring
        if (nd > 0) {
            // Entering stage st: sa holds block 0's scores (reference set), kf block 1's K operands.
            bf32x16_t sa[NT], sb[NT];
            u32x4_t kf[C::KS], pk[NT][2];
            u32x2_t vf[4 * C::DT];
            float mx[NT];
#pragma unroll
            for (int t = 0; t < C::KS; ++t) read_k(kf, koff + slot(0), 0, t);
#pragma unroll
            for (int i = 0; i < NT * C::KS; ++i) score_step(sa, kf, i);
#pragma unroll
            for (int i = 0; i < 8 * NT; ++i) max_step(mx, sa, i);
            rescale(mx);
#pragma unroll
            for (int t = 0; t < C::KS; ++t) read_k(kf, koff + slot(0), 32, t);
            for (int st = 0; st < nd; ++st) {
                const uint32_t vbuf = voff + slot(st), kbuf = koff + slot(st + 1);
                phase_a(sb, sa, pk, kf, vf, vbuf, 0);
                const Pending pd = pending(st + AHEAD, ahead);
                ahead = pages(st + AHEAD + 1);
                stage_barrier<FLIGHT>();
                const Turn u = turn_of(st + 2);
                if constexpr (FP8) read_raw(u, 0);
                phase_b(
                    [&](int i, int steps) __attribute__((always_inline)) {
                        if constexpr (FP8) {
#pragma unroll
                            for (int m = i * (ITEMS / 2) / steps; m < (i + 1) * (ITEMS / 2) / steps; ++m) turn(u, m);
                        } else {
#pragma unroll
                            for (int j = i * PPW / steps; j < (i + 1) * PPW / steps; ++j) issue_piece(pd, j);
                        }
                    },
                    pk, vf, sb, mx, kf, kbuf, 0);
                rescale(mx);
                phase_a(sa, sb, pk, kf, vf, vbuf, 32);
                phase_b(
                    [&](int i, int steps) __attribute__((always_inline)) {
                        if constexpr (FP8) {
#pragma unroll
                            for (int m = i * (ITEMS / 2) / steps; m < (i + 1) * (ITEMS / 2) / steps; ++m) turn(u, ITEMS / 2 + m);
                        }
                    },
                    pk, vf, sa, mx, kf, kbuf, 32);
                if constexpr (FP8) issue_stage(pd);  // the raw slot has been read
                if (st + 1 < nd) rescale(mx);
            }
        }
        int seen[NT];  // keys that the lane's rows see
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) seen[nt] = paged_seen(a, sq, (row0 + min(wrow0 + 32 * nt + l32, nrows - 1)) / a.G);
        for (int st = nd; st < nst; ++st) {
            {
                const Pending pd = pending(st + AHEAD, ahead);
                ahead = pages(st + AHEAD + 1);
                stage_barrier<FLIGHT>();
                if constexpr (FP8) {
                    turn_stage(st + 2);
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the raw slot has been read
                }
                issue_stage(pd);
            }
            const uint32_t vbuf = voff + slot(st), kbuf = koff + slot(st);
            const int t = t0 + st * kUnit;
            int most = 0;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) most = max(most, seen[nt]);
            if (!active) continue;
#pragma unroll 1
            for (int kb = 0; kb < kUnit; kb += 32) {
                auto there = [&](int x) { return (uint32_t)paged_entry(table, min(x >> a.page_shift, a.max_pages - 1)) < (uint32_t)a.num_pages; };
                const bool there0 = !holes || there(t + kb), there1 = !holes || there(t + kb + 16);
                if (!(there0 | there1) || !__any(most > t + kb)) continue;
                u32x4_t kf[C::KS], pk[NT][2];
                u32x2_t vf[4 * C::DT];
                bf32x16_t s[NT];
                float mx[NT];
#pragma unroll
                for (int i = 0; i < C::KS; ++i) read_k(kf, kbuf, kb, i);
#pragma unroll
                for (int j = 0; j < 4 * C::DT; ++j) read_v(vf, vbuf, kb, j);
                typedef __attribute__((ext_vector_type(2))) uint16_t u16x2_t;
                u16x2_t top = {0, 0};  // the largest magnitudes, as their bits
#pragma unroll
                for (int j = 0; j < 4 * C::DT; ++j) {
                    top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2_t, vf[j].x & 0x7fff7fffu));
                    top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2_t, vf[j].y & 0x7fff7fffu));
                }
                const bool apart = __any(max(top.x, top.y) >= 0x7f80);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const int lim = seen[nt] - t - kb;  // visible keys of the lane's row in the block
                    __builtin_amdgcn_sched_barrier(0);
                    if (!__any(lim > 0)) continue;
#pragma unroll
                    for (int i = 0; i < C::KS; ++i) score_step(s, kf, i * NT + nt);
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const bool hidden = (8 * (i >> 2) + (i & 3) >= lim - 4 * hi) | !(i < 8 ? there0 : there1);
                        s[nt][i] = hidden ? kNegInf : s[nt][i];
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) max_step(mx, s, 8 * nt + i);
                    if (__any(mx[nt] * c > m_ref[nt] + 8.f)) rescale_tile(mx[nt], nt);
#pragma unroll
                    for (int i = 0; i < 8; ++i) prob_step(pk, s, 8 * nt + i);
                    // 0 times an infinite or NaN value is NaN: such values are left out of
                    // the products, then added key by key to the rows that see the key
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int dt = 0; dt < C::DT; ++dt) {
                            u32x4_t v = v_op(vf, k, dt);
                            if (apart) {
                                asm volatile("" : "+v"(v));
#pragma unroll
                                for (int e = 0; e < 4; ++e) v[e] &= ~strange_bf16x2(v[e]);
                            }
                            o[nt][dt] = branch_mfma(v, pk[nt][k], o[nt][dt]);
                        }
                    if (!apart) continue;
#pragma unroll
                    for (int j = 0; j < 2 * C::DT; ++j) {
                        const int k = j / C::DT, dt = j % C::DT;
                        const u32x4_t v0 = v_op(vf, k, dt);
                        bf32x16_t sum = o[nt][dt];
#pragma unroll 1
                        for (int key = 0; key < 16; ++key) {
                            const bool sees = (16 * k + key < lim) & (k ? there1 : there0);
                            const bool mine = hi == ((key >> 2) & 1);
                            const int word = 2 * (key >> 3) + ((key & 3) >> 1);
                            const uint32_t half = (key & 1) ? 0xffff0000u : 0xffffu;
                            u32x4_t v = v0;
                            asm volatile("" : "+v"(v));  // nothing of this rare loop before it
#pragma unroll
                            for (int e = 0; e < 4; ++e) v[e] &= strange_bf16x2(v[e]) & ((mine & (e == word)) ? half : 0u);
                            const bf32x16_t x = branch_mfma(v, pk[nt][k], sum);
#pragma unroll
                            for (int i = 0; i < 16; ++i) sum[i] = sees ? x[i] : sum[i];
                        }
                        o[nt][dt] = sum;
                    }
                }
            }
        }
        wait_vmcnt<0>();  // no DMA into the LDS outlives the part

        if (!active) continue;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const float l = lsum[nt] + __shfl_xor(lsum[nt], 32);  // both lanes of the row
            const int r = wrow0 + 32 * nt + l32;
            if (r >= nrows) continue;
            if (!part.whole) {
                const long at = (long)part.slot * C::RT + r;
#pragma unroll
                for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        *reinterpret_cast<f32x4_t*>(a.part_o + at * D + 32 * dt + 8 * k + 4 * hi) =
                            f32x4_t{o[nt][dt][4 * k], o[nt][dt][4 * k + 1], o[nt][dt][4 * k + 2], o[nt][dt][4 * k + 3]};
                if (hi == 0) *reinterpret_cast<float2*>(a.part_ml + 2 * at) = make_float2(m_ref[nt], l);
                continue;
            }
            const long qr = paged_qrow(a, sq, part.head, row0 + r);
            const bool any = __float_as_uint(l) != 0;  // l is 0, positive or NaN
            const float inv = any ? 1.f / l : 0.f;
            uint16_t* dst = static_cast<uint16_t*>(a.out) + qr * D;
#pragma unroll
            for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    *reinterpret_cast<uint2*>(dst + 32 * dt + 8 * k + 4 * hi) =
                        make_uint2(pack_bf16x2(o[nt][dt][4 * k] * inv, o[nt][dt][4 * k + 1] * inv),
                                   pack_bf16x2(o[nt][dt][4 * k + 2] * inv, o[nt][dt][4 * k + 3] * inv));
            if (hi == 0 && a.lse) a.lse[qr] = any ? kLn2 * (m_ref[nt] + __log2f(l)) : kNegInf;
        }
    }
}

}  // namespace pdec
