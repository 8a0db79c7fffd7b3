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
// Units that all rows of a wave see whole take that pipelined loop.  Units
// with hidden keys (the chunk's own tokens, the sequence's end, absent pages)
// take a plain one, tile by tile, where a value that is not finite meets only
// the rows that see it.
//
// What bounds it: the matrix cores, with the softmax beside them, as for whole
// branches.  lse is exact to float32 here, so the row sums are of the
// unrounded P, on the vector units.
#pragma once

#include "kernel_branch.h"
#include "paged_common.h"

namespace pdec {

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

template <int D, int NT>
__global__ __launch_bounds__(256) void paged_rows_kernel(PagedArgs a)
{
    constexpr int NW = 4;
    using C = BranchCfg<D, NT, NW>;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[C::NSTAGE * C::STAGE];

    const int tid = wi_id();
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lane = tid & 63, l32 = lane & 31, hi = lane >> 5;
    const float c = a.qscale;
    PagedRun run;
    PagedPart part;
    const int worker = paged_worker(a, wg_id(), (int)__builtin_amdgcn_grid_size_x() / 256);
    if (!paged_begin(a, worker, run)) {
        if (tid == 0 && !a.whole && !a.by_pair) a.cut[worker] = make_int4(-1, 0, 0, 0);
        return;
    }

    // ---- DMA: this wave moves keys 32 (w % 2) .. + 31 of a unit, of K (w < 2) or V ----
    const bool w_is_v = w >= NW / 2;
    const uint32_t strideB = (uint32_t)a.H_kv * D * 2;
    const int pkey = lane / C::CH;  // key of the lane within a piece
    const int key0 = 32 * (w % 2) + pkey;
    uint32_t off[4];  // byte offset of the lane's chunk in piece i of a half, of period 4 in i
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int key = key0 + i * C::KPI;
        off[i] = (uint32_t)(pkey + (i % (C::PPW / 2)) * C::KPI) * strideB +
                 16u * ((lane % C::CH) ^ (w_is_v ? branch_vswz<D>(key) : branch_kswz<D>(key)));
    }
    static_assert(16 % C::KPI == 0 && C::PPW * C::KPI == 32, "a wave's pieces are two halves of 16 keys");
    const uint32_t m_base = lds_u32(lds) + (w_is_v ? C::STAGE_K : 0) + 32 * (w % 2) * C::ROWB;
    const uint64_t pool = sgpr_base(w_is_v ? a.v_pages : a.k_pages);

    // operand reads, as for whole branches
    const int koff = l32 * C::ROWB + 16 * (hi ^ branch_kswz<D>(l32));
    int voff[C::DT];
    {
        const int q = lane >> 4, i = lane & 15;
        const int key = 4 * (q >> 1) + (i >> 2);
#pragma unroll
        for (int dt = 0; dt < C::DT; ++dt)
            voff[dt] = key * C::ROWB + 16 * ((4 * dt + 2 * (q & 1) + ((i & 3) >> 1)) ^ branch_vswz<D>(key)) + 8 * (i & 1);
    }
    auto slot = [&](int st) __attribute__((always_inline)) { return lds + (st % C::NSTAGE) * C::STAGE; };
    auto read_k = [&](u32x4_t (&kf)[C::KS], const unsigned char* buf, int kb, int t) __attribute__((always_inline)) {
        kf[t] = *reinterpret_cast<const u32x4_t*>(buf + kb * C::ROWB + (koff ^ (32 * t)));
    };
    // half r (8 keys) of V operand (s, dt), index j = 2 (DT s + dt) + r: lane's keys 16 s + 8 r + 4 (l / 32) .. + 3
    auto read_v = [&](u32x2_t (&vf)[4 * C::DT], const unsigned char* buf, int kb, int j) __attribute__((always_inline)) {
        const int s = j / (2 * C::DT), dt = (j / 2) % C::DT;
        const unsigned char* va = buf + C::STAGE_K + (kb + 16 * s + 8 * (j & 1)) * C::ROWB + voff[dt];
        vf[j] = __builtin_bit_cast(u32x2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                                (__attribute__((address_space(3))) s16x4_t*)va));
    };
    auto v_op = [&](const u32x2_t (&vf)[4 * C::DT], int s, int dt) __attribute__((always_inline)) {
        const u32x2_t x0 = vf[2 * (C::DT * s + dt)], x1 = vf[2 * (C::DT * s + dt) + 1];
        return u32x4_t{x0.x, x0.y, x1.x, x1.y};
    };

    while (paged_next(a, run, part, tid == 0)) {
        const PagedSeq sq = paged_seq(a, part.s);
        const int R = sq.n * a.G, row0 = part.group * C::RT, nrows = min(C::RT, R - row0);
        const int32_t* table = a.block_table + (long)part.s * a.max_pages;
        // units at the front without a page (a cache that drops its oldest pages) are left out
        const int u0 = min(paged_find(a, part.s, part.u0, part.u1, true), part.u1);
        const int nst = part.u1 - u0, t0 = u0 * kUnit;
        const int wrow0 = C::WROWS * w;
        const bool active = wrow0 < nrows;
        const uint64_t base0 = pool + 2 * (uint64_t)part.head * D;

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
        struct Pending { uint64_t base[2]; uint32_t dst; uint64_t lanes; };
        auto pending = [&](int st, const Pages& x) __attribute__((always_inline)) {
            const int t = t0 + min(st, nst - 1) * kUnit + 32 * (w & 1);
            Pending p;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int page = (uint32_t)x.half[h] < (uint32_t)a.num_pages ? x.half[h] : 0;
                const int row = (t + 16 * h) & ((1 << a.page_shift) - 1);
                p.base[h] = base0 + (((uint64_t)(uint32_t)page << a.page_shift) + (uint32_t)row) * strideB;
            }
            p.dst = m_base + (st % C::NSTAGE) * C::STAGE;
            p.lanes = ring_lanes(st, nst);
            return p;
        };
        auto issue_piece = [&](const Pending& pd, int i) __attribute__((always_inline)) {
            dma_16B_page(pd.base[i / (C::PPW / 2)], off[i & 3], pd.dst + 1024 * i, pd.lanes);
        };
        auto issue_stage = [&](const Pending& pd) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < C::PPW; ++i) issue_piece(pd, i);
        };

        // ---- this lane's rows: 32 nt + l % 32 of the wave ----
        int seen[NT];  // keys that the lane's row sees
        u32x4_t qf[NT][C::KS];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            // rows past the item's last repeat it; their results are not stored
            const int r = row0 + min(wrow0 + 32 * nt + l32, nrows - 1);
            seen[nt] = paged_seen(a, sq, r / a.G);
            const uint16_t* q = static_cast<const uint16_t*>(a.q) + paged_qrow(a, sq, part.head, r) * D + 8 * hi;
#pragma unroll
            for (int t = 0; t < C::KS; ++t) qf[nt][t] = *reinterpret_cast<const u32x4_t*>(q + 16 * t);
        }
        const int least = __builtin_amdgcn_readfirstlane(paged_seen(a, sq, (row0 + min(wrow0, nrows - 1)) / a.G));
        // The wave's first nd stages are seen whole by all of its rows.
        const int nd = !active ? 0 : max(min(paged_find(a, part.s, u0, min(part.u1, least / kUnit), false), least / kUnit) - u0, 0);
        lds_barrier();  // no wave reads the ring for the part before any more
#pragma unroll
        for (int st = 0; st < C::NSTAGE - 1; ++st)
            if (nst > 0) issue_stage(pending(st, pages(st)));
        Pages ahead = pages(C::NSTAGE - 1);  // the pages of the next stage to move
        // the query loads and the DMA complete in no order relative to each other
        wait_vmcnt<0>();
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
            mx[nt] = k == 0 ? fmaxf(s[nt][0], s[nt][1]) : fmaxf(fmaxf(mx[nt], s[nt][k]), s[nt][k + 1]);
        };
        // a row's reference max moves only when its block max exceeds it by more than 8
        auto rescale_tile = [&](float mx, int nt) __attribute__((always_inline)) {
            const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
            const float mt = fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1])) * c;
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
        // P of element pair i (0 .. 8 NT - 1), rounded to bf16 for the product; the row sums take it unrounded
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
                           const u32x4_t (&kf)[C::KS], u32x2_t (&vf)[4 * C::DT], const unsigned char* buf,
                           int kb) __attribute__((always_inline)) {
            constexpr int STEPS = NT * C::KS;
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                score_step(sn, kf, i);
#pragma unroll
                for (int j = i * 4 * C::DT / STEPS; j < (i + 1) * 4 * C::DT / STEPS; ++j) read_v(vf, buf, kb, j);
#pragma unroll
                for (int j = i * 8 * NT / STEPS; j < (i + 1) * 8 * NT / STEPS; ++j) prob_step(pk, sc, j);
            }
        };
        // B: this block's P V products under the next block's maxima, the K
        // operands of the block after it and, with DMA, a later stage's pieces.
        auto phase_b = [&](auto dma, const u32x4_t (&pk)[NT][2], const u32x2_t (&vf)[4 * C::DT],
                           const bf32x16_t (&sn)[NT], float (&mx)[NT], u32x4_t (&kf)[C::KS], const unsigned char* nbuf,
                           int nkb, const Pending& pd) __attribute__((always_inline)) {
            constexpr int STEPS = 2 * C::DT * NT;
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                pv_step(pk, vf, i);
#pragma unroll
                for (int j = i * C::KS / STEPS; j < (i + 1) * C::KS / STEPS; ++j) read_k(kf, nbuf, nkb, j);
                if constexpr (decltype(dma)::value) {
#pragma unroll
                    for (int j = i * C::PPW / STEPS; j < (i + 1) * C::PPW / STEPS; ++j) issue_piece(pd, j);
                }
#pragma unroll
                for (int j = i * 8 * NT / STEPS; j < (i + 1) * 8 * NT / STEPS; ++j) max_step(mx, sn, j);
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) asm volatile("" : "+v"(mx[nt]));
        };
        // Every wave passes one barrier per stage, in either loop; behind the one of
        // stage st, stage st + 1 has landed and stage st - 1 been consumed for all of
        // them, and the slot of the latter takes stage st + 3, whose pages were read
        // one stage ago.
        if (nst > 0) lds_barrier();  // the first three stages have landed
        if (nd > 0) {
            // Entering stage st: sa holds block 0's scores (reference set), kf block 1's K operands.
            bf32x16_t sa[NT], sb[NT];
            u32x4_t kf[C::KS], pk[NT][2];
            u32x2_t vf[4 * C::DT];
            float mx[NT];
#pragma unroll
            for (int t = 0; t < C::KS; ++t) read_k(kf, slot(0), 0, t);
#pragma unroll
            for (int i = 0; i < NT * C::KS; ++i) score_step(sa, kf, i);
#pragma unroll
            for (int i = 0; i < 8 * NT; ++i) max_step(mx, sa, i);
            rescale(mx);
#pragma unroll
            for (int t = 0; t < C::KS; ++t) read_k(kf, slot(0), 32, t);
            for (int st = 0; st < nd; ++st) {
                const unsigned char* buf = slot(st);
                const unsigned char* nbuf = slot(st + 1);
                phase_a(sb, sa, pk, kf, vf, buf, 0);
                const Pending pd = pending(st + 3, ahead);
                ahead = pages(st + 4);
                stage_barrier<C::PPW>();
                phase_b(std::true_type{}, pk, vf, sb, mx, kf, nbuf, 0, pd);
                rescale(mx);
                phase_a(sa, sb, pk, kf, vf, buf, 32);
                phase_b(std::false_type{}, pk, vf, sa, mx, kf, nbuf, 32, pd);
                if (st + 1 < nd) rescale(mx);
            }
        }
        for (int st = nd; st < nst; ++st) {
            {
                const Pending pd = pending(st + 3, ahead);
                ahead = pages(st + 4);
                stage_barrier<C::PPW>();
                issue_stage(pd);
            }
            const unsigned char* buf = slot(st);
            const int t = t0 + st * kUnit;
            int most = 0;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) most = max(most, seen[nt]);
            if (!active) continue;
#pragma unroll 1
            for (int kb = 0; kb < kUnit; kb += 32) {
                auto there = [&](int x) { return (uint32_t)paged_entry(table, min(x >> a.page_shift, a.max_pages - 1)) < (uint32_t)a.num_pages; };
                const bool there0 = there(t + kb), there1 = there(t + kb + 16);
                if (!(there0 | there1) || !__any(most > t + kb)) continue;
                u32x4_t kf[C::KS], pk[NT][2];
                u32x2_t vf[4 * C::DT];
                bf32x16_t s[NT];
                float mx[NT];
#pragma unroll
                for (int i = 0; i < C::KS; ++i) read_k(kf, buf, kb, i);
#pragma unroll
                for (int j = 0; j < 4 * C::DT; ++j) read_v(vf, buf, kb, j);
                uint32_t odd = 0;
#pragma unroll
                for (int j = 0; j < 4 * C::DT; ++j) odd |= strange_bf16x2(vf[j].x) | strange_bf16x2(vf[j].y);
                const bool apart = __any(odd != 0);
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
                    for (int k = 0; k < 2; ++k)
#pragma unroll 1
                        for (int key = 0; key < 16; ++key) {
                            const bool sees = (16 * k + key < lim) & (k ? there1 : there0);
                            const bool mine = hi == ((key >> 2) & 1);
                            const int word = 2 * (key >> 3) + ((key & 3) >> 1);
                            const uint32_t half = (key & 1) ? 0xffff0000u : 0xffffu;
#pragma unroll
                            for (int dt = 0; dt < C::DT; ++dt) {
                                u32x4_t v = v_op(vf, k, dt);
                                asm volatile("" : "+v"(v));  // nothing of this rare loop before it
#pragma unroll
                                for (int e = 0; e < 4; ++e) v[e] &= strange_bf16x2(v[e]) & ((mine & (e == word)) ? half : 0u);
                                const bf32x16_t x = branch_mfma(v, pk[nt][k], o[nt][dt]);
#pragma unroll
                                for (int i = 0; i < 16; ++i) o[nt][dt][i] = sees ? x[i] : o[nt][dt][i];
                            }
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
