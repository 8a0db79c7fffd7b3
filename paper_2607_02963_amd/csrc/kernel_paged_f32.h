// Attention over paged caches on v_mfma_f32_16x16x4_f32: float32 queries, over
// float32 or 8-bit pages.
//
// The work-group is 4 waves; wave w takes keys 16 w .. 16 w + 15 of every unit
// (one page, as pages hold 16 tokens at least) with an online-softmax state of
// its own, for the item's 16 NT rows; the four states are merged in LDS at the
// end of each part.  The products are those of the dense float32 step
// (kernel_f32.h): K, V and Q go straight from memory to registers, a lane
// holding D / 4 consecutive elements of a key (query) row and D / 16 of each of
// four value rows.
//
// 8-bit rows are widened in registers.  A key's scale multiplies its score, a
// value's scale the value: powers of two, so neither rounds.
//
// What bounds it: for few rows the memory round trips and then the bytes of the
// pages (one token of 28 heads over 32768 keys 39 us; the next unit's keys and
// values are under way while this one is worked on, 44 us without), for many the
// float32 products (133 TFLOP/s in a large library product).
#pragma once

#include "kernel_mfma.h"
#include "paged_common.h"

namespace pdec {

struct fp8_t { uint8_t bits; };  // one e4m3 element of a cache row

// N consecutive cache elements of one row as raw words.
template <typename TC, int N>
struct PagedRaw {
    static constexpr int BYTES = N * (int)sizeof(TC), WORDS = BYTES / 4;
    uint32_t w[WORDS];
    __device__ inline void load(const unsigned char* p)
    {
        if constexpr (BYTES % 16 == 0) {
#pragma unroll
            for (int i = 0; i < WORDS / 4; ++i) {
                const u32x4_t x = reinterpret_cast<const u32x4_t*>(p)[i];
#pragma unroll
                for (int k = 0; k < 4; ++k) w[4 * i + k] = x[k];
            }
        } else {
#pragma unroll
            for (int i = 0; i < WORDS; ++i) w[i] = reinterpret_cast<const uint32_t*>(p)[i];
        }
    }
    __device__ inline float get(int i) const
    {
        if constexpr (sizeof(TC) == 4) return __uint_as_float(w[i]);
        else {
            const f32x2_t x = (i & 2) ? __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i >> 2], true)
                                      : __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i >> 2], false);
            return (i & 1) ? x.y : x.x;
        }
    }
};

__device__ inline f32x4_t paged_mfma4(float a, float b, f32x4_t c)
{
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

template <int D, int NT, typename TC>
__global__ __launch_bounds__(256, NT == 1 || D == 64 ? 2 : 1) void paged_f32_kernel(PagedArgs a)
{
    constexpr int NW = 4, RT = 16 * NT;
    constexpr int KPL = D / 4;   // elements of a key (query) row per lane
    constexpr int DT = D / 16;   // 16-wide d tiles
    constexpr int OROW = D + 4;  // row pitch of the merge buffer, in floats
    constexpr int ESZ = (int)sizeof(TC);
    constexpr bool SCALED = sizeof(TC) == 1;
    __shared__ __attribute__((aligned(16))) float o_s[NW * RT * OROW];
    __shared__ float m_s[NW][RT], l_s[NW][RT];

    const int tid = threadIdx.x;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lane = tid & 63, l16 = lane & 15, lg = lane >> 4;
    PagedRun run;
    PagedPart part;
    if (!paged_begin(a, paged_worker(a, blockIdx.x), run, tid == 0)) return;
    const float c = a.qscale;
    const long rowb = (long)a.H_kv * D * ESZ;  // bytes of one token's row in a page

    while (paged_next(a, run, part)) {
        if (tid == 0) paged_note(a, run, part);
        const PagedSeq sq = part.seq;
        const int R = sq.n * a.G, row0 = part.group * RT, nrows = min(RT, R - row0);
        int seen[NT];  // keys that the lane's row sees; none for rows past the last
        float qv[NT][KPL];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int r = 16 * nt + l16, rr = row0 + min(r, nrows - 1);
            seen[nt] = r < nrows ? paged_seen(a, sq, rr / a.G) : 0;
            PagedRaw<float, KPL> x;
            x.load(static_cast<const unsigned char*>(a.q) + (paged_qrow(a, sq, part.head, rr) * D + KPL * lg) * 4);
#pragma unroll
            for (int j = 0; j < KPL; ++j) qv[nt][j] = x.get(j);
        }
        const int least = nrows == RT ? paged_seen(a, sq, row0 / a.G) : 0;  // keys that every row sees
        const int most = paged_seen(a, sq, (row0 + nrows - 1) / a.G);      // that some row sees

        f32x4_t o[NT][DT];
        float m_ref[NT], l_lane[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            m_ref[nt] = kMinRef;
            l_lane[nt] = 0.f;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) o[nt][dt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
        }

        PagedRaw<TC, KPL> kx;
        PagedRaw<TC, DT> vx[4];
        uint32_t ks = 0, vs = 0;  // scales of keys 4 lg .. 4 lg + 3
        // The wave's 16 keys of a unit are on one page.  Units none of whose keys a row
        // sees, and keys without a page, are passed over.
        const int32_t* table = a.block_table + (long)part.s * a.max_pages;
        auto next = [&](int u, int& page) {
            for (; u < part.u1; ++u) {
                const int t = u * kUnit + 16 * w;
                page = t < most ? paged_entry(table, min(t >> a.page_shift, a.max_pages - 1)) : -1;
                if ((uint32_t)page < (uint32_t)a.num_pages) break;
            }
            return u;
        };
        auto row_of = [&](int u, int page) { return ((long)page << a.page_shift) + ((u * kUnit + 16 * w) & ((1 << a.page_shift) - 1)); };
        auto scale_at = [&](int u, int page) {
            return (((long)page * a.H_kv + part.head) << a.page_shift) + ((u * kUnit + 16 * w) & ((1 << a.page_shift) - 1)) + 4 * lg;
        };
        auto load_k = [&](int u, int page) {
            kx.load(static_cast<const unsigned char*>(a.k_pages) + (row_of(u, page) + l16) * rowb + ((long)part.head * D + KPL * lg) * ESZ);
            if constexpr (SCALED) ks = *reinterpret_cast<const uint32_t*>(a.k_scales + scale_at(u, page));
        };
        auto load_v = [&](int u, int page) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                vx[i].load(static_cast<const unsigned char*>(a.v_pages) + (row_of(u, page) + 4 * lg + i) * rowb + ((long)part.head * D + DT * l16) * ESZ);
            if constexpr (SCALED) vs = *reinterpret_cast<const uint32_t*>(a.v_scales + scale_at(u, page));
        };
        int page = -1, u = next(part.u0, page);
        if (u < part.u1) {
            load_k(u, page);
            load_v(u, page);
        }
        while (u < part.u1) {
            const int t = u * kUnit + 16 * w;
            const uint32_t ksc = ks;
            f32x4_t s[NT], s1[NT];  // two sums where there is one tile: the products of a sum wait for each other
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) s[nt] = s1[nt] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int j = 0; j < KPL; ++j)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    if (NT == 1 && (j & 1)) s1[nt] = paged_mfma4(kx.get(j), qv[nt][j], s1[nt]);
                    else s[nt] = paged_mfma4(kx.get(j), qv[nt][j], s[nt]);
                }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
                if (NT == 1) s[nt] += s1[nt];
            u = next(u + 1, page);
            if (u < part.u1) load_k(u, page);  // under this unit's softmax and P V
            float p[NT][4], mx[NT], vf[4][DT];
            const bool all_see = t + 16 <= least;
            bool need = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float x = SCALED ? s[nt][i] * paged_scale(ksc, i) : s[nt][i];
                    p[nt][i] = t + 4 * lg + i < seen[nt] ? x : kNegInf;
                }
                mx[nt] = fmaxf(fmaxf(p[nt][0], p[nt][1]), fmaxf(p[nt][2], p[nt][3]));
                need |= mx[nt] * c > m_ref[nt] + 8.f;
            }
            if (__any(need)) {  // rare after a row's first keys
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const float mt = max_over_groups(mx[nt]) * c;
                    const bool up = mt > m_ref[nt] + 8.f;
                    const float alpha = up ? fast_exp2(m_ref[nt] - mt) : 1.f;
                    m_ref[nt] = up ? mt : m_ref[nt];
                    l_lane[nt] *= alpha;
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) o[nt][dt] *= alpha;
                }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    p[nt][i] = fast_exp2(fmaf(p[nt][i], c, -m_ref[nt]));  // 0 for a hidden key
                    l_lane[nt] += p[nt][i];
                }
            // 0 times an infinite or NaN value is NaN.  Where some row does not see
            // all of the block, such values are left out of the products and then
            // added key by key to the rows that see the key.
            bool odd = false;
            auto strange = [](float x) { return (__float_as_uint(x) & 0x7f800000u) == 0x7f800000u; };
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float sc = SCALED ? paged_scale(vs, i) : 1.f;
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) {
                    vf[i][dt] = SCALED ? vx[i].get(dt) * sc : vx[i].get(dt);
                    if (!all_see) odd |= strange(vf[i][dt]);
                }
            }
            // 8-bit values have been widened into other registers: the next ones come
            // under the products, float32 ones under the next scores
            if (SCALED && u < part.u1) load_v(u, page);
            auto products = [&]() {
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) o[nt][dt] = paged_mfma4(vf[i][dt], p[nt][i], o[nt][dt]);
            };
            if (!__any(odd)) {
                products();
            } else {
                float vo[4][DT];
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int dt = 0; dt < DT; ++dt) {
                        vo[i][dt] = strange(vf[i][dt]) ? vf[i][dt] : 0.f;
                        vf[i][dt] = strange(vf[i][dt]) ? 0.f : vf[i][dt];
                    }
                products();
#pragma unroll 1
                for (int q = 0; q < 4; ++q)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const bool mine = lg == q;
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            const bool sees = t + 4 * q + i < seen[nt];
#pragma unroll
                            for (int dt = 0; dt < DT; ++dt) {
                                const f32x4_t x = paged_mfma4(mine ? vo[i][dt] : 0.f, mine ? p[nt][i] : 0.f, o[nt][dt]);
#pragma unroll
                                for (int k = 0; k < 4; ++k) o[nt][dt][k] = sees ? x[k] : o[nt][dt][k];
                            }
                        }
                    }
            }
            if (!SCALED && u < part.u1) load_v(u, page);
        }

        // ---- merge of the four waves; lane: row l % 16 of tile nt, d = D/4 (l / 16) + DT j + dt ----
        __syncthreads();  // the last part's states have been read
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float l = l_lane[nt];
            l += __shfl_xor(l, 16);
            l += __shfl_xor(l, 32);
            const int r = 16 * nt + l16;
            if (lg == 0) {
                m_s[w][r] = m_ref[nt];
                l_s[w][r] = l;
            }
            float* dst = o_s + (w * RT + r) * OROW + KPL * lg;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int dt = 0; dt < DT; ++dt) dst[DT * j + dt] = o[nt][dt][j];
        }
        __syncthreads();
        for (int i = tid; i < nrows * (D / 4); i += 256) {
            const int r = i / (D / 4), d4 = i % (D / 4);
            float M = m_s[0][r];
#pragma unroll
            for (int x = 1; x < NW; ++x) M = fmaxf(M, m_s[x][r]);
            float L = 0.f;
            f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int x = 0; x < NW; ++x) {
                const float f = fast_exp2(m_s[x][r] - M);  // 0 for a wave that saw none of the row's keys
                L += f * l_s[x][r];
                acc += f * *reinterpret_cast<const f32x4_t*>(o_s + (x * RT + r) * OROW + 4 * d4);
            }
            if (!part.whole) {
                const long at = (long)part.slot * RT + r;
                *reinterpret_cast<f32x4_t*>(a.part_o + at * D + 4 * d4) = acc;
                if (d4 == 0) *reinterpret_cast<float2*>(a.part_ml + 2 * at) = make_float2(M, L);
                continue;
            }
            const long qr = paged_qrow(a, sq, part.head, row0 + r);
            const float inv = L > 0.f || L != L ? 1.f / L : 0.f;
            acc *= inv;
            *reinterpret_cast<f32x4_t*>(static_cast<float*>(a.out) + qr * D + 4 * d4) = acc;
            if (d4 == 0 && a.lse) a.lse[qr] = L > 0.f || L != L ? kLn2 * (M + log2f(L)) : kNegInf;
        }
    }
}

}  // namespace pdec
