// Address/undefined-behaviour sanitizer run of the host logic of block tables, rotary
// positions and the append with them, over random and extreme sizes, strides and
// specs.  Each launching call gets an argument that the library refuses.  Exit
// status 0: no error.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <random>

#include "pdec.h"

namespace pdec {
bool debug_mode() { return false; }
}  // namespace pdec

#define CHECK(c)                                                               \
    do {                                                                       \
        if (!(c)) {                                                            \
            std::fprintf(stderr, "check failed: %s (line %d)\n", #c, __LINE__); \
            return 1;                                                          \
        }                                                                      \
    } while (0)

template <typename T = int32_t>
static T* fake(int n) { return reinterpret_cast<T*>((uintptr_t)0x100000 * n); }

int main()
{
    std::mt19937 rng(7);
    const int32_t sizes[] = {-1, 0, 1, 2, 3, 7, 28, 64, 1000, 1 << 16, 1 << 20, (1 << 20) + 1, (1 << 27) - 1, 1 << 27, (1 << 27) + 1, 1 << 30, INT32_MAX, INT32_MIN};
    const int64_t strides[] = {0, -1, 1, 8, 128, 512, 4096, INT64_MAX, INT64_MIN, (int64_t)1 << 40, ((int64_t)1 << 33) + 8, -4096};
    const double reals[] = {0, -1, 1, 2.5, 1e4, 1e308, -1e308, 1e-320, NAN, INFINITY, -INFINITY};
    auto any = [&](int small) { return (rng() % 4) ? (int32_t)(1 + rng() % small) : sizes[rng() % (sizeof(sizes) / sizeof(sizes[0]))]; };
    auto real = [&](double usual) { return (rng() % 6) ? usual : reals[rng() % (sizeof(reals) / sizeof(reals[0]))]; };
    auto stride = [&](int64_t row) { return (rng() % 6) ? row : strides[rng() % (sizeof(strides) / sizeof(strides[0]))]; };
    int tables = 0;
    for (int i = 0; i < 200000; ++i) {
        pdec_table_dims d;
        d.num_seqs = any(100);
        d.num_tokens = any(5000);
        d.page_size = (rng() % 8) ? 16 << (rng() % 7) : any(2048);
        d.num_pages = any(10000);
        d.max_pages = any(1000);
        d.max_len = rng() % 2 ? 0 : any(20000);
        const size_t bytes = pdec_table_workspace_size(&d);
        if (bytes) {
            ++tables;
            CHECK(bytes <= (size_t)1 << 24 && bytes >= 8 * (size_t)d.num_seqs && bytes % 16 == 0);
            CHECK(pdec_paged_reserve(&d, fake(1), fake(2), fake(3), fake(4), fake(5), fake(6), fake(7), nullptr, nullptr, fake<void>(8), bytes - 1, nullptr) == PDEC_ERR_WORKSPACE);
            CHECK(pdec_paged_release(&d, nullptr, fake(2), fake(3), fake(4), fake(5), fake(6), fake<void>(8), bytes - 1, nullptr) == PDEC_ERR_WORKSPACE);
        }
        CHECK(pdec_paged_reserve(&d, nullptr, fake(2), fake(3), fake(4), fake(5), fake(6), fake(7), nullptr, nullptr, fake<void>(8), SIZE_MAX, nullptr) != PDEC_OK);
        CHECK(pdec_paged_release(&d, nullptr, nullptr, fake(3), fake(4), fake(5), fake(6), fake<void>(8), SIZE_MAX, nullptr) != PDEC_OK);

        pdec_rope_spec r;
        std::memset(&r, 0, sizeof(r));
        r.head_dim = (rng() % 8) ? 64 << (rng() % 2) : any(256);
        r.rotary_dim = (rng() % 8) ? 16 * (int32_t)(rng() % 9) : any(256);
        r.interleaved = (int32_t)(rng() % (rng() % 8 ? 2 : 4));
        r.scaling = (int32_t)(rng() % 6) - (rng() % 8 ? 0 : 1);
        r.theta = real(1e4);
        r.factor = real(4);
        r.original_len = real(4096);
        r.slow_turns = real(1);
        r.fast_turns = real(32);
        r.magnitude = real(0);
        r.freqs = rng() % 2 ? fake<double>(9) : nullptr;
        const int32_t dtype = (int32_t)(rng() % 4), hq = any(64), hk = rng() % 4 ? any(16) : 0;
        const int64_t D = r.head_dim, T = rng() % 8 ? any(10000) : strides[rng() % (sizeof(strides) / sizeof(strides[0]))];
        // positions missing: refused whatever the rest
        CHECK(pdec_rope(&r, T, hq, hk, dtype, (int32_t)(rng() % 3), nullptr, fake<void>(1), stride(hq * D), fake<void>(2), stride(hq * D), fake<void>(3), stride(hk * D), fake<void>(4), stride(hk * D), nullptr) != PDEC_OK);
        // rows without an output
        CHECK(pdec_rope(&r, T, hq, hk, dtype, 0, fake(5), fake<void>(1), stride(hq * D), nullptr, stride(hq * D), fake<void>(3), stride(hk * D), fake<void>(4), stride(hk * D), nullptr) != PDEC_OK);

        pdec_paged_dims p;
        std::memset(&p, 0, sizeof(p));
        p.num_seqs = any(100);
        p.num_tokens = any(5000);
        p.num_kv_heads = any(8);
        p.num_q_heads = (int32_t)((int64_t)p.num_kv_heads * (1 + rng() % 16) & INT32_MAX);
        p.head_dim = rng() % 8 ? r.head_dim : any(256);
        p.page_size = 16 << (rng() % 7);
        p.num_pages = any(10000);
        p.max_pages = any(1000);
        p.dtype = (int32_t)(rng() % 2);
        p.cache_dtype = rng() % 2 ? p.dtype : (int32_t)(rng() % 5);
        const int64_t q = (int64_t)p.num_q_heads * p.head_dim, k = (int64_t)p.num_kv_heads * p.head_dim;
        CHECK(pdec_paged_rope_kv_append(&p, &r, fake<void>(1), stride(q), fake<void>(2), stride(q), fake<void>(3), stride(k), fake<void>(4), stride(k), nullptr, fake(5), fake(6), fake(7), fake(7), fake<void>(8), fake<void>(9), fake<uint8_t>(10), fake<uint8_t>(11), nullptr) != PDEC_OK);
    }
    CHECK(tables > 5000);
    CHECK(pdec_table_workspace_size(nullptr) == 0);
    std::printf("ok %d\n", tables);
    return 0;
}
