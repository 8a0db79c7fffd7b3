// Address/undefined-behaviour sanitizer run of the paged calls' host logic: dims
// checks, plan, workspace size and length check over random and extreme sizes, and
// the refusals of every launching call.  Nothing here reaches a launch: each call
// gets an argument that the library refuses first.  Exit status 0: no error.
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

static void* fake(int n) { return reinterpret_cast<void*>((uintptr_t)0x100000 * n); }

int main()
{
    std::mt19937 rng(5);
    const int32_t sizes[] = {-1, 0, 1, 2, 3, 7, 28, 64, 1000, 1 << 16, 1 << 20, (1 << 27) - 1, 1 << 27, (1 << 27) + 1, 1 << 30, INT32_MAX, INT32_MIN};
    auto any = [&](int small) { return (rng() % 4) ? (int32_t)(1 + rng() % small) : sizes[rng() % (sizeof(sizes) / sizeof(sizes[0]))]; };
    int good = 0;
    for (int i = 0; i < 200000; ++i) {
        pdec_paged_dims d;
        std::memset(&d, 0, sizeof(d));
        d.num_seqs = any(100);
        d.num_tokens = any(5000);
        d.num_kv_heads = any(8);
        d.num_q_heads = (rng() % 8) ? (int32_t)((int64_t)d.num_kv_heads * (1 + rng() % 16) & INT32_MAX) : any(64);
        d.head_dim = (rng() % 8) ? 64 << (rng() % 2) : any(256);
        d.page_size = (rng() % 8) ? 16 << (rng() % 7) : any(2048);
        d.num_pages = any(10000);
        d.max_pages = any(1000);
        d.max_chunk = rng() % 2 ? 0 : any(5000);
        d.max_len = rng() % 2 ? 0 : any(20000);
        d.dtype = (int32_t)(rng() % (rng() % 8 ? 2 : 4));
        d.cache_dtype = rng() % 2 ? d.dtype : rng() % 8 ? (int32_t)PDEC_DTYPE_E4M3 : (int32_t)(rng() % 4);
        d.causal = (int32_t)(rng() % 3);
        d.softmax_scale = rng() % 2 ? 0.f : 0.1f;
        const size_t bytes = pdec_paged_workspace_size(&d);
        pdec_paged_plan plan;
        CHECK((bytes > 0) == (pdec_query_paged_plan(&d, &plan) == PDEC_OK));
        int32_t cu[2] = {0, 1}, lens[1] = {1};
        if (d.num_seqs == 1) {
            const int rc = pdec_check_paged_lengths(&d, cu, lens, (int)(rng() % 2));
            CHECK(bytes == 0 || rc == PDEC_OK);
        }
        if (bytes) {
            ++good;
            CHECK(bytes < (size_t)1 << 30);
            CHECK(plan.rows_few || plan.rows_many);
            CHECK(pdec_paged_attn(&d, fake(1), fake(2), fake(3), (uint8_t*)fake(4), (uint8_t*)fake(5), (int32_t*)fake(6),
                                  (int32_t*)fake(7), (int32_t*)fake(8), fake(9), (float*)fake(10), fake(11), bytes - 1,
                                  nullptr) == PDEC_ERR_WORKSPACE || bytes == 16);
        }
        CHECK(pdec_paged_attn(&d, nullptr, fake(2), fake(3), (uint8_t*)fake(4), (uint8_t*)fake(5), (int32_t*)fake(6),
                              (int32_t*)fake(7), (int32_t*)fake(8), fake(9), nullptr, fake(11), bytes, nullptr) != PDEC_OK);
        CHECK(pdec_paged_kv_append(&d, nullptr, fake(2), (int32_t*)fake(3), (int32_t*)fake(4), (int32_t*)fake(5),
                                   (int32_t*)fake(6), fake(7), fake(8), (uint8_t*)fake(9), (uint8_t*)fake(10), nullptr) != PDEC_OK);
        CHECK(pdec_paged_kv_read(&d, fake(1), fake(2), (uint8_t*)fake(3), (uint8_t*)fake(4), (int32_t*)fake(5),
                                 (int32_t*)fake(6), (int32_t*)fake(7), nullptr, fake(9), nullptr) != PDEC_OK);
    }
    CHECK(good > 5000);
    CHECK(pdec_paged_workspace_size(nullptr) == 0 && pdec_query_paged_plan(nullptr, nullptr) == PDEC_ERR_INVALID_ARG);
    for (int64_t rows : {(int64_t)0, (int64_t)-1, INT64_MIN, INT64_MAX, (int64_t)1 << 40, ((int64_t)1 << 29) + 1})
        CHECK(pdec_merge_states(rows, 128, PDEC_DTYPE_BF16, fake(1), (float*)fake(2), fake(3), (float*)fake(4), fake(5), (float*)fake(6), nullptr) != PDEC_OK);
    std::printf("ok %d\n", good);
    return 0;
}
