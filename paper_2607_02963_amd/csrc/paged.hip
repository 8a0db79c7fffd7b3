// C ABI of the paged caches (include/pdec.h): argument checks, the plan of an
// attention call, and the launches of kernel_paged_*.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "pdec.h"

#include "kernel_paged_f32.h"
#include "kernel_paged_finish.h"
#include "kernel_paged_io.h"
#include "paged_host.h"

namespace pdec {

namespace {

template <int D, typename TC>
void launch_f32_rows(const PagedArgs& a, hipStream_t s)
{
    const dim3 grid((unsigned)a.blocks), block(256);
    if (a.rows == 16) hipLaunchKernelGGL((paged_f32_kernel<D, 1, TC>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((paged_f32_kernel<D, 2, TC>), grid, block, 0, s, a);
}

}  // namespace

void launch_paged_f32(const PagedArgs& a, int head_dim, bool fp8, hipStream_t s)
{
    if (head_dim == 128) fp8 ? launch_f32_rows<128, fp8_t>(a, s) : launch_f32_rows<128, float>(a, s);
    else fp8 ? launch_f32_rows<64, fp8_t>(a, s) : launch_f32_rows<64, float>(a, s);
}

namespace {

template <int D, typename T>
void launch_finish(const PagedArgs& a, hipStream_t s)
{
    const int pairs = a.H_kv / a.heads * a.num_seqs * a.groups;
    const int rows = a.heads * (int)std::min<long>(a.rows, (long)a.max_chunk * a.G);
    const unsigned x = (unsigned)(a.by_pair ? pairs : a.workers);
    // States per pair, if all work-groups have work: a row's waves share them.  Sixteen
    // waves a row where the rows leave compute units free (28 rows of 64 states: a call
    // of 23.6 us to 21.9), four where there are many (896 rows: 9.2 us, sixteen 13.7).
    const int states = a.workers / pairs;
    if (states >= 32 && pairs * rows <= 256) hipLaunchKernelGGL((paged_finish_kernel<D, T, 16>), dim3(x, (unsigned)rows), dim3(1024), 0, s, a);
    else if (states >= 8) hipLaunchKernelGGL((paged_finish_kernel<D, T, 4>), dim3(x, (unsigned)rows), dim3(256), 0, s, a);
    else {
        constexpr int RPB = FinishCfg<D, 1>::RPB;
        hipLaunchKernelGGL((paged_finish_kernel<D, T, 1>), dim3(x, (unsigned)((rows + RPB - 1) / RPB)), dim3(256), 0, s, a);
    }
}

}  // namespace

void launch_paged_finish(const PagedArgs& a, int head_dim, int dtype, hipStream_t s)
{
    const bool f32 = dtype == PDEC_DTYPE_F32;
    if (head_dim == 128) f32 ? launch_finish<128, float>(a, s) : launch_finish<128, uint16_t>(a, s);
    else f32 ? launch_finish<64, float>(a, s) : launch_finish<64, uint16_t>(a, s);
}

}  // namespace pdec

namespace {

using namespace pdec;

int chunk_bound(const pdec_paged_dims* d) { return d->max_chunk > 0 ? std::min(d->max_chunk, d->num_tokens) : d->num_tokens; }
// Sequences of at most so many rows per kv head are the few-row kernel's: up to two
// 16-row tiles at D = 128, four at D = 64 (both sides measured: kernel_paged_few.h);
// three at D = 128 over 4-bit pages (kernel_paged_few4.h).
int few_rows(const pdec_paged_dims* d) { return d->head_dim == 64 ? 64 : d->cache_dtype == PDEC_DTYPE_E2M1 ? 48 : 32; }

struct AttnPlan {
    PagedArgs few{}, many{};
    bool use_few = false, use_many = false;
    size_t few_bytes = 0, many_bytes = 0;
};

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// Where no pair has more units than this nothing is cut, a work-group takes a pair
// and there is no finish pass.  Whole and cut, one token over 60 to 250 bfloat16 keys
// 11 and 15 us, 32 tokens over 8-bit pages 12 and 15, 8 chunks of 60 18-25 and 25-33.
// Above, few pairs of a long axis want cutting (one float32 token over 1000 keys 14 us,
// whole 22); 400 keys are as well or better whole (14 and 11 us, 36 and 28).
constexpr int kWholeUnits = 4;

// The division of one launch's work over `workers` work-groups (paged_common.h: `least`
// and `pad` in positions, of which a unit is `price` at most), and its workspace bytes;
// false if its count of positions passes 32 bits.
bool divide(const pdec_paged_dims* d, PagedArgs& a, int workers, int least, int pad, int price, size_t* bytes)
{
    const int64_t R = (int64_t)a.max_chunk * a.G;
    if (R > INT32_MAX / 2) return false;
    a.groups = (int)((std::min<int64_t>(R, a.rows_to) + a.rows - 1) / a.rows);
    const int64_t units = (a.max_len + kUnit - 1) / kUnit;
    const int64_t real_groups = (int64_t)d->num_tokens * a.G / a.rows + d->num_seqs;  // at most, over the batch
    // (the number of groups passes 2^50 for sizes that no tensor has: no product with it)
    if (real_groups > INT32_MAX / 2 / a.H_kv / (units * price + pad + 1)) return false;
    const int64_t pairs = (int64_t)d->num_seqs * a.groups * (a.H_kv / a.heads);
    if (pairs > INT32_MAX / 2) return false;
    a.workers = workers;
    a.least = least;
    a.pad = pad;
    a.whole = units <= kWholeUnits ? 1 : 0;
    a.by_pair = pairs <= workers ? 1 : 0;
    a.blocks = a.whole ? (int)((pairs + 7) / 8 * 8) : workers;
    if ((int64_t)a.blocks * 512 > UINT32_MAX) return false;  // threads of the launch
    *bytes = 0;
    if (!a.whole)
        *bytes = align256((size_t)workers * sizeof(int4)) + align256((size_t)2 * workers * a.heads * a.rows * 2 * sizeof(float)) +
                 (size_t)2 * workers * a.heads * a.rows * d->head_dim * sizeof(float);
    return true;
}

void place(PagedArgs& a, char* ws)
{
    if (a.whole) return;
    a.cut = reinterpret_cast<int4*>(ws);
    ws += align256((size_t)a.workers * sizeof(int4));
    a.part_ml = reinterpret_cast<float*>(ws);
    ws += align256((size_t)2 * a.workers * a.heads * a.rows * 2 * sizeof(float));
    a.part_o = reinterpret_cast<float*>(ws);
}

int plan_attn(const pdec_paged_dims* d, AttnPlan& p)
{
    const int rc = check_dims(d);
    if (rc != PDEC_OK) return rc;
    PagedArgs a{};
    a.num_seqs = d->num_seqs;
    a.num_tokens = d->num_tokens;
    a.H_q = d->num_q_heads;
    a.H_kv = d->num_kv_heads;
    a.G = d->num_q_heads / d->num_kv_heads;
    a.page_shift = shift_of(d->page_size);
    a.num_pages = d->num_pages;
    a.max_pages = d->max_pages;
    a.max_chunk = chunk_bound(d);
    a.max_len = len_bound(d);
    a.causal = d->causal;
    const float scale = d->softmax_scale > 0.f ? d->softmax_scale : 1.f / std::sqrt((float)d->head_dim);
    a.qscale = scale * 1.44269504088896340736f;
    const int64_t R = (int64_t)a.max_chunk * a.G;
    a.rows_from = 0;
    a.rows_to = INT32_MAX;
    a.heads = 1;
    p.few = p.many = a;
    p.use_many = d->dtype == PDEC_DTYPE_BF16 && R > few_rows(d);
    // One sequence is the many rows' whatever its chunk, and so are all where none has
    // more rows than a 128-row item: a second kernel and its finish pass cost more than
    // the rows left empty (24 sequences of 300 to 4000 keys, one of 16 new tokens and the
    // others of one 35.1 us, with both kernels 49.7; 1 to 16 tokens 42.9 and 61.1).  Over
    // 256-row items each goes by its own.
    p.use_few = !p.use_many || (d->num_seqs > 1 && R > 128);
    if (p.use_many) {
        // two 32-row tiles in each wave: a key read from LDS meets twice the rows
        p.many.rows = R <= 128 ? 128 : 256;
        if (p.use_few) {
            p.many.rows_from = few_rows(d) + 1;
            p.few.rows_to = few_rows(d);
        }
        // a work-group per compute unit; a start's price was swept (six chunks of 301 to 1023
        // tokens, 8-bit and bfloat16: 3 526 and 480 us, 6 456 and 418, 9 464 and 421, 14 471 and 424)
        if (!divide(d, p.many, 256, 4, 6, 1, &p.many_bytes)) return PDEC_ERR_UNSUPPORTED;
    }
    if (p.use_few) {
        const int64_t most = std::min<int64_t>(R, p.few.rows_to);
        const bool f32 = d->dtype == PDEC_DTYPE_F32, four = d->cache_dtype == PDEC_DTYPE_E2M1;
        p.few.rows = most <= 16 ? 16 : most <= 32 || f32 ? 32 : most <= 48 ? 48 : 64;
        if (f32 && four && d->head_dim == 128) p.few.rows = 16;  // the registers of three terms (kernel_paged_few4.h)
        // heads' rows of a cache line or half of one: two heads to a work-group (kernel_paged_few.h)
        if (!f32 && !four && (d->cache_dtype == PDEC_DTYPE_E4M3 || d->head_dim == 64) && a.H_kv % 2 == 0) p.few.heads = 2;
        // a start's price, in positions; over 4-bit pages, whose units are the shortest, it was swept.  Units of
        // one tile (4, 8, 16, 24, 32): 32 tokens over 1200 to 16384 keys, heads of 128, 44.2, 42.7, 40.5, 41.1,
        // 41.3 us; heads of 64 (8, 16, 24, 32, 48): 20 tokens over 1000 to 8000 keys 23.7, 22.0, 21.7, 22.4, 23.8, 40
        // over 2000 to 30000 79, 77, 76, 76, 75.6, and of five batches more all within 3% of their best at 24.  Items of more rows, whose units are 3 positions and up (paged_price; 36, 48, 72, 96): 2 to 9
        // drafted tokens of 13 sequences, heads of 64, -, 25.9, 24.7, 25.7, 1 to 4 of 32 sequences, heads of 128,
        // 47.7, 47.1, 45.9, - (units alike, at the best price: 25.5, 49.1)
        const bool weighed = four && p.few.rows > 16;
        const int pad = weighed ? 72 : four ? (d->head_dim == 128 ? 16 : 24) : f32 ? 1 : 4, price = weighed ? 2 + p.few.rows / 16 : 1;
        if (!divide(d, p.few, f32 && !four ? 512 : 256, 2 * price, pad, price, &p.few_bytes)) return PDEC_ERR_UNSUPPORTED;
    }
    return PDEC_OK;
}

// What a caller is asked for, also where nothing is cut and nothing is stored.
size_t workspace_of(const AttnPlan& p) { return std::max<size_t>(align256(p.few_bytes) + p.many_bytes, 16); }

// Tokens from which a wave of the append takes four: 16384 tokens of 4 heads of 128 took
// 15.3 us by one and take 12.0; up to 4096 both take the call's own 8.9.
constexpr int kAppendMany = 2048;
// Dense bytes from which the rows of a 4-bit cache, four times its own bytes, pass the caches by.  They
// are read back to be read: with readers of both tensors behind, in a graph, kept and past the caches: 1000
// rows of 4 heads of 128 (2 MB) 7.8 and 8.0 us, 5000 to 12000 alike, 16000 (33 MB) 21.0 and 22.7, 24000 (49 MB)
// 28.9 and 31.3, 30000 37.5 and 37.6, 60000 70.3 and 67.6.  By themselves 5000 5.1 and 4.3, 16000 8.9 and 7.6,
// 30000 14.3 and 13.5, 60000 28.9 and 24.6 (30700 with 7600 appended before 25.5 and 21.4).
constexpr int64_t kReadOnce = 48 << 20;
constexpr int kReadRows = 4;  // rows per wave of the read-back (32768 rows: 24.2 us, by 8 26.8, by 16 25.7)

template <int D, typename T, PagedForm FORM, int N>
void launch_append(const PagedIoArgs& a, hipStream_t s)
{
    const dim3 grid((unsigned)std::max((a.num_tokens + 4 * N - 1) / (4 * N), (a.num_seqs + 63) / 64), 2);
    hipLaunchKernelGGL((paged_append_kernel<D, T, FORM, N>), grid, dim3(256), 0, s, a);
}

template <int D, typename T, PagedForm FORM>
void launch_read(const PagedIoArgs& a, hipStream_t s)
{
    const dim3 grid((unsigned)((a.num_tokens + 4 * kReadRows - 1) / (4 * kReadRows)), 2);
    const int64_t bytes = 2 * (int64_t)a.num_tokens * a.H_kv * D * (int64_t)sizeof(T);
    if constexpr (FORM == kE2m1Rows) {
        if (bytes > kReadOnce) {
            hipLaunchKernelGGL((paged_read_kernel<D, T, FORM, kReadRows, true>), grid, dim3(256), 0, s, a);
            return;
        }
    }
    hipLaunchKernelGGL((paged_read_kernel<D, T, FORM, kReadRows, false>), grid, dim3(256), 0, s, a);
}

}  // namespace

extern "C" {

int pdec_check_paged_lengths(const pdec_paged_dims* d, const int32_t* cu, const int32_t* seq_lens, int32_t attn)
{
    const int rc = check_dims(d);
    if (rc != PDEC_OK) return rc;
    if (!cu || !seq_lens) return PDEC_ERR_INVALID_ARG;
    if (cu[0] != 0 || cu[d->num_seqs] > d->num_tokens) return PDEC_ERR_BAD_LENGTHS;
    for (int s = 0; s < d->num_seqs; ++s) {
        if (cu[s + 1] < cu[s] || seq_lens[s] < 0 || seq_lens[s] > len_bound(d)) return PDEC_ERR_BAD_LENGTHS;
        if (attn && cu[s + 1] - cu[s] > chunk_bound(d)) return PDEC_ERR_BAD_LENGTHS;
    }
    return PDEC_OK;
}

int pdec_paged_kv_append(const pdec_paged_dims* d, const void* k_new, const void* v_new, const int32_t* cu_tokens,
                         const int32_t* block_table, const int32_t* lens_in, int32_t* lens_out, void* k_pages,
                         void* v_pages, uint8_t* k_scales, uint8_t* v_scales, void* stream)
{
    int rc = check_dims(d);
    if (rc != PDEC_OK) return rc;
    if (!aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(cu_tokens, 4) || !aligned(block_table, 4) ||
        !aligned(lens_in, 4) || !aligned(lens_out, 4) || lens_in == lens_out ||
        !cache_pointers(d, k_pages, v_pages, k_scales, v_scales))
        return PDEC_ERR_INVALID_ARG;
    if (debug_mode() && (rc = debug_check(d, cu_tokens, lens_in, 0, stream)) != PDEC_OK) return rc;
    PagedIoArgs a = io_args(d);
    a.k_rows = k_new;
    a.v_rows = v_new;
    a.k_pages = k_pages;
    a.v_pages = v_pages;
    a.k_scales = k_scales;
    a.v_scales = v_scales;
    a.block_table = block_table;
    a.cu = cu_tokens;
    a.lens = lens_in;
    a.lens_out = lens_out;
    hipStream_t s = static_cast<hipStream_t>(stream);
    for_types(d, [&](auto dim, auto t, auto q) { 
        if (a.num_tokens < kAppendMany) launch_append<dim(), decltype(t), q(), 1>(a, s);
        else launch_append<dim(), decltype(t), q(), 4>(a, s);
    });
    return launched();
}

int pdec_paged_kv_read(const pdec_paged_dims* d, const void* k_pages, const void* v_pages, const uint8_t* k_scales,
                       const uint8_t* v_scales, const int32_t* block_table, const int32_t* seq_lens,
                       const int32_t* cu_rows, void* k_out, void* v_out, void* stream)
{
    int rc = check_dims(d);
    if (rc != PDEC_OK) return rc;
    if (!aligned(k_out, 16) || !aligned(v_out, 16) || !aligned(cu_rows, 4) || !aligned(block_table, 4) ||
        !aligned(seq_lens, 4) || !cache_pointers(d, k_pages, v_pages, k_scales, v_scales))
        return PDEC_ERR_INVALID_ARG;
    if (debug_mode() && (rc = debug_check(d, cu_rows, seq_lens, 0, stream)) != PDEC_OK) return rc;
    PagedIoArgs a = io_args(d);
    a.k_rows = k_out;
    a.v_rows = v_out;
    a.k_pages = const_cast<void*>(k_pages);
    a.v_pages = const_cast<void*>(v_pages);
    a.k_scales = const_cast<uint8_t*>(k_scales);
    a.v_scales = const_cast<uint8_t*>(v_scales);
    a.block_table = block_table;
    a.cu = cu_rows;
    a.lens = seq_lens;
    hipStream_t s = static_cast<hipStream_t>(stream);
    for_types(d, [&](auto dim, auto t, auto q) { launch_read<dim(), decltype(t), q()>(a, s); });
    return launched();
}

size_t pdec_paged_workspace_size(const pdec_paged_dims* d)
{
    AttnPlan p;
    return plan_attn(d, p) == PDEC_OK ? workspace_of(p) : 0;
}

int pdec_query_paged_plan(const pdec_paged_dims* d, pdec_paged_plan* plan)
{
    if (!plan) return PDEC_ERR_INVALID_ARG;
    AttnPlan p;
    const int rc = plan_attn(d, p);
    if (rc != PDEC_OK) return rc;
    plan->rows_few = p.use_few ? p.few.rows : 0;
    plan->rows_many = p.use_many ? p.many.rows : 0;
    plan->workers = p.use_few ? p.few.workers : p.many.workers;
    plan->merge_pass = (p.use_few && !p.few.whole) || (p.use_many && !p.many.whole) ? 1 : 0;
    return PDEC_OK;
}

int pdec_paged_attn(const pdec_paged_dims* d, const void* q, const void* k_pages, const void* v_pages,
                    const uint8_t* k_scales, const uint8_t* v_scales, const int32_t* block_table,
                    const int32_t* cu_tokens, const int32_t* seq_lens, void* out, float* lse, void* workspace,
                    size_t workspace_bytes, void* stream)
{
    AttnPlan p;
    int rc = plan_attn(d, p);
    if (rc != PDEC_OK) return rc;
    if (!aligned(q, 16) || !aligned(out, 16) || (lse && !aligned(lse, 4)) || !aligned(block_table, 4) ||
        !aligned(cu_tokens, 4) || !aligned(seq_lens, 4) || !aligned(workspace, 16) ||
        !cache_pointers(d, k_pages, v_pages, k_scales, v_scales))
        return PDEC_ERR_INVALID_ARG;
    if (workspace_bytes < workspace_of(p)) return PDEC_ERR_WORKSPACE;
    if (debug_mode() && (rc = debug_check(d, cu_tokens, seq_lens, 1, stream)) != PDEC_OK) return rc;
    hipStream_t s = static_cast<hipStream_t>(stream);
    for (PagedArgs* a : {&p.few, &p.many}) {
        a->q = q;
        a->k_pages = k_pages;
        a->v_pages = v_pages;
        a->k_scales = k_scales;
        a->v_scales = v_scales;
        a->block_table = block_table;
        a->cu_tokens = cu_tokens;
        a->seq_lens = seq_lens;
        a->out = out;
        a->lse = lse;
    }
    char* const ws = static_cast<char*>(workspace);
    auto finish = [&](const PagedArgs& a) {
        if (!a.whole) launch_paged_finish(a, d->head_dim, d->dtype, s);
        return launched();
    };
    if (p.use_many) {
        place(p.many, ws + align256(p.few_bytes));
        launch_paged_rows(p.many, d->head_dim, d->cache_dtype, s);
        if ((rc = launched()) != PDEC_OK || (rc = finish(p.many)) != PDEC_OK) return rc;
    }
    if (p.use_few) {
        place(p.few, ws);
        const bool fp8 = d->cache_dtype == PDEC_DTYPE_E4M3, f32 = d->dtype == PDEC_DTYPE_F32;
        if (d->cache_dtype == PDEC_DTYPE_E2M1) launch_paged_few4(p.few, d->head_dim, f32, s);
        else if (f32) launch_paged_f32(p.few, d->head_dim, fp8, s);
        else launch_paged_few(p.few, d->head_dim, fp8, s);
        if ((rc = launched()) != PDEC_OK || (rc = finish(p.few)) != PDEC_OK) return rc;
    }
    return PDEC_OK;
}

int pdec_merge_states(int64_t num_rows, int32_t head_dim, int32_t dtype, const void* out_a, const float* lse_a,
                      const void* out_b, const float* lse_b, void* out, float* lse, void* stream)
{
    if (num_rows < 1 || !aligned(out_a, 16) || !aligned(out_b, 16) || !aligned(out, 16) || !aligned(lse_a, 4) ||
        !aligned(lse_b, 4) || (lse && !aligned(lse, 4)))
        return PDEC_ERR_INVALID_ARG;
    if (dtype != PDEC_DTYPE_F32 && dtype != PDEC_DTYPE_BF16) return PDEC_ERR_UNSUPPORTED;
    if (head_dim != 64 && head_dim != 128) return PDEC_ERR_UNSUPPORTED;
    const int64_t blocks = (std::min<int64_t>(num_rows, (int64_t)1 << 33) * (head_dim / 8) + 255) / 256;
    if (num_rows > ((int64_t)1 << 32) || blocks * 256 > UINT32_MAX) return PDEC_ERR_UNSUPPORTED;  // threads of the launch
    const dim3 grid((unsigned)blocks), block(256);
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool f32 = dtype == PDEC_DTYPE_F32;
    if (head_dim == 128) {
        if (f32) hipLaunchKernelGGL((merge_states_kernel<128, float>), grid, block, 0, s, (long)num_rows, out_a, lse_a, out_b, lse_b, out, lse);
        else hipLaunchKernelGGL((merge_states_kernel<128, uint16_t>), grid, block, 0, s, (long)num_rows, out_a, lse_a, out_b, lse_b, out, lse);
    } else {
        if (f32) hipLaunchKernelGGL((merge_states_kernel<64, float>), grid, block, 0, s, (long)num_rows, out_a, lse_a, out_b, lse_b, out, lse);
        else hipLaunchKernelGGL((merge_states_kernel<64, uint16_t>), grid, block, 0, s, (long)num_rows, out_a, lse_a, out_b, lse_b, out, lse);
    }
    return launched();
}

}  // extern "C"
