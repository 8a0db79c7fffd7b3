// C ABI of what a serving step does around its paged cache (include/pdec.h): block
// tables, rotary positions, and the append with them.
#include <hip/hip_runtime.h>

#include "pdec.h"

#include "kernel_paged_rope.h"
#include "kernel_paged_table.h"
#include "paged_host.h"

namespace {

using namespace pdec;

// Sequences of a table call: its work-groups sum the counts of all before theirs.
constexpr int kMostTableSeqs = 1 << 20;

int check_table_dims(const pdec_table_dims* d)
{
    if (!d) return PDEC_ERR_INVALID_ARG;
    if (d->num_seqs < 1 || d->num_tokens < 1 || d->page_size < 1 || d->num_pages < 1 || d->max_pages < 1 || d->max_len < 0)
        return PDEC_ERR_INVALID_ARG;
    if (d->page_size < 16 || d->page_size > 1024 || (d->page_size & (d->page_size - 1)) != 0) return PDEC_ERR_UNSUPPORTED;
    if (d->num_tokens > kMostRows || d->num_seqs > kMostTableSeqs) return PDEC_ERR_UNSUPPORTED;
    const int64_t most = (int64_t)d->max_pages * d->page_size;
    if (most > ((int64_t)1 << 30)) return PDEC_ERR_UNSUPPORTED;
    if (d->max_len > most) return PDEC_ERR_INVALID_ARG;
    return PDEC_OK;
}

PagedTableArgs table_args(const pdec_table_dims* d)
{
    PagedTableArgs a{};
    a.num_seqs = d->num_seqs;
    a.num_tokens = d->num_tokens;
    a.page_shift = shift_of(d->page_size);
    a.num_pages = d->num_pages;
    a.max_pages = d->max_pages;
    a.max_len = d->max_len > 0 ? d->max_len : d->max_pages * d->page_size;
    return a;
}

// Chunks of sequences whose counts are summed by a pass of their own; 0: none are.  Reserving and
// releasing 2048 sequences takes 27 us without such a pass and 33 with it, 4096 51 and 45, 16384 354 and
// 117, 2^20 1.04 s and 6.5 ms: without it each work-group reads the counts of all before it.
constexpr int kTableTotals = kTableChunk;
int table_chunks(const pdec_table_dims* d) { return d->num_seqs > kTableTotals ? (d->num_seqs + kTableChunk - 1) / kTableChunk : 0; }
size_t table_counts(const pdec_table_dims* d) { return ((size_t)d->num_seqs + 1) / 2 * 2 * sizeof(int2); }

// One work-group keeps its sequences' counts to itself.
size_t table_workspace(const pdec_table_dims* d)
{
    return d->num_seqs <= kTableOne ? 0 : table_counts(d) + table_chunks(d) * sizeof(ulonglong2);
}

void table_place(PagedTableArgs& a, const pdec_table_dims* d, void* workspace)
{
    a.counts = static_cast<int2*>(workspace);
    a.totals = table_chunks(d) > 0 ? reinterpret_cast<ulonglong2*>(static_cast<char*>(workspace) + table_counts(d)) : nullptr;
}

template <bool RESERVE>
int launch_table(const PagedTableArgs& a, hipStream_t s)
{
    if (a.num_seqs <= kTableOne) {
        if (a.num_seqs <= 2 * kTableWaves) hipLaunchKernelGGL((paged_table_one_kernel<RESERVE, 2>), dim3(1), dim3(64 * kTableWaves), 0, s, a);
        else hipLaunchKernelGGL((paged_table_one_kernel<RESERVE, 4>), dim3(1), dim3(64 * kTableWaves), 0, s, a);
        return launched();
    }
    const dim3 grid((unsigned)((a.num_seqs + 3) / 4));
    hipLaunchKernelGGL((paged_table_count_kernel<RESERVE>), grid, dim3(256), 0, s, a);
    if (launched() != PDEC_OK) return PDEC_ERR_HIP;
    if (a.totals) {
        hipLaunchKernelGGL(paged_table_totals_kernel, dim3((unsigned)((a.num_seqs + kTableChunk - 1) / kTableChunk)), dim3(256), 0, s, a);
        if (launched() != PDEC_OK) return PDEC_ERR_HIP;
        hipLaunchKernelGGL((paged_table_kernel<RESERVE, true>), grid, dim3(256), 0, s, a);
    } else {
        hipLaunchKernelGGL((paged_table_kernel<RESERVE, false>), grid, dim3(256), 0, s, a);
    }
    return launched();
}

// The spec as the kernels take it, checked.
int rope_spec(const pdec_rope_spec* d, int backward, RopeSpec& r)
{
    if (!d || d->interleaved < 0 || d->interleaved > 1 || d->scaling < PDEC_ROPE_PLAIN || d->scaling > PDEC_ROPE_TABLE ||
        backward < 0 || backward > 1 || d->rotary_dim < 0)
        return PDEC_ERR_INVALID_ARG;
    if (d->head_dim != 64 && d->head_dim != 128) return PDEC_ERR_UNSUPPORTED;
    r = RopeSpec{};
    r.R = d->rotary_dim > 0 ? d->rotary_dim : d->head_dim;
    if (r.R > d->head_dim) return PDEC_ERR_INVALID_ARG;
    if (r.R % 16 != 0) return PDEC_ERR_UNSUPPORTED;
    auto positive = [](double x) { return x > 0 && std::isfinite(x); };
    const bool scaled = d->scaling == PDEC_ROPE_LINEAR || d->scaling == PDEC_ROPE_NTK || d->scaling == PDEC_ROPE_BY_PARTS;
    if (!std::isfinite(d->magnitude) || (scaled && !positive(d->factor))) return PDEC_ERR_INVALID_ARG;
    if (d->scaling == PDEC_ROPE_TABLE) {
        if (!aligned(d->freqs, 8)) return PDEC_ERR_INVALID_ARG;
        r.freqs = d->freqs;
    } else if (!positive(d->theta)) {
        return PDEC_ERR_INVALID_ARG;
    }
    r.interleaved = d->interleaved;
    r.back = backward;
    r.magnitude = d->magnitude != 0 ? d->magnitude : 1.0;
    r.log2_theta = d->scaling == PDEC_ROPE_TABLE ? 0.0 : std::log2(d->theta);
    if (d->scaling == PDEC_ROPE_NTK) r.log2_theta += std::log2(d->factor) * r.R / (r.R - 2.0);
    r.inv_factor = d->scaling == PDEC_ROPE_LINEAR || d->scaling == PDEC_ROPE_BY_PARTS ? 1.0 / d->factor : 1.0;
    if (d->scaling == PDEC_ROPE_BY_PARTS) {
        if (!positive(d->original_len) || !std::isfinite(d->slow_turns) || !std::isfinite(d->fast_turns) ||
            !(d->slow_turns < d->fast_turns))
            return PDEC_ERR_INVALID_ARG;
        r.by_parts = 1;
        r.turns_per_f = d->original_len * 0.15915494309189533577;  // 1 / 2 pi
        r.slow = d->slow_turns;
        r.inv_range = 1.0 / (d->fast_turns - d->slow_turns);
    }
    return PDEC_OK;
}

// A row's stride: whole 16 bytes, no shorter than the row.
bool row_stride(int64_t stride, int64_t elems, int dtype)
{
    return stride >= elems && stride % (dtype == PDEC_DTYPE_F32 ? 4 : 8) == 0 && stride <= INT64_MAX / 8 / kMostRows;
}

// Waves that share a token's heads: as many as fill the card where tokens are few.
int rope_split(int64_t tokens, int steps) { return (int)std::max<int64_t>(std::min<int64_t>(steps, 2048 / tokens), 1); }

// At least `groups` work-groups, in x and z: the threads in x stay within 32 bits.
constexpr int kRopeWide = 1 << 20;
dim3 rope_grid(int groups, int split)
{
    const int wide = std::min(groups, kRopeWide);
    return dim3((unsigned)wide, (unsigned)split, (unsigned)((groups + wide - 1) / wide));
}

}  // namespace

extern "C" {

size_t pdec_table_workspace_size(const pdec_table_dims* d) { return check_table_dims(d) == PDEC_OK ? table_workspace(d) : 0; }

int pdec_paged_reserve(const pdec_table_dims* d, const int32_t* new_tokens, const int32_t* seq_lens, int32_t* block_table,
                       const int32_t* free_pages, const int32_t* free_in, int32_t* free_out, int32_t* cu_tokens,
                       int32_t* positions, int64_t* slots, void* workspace, size_t workspace_bytes, void* stream)
{
    const int rc = check_table_dims(d);
    if (rc != PDEC_OK) return rc;
    if (!aligned(new_tokens, 4) || !aligned(seq_lens, 4) || !aligned(block_table, 4) || !aligned(free_pages, 4) ||
        !aligned(free_in, 4) || !aligned(free_out, 4) || free_in == free_out || !aligned(cu_tokens, 4) ||
        (positions && !aligned(positions, 4)) || (slots && !aligned(slots, 8)) || (table_workspace(d) > 0 && !aligned(workspace, 16)))
        return PDEC_ERR_INVALID_ARG;
    if (workspace_bytes < table_workspace(d)) return PDEC_ERR_WORKSPACE;
    PagedTableArgs a = table_args(d);
    a.first = new_tokens;
    a.lens = seq_lens;
    a.block_table = block_table;
    a.free_pages = const_cast<int32_t*>(free_pages);
    a.free_in = free_in;
    a.free_out = free_out;
    a.cu = cu_tokens;
    a.positions = positions;
    a.slots = slots;
    table_place(a, d, workspace);
    return launch_table<true>(a, static_cast<hipStream_t>(stream));
}

int pdec_paged_release(const pdec_table_dims* d, const int32_t* keep_from, const int32_t* keep_len, int32_t* block_table,
                       int32_t* free_pages, const int32_t* free_in, int32_t* free_out, void* workspace,
                       size_t workspace_bytes, void* stream)
{
    const int rc = check_table_dims(d);
    if (rc != PDEC_OK) return rc;
    if ((keep_from && !aligned(keep_from, 4)) || !aligned(keep_len, 4) || !aligned(block_table, 4) || !aligned(free_pages, 4) ||
        !aligned(free_in, 4) || !aligned(free_out, 4) || free_in == free_out || (table_workspace(d) > 0 && !aligned(workspace, 16)))
        return PDEC_ERR_INVALID_ARG;
    if (workspace_bytes < table_workspace(d)) return PDEC_ERR_WORKSPACE;
    PagedTableArgs a = table_args(d);
    a.first = keep_from;
    a.lens = keep_len;
    a.block_table = block_table;
    a.free_pages = free_pages;
    a.free_in = free_in;
    a.free_out = free_out;
    table_place(a, d, workspace);
    return launch_table<false>(a, static_cast<hipStream_t>(stream));
}

int pdec_rope(const pdec_rope_spec* spec, int64_t num_tokens, int32_t num_q_heads, int32_t num_k_heads, int32_t dtype,
              int32_t backward, const int32_t* positions, const void* q, int64_t q_stride, void* q_out,
              int64_t q_out_stride, const void* k, int64_t k_stride, void* k_out, int64_t k_out_stride, void* stream)
{
    RopeRowsArgs a{};
    const int rc = rope_spec(spec, backward, a.spec);
    if (rc != PDEC_OK) return rc;
    const int D = spec->head_dim;
    if (num_tokens < 1 || num_q_heads < 1 || num_k_heads < 0 || !aligned(positions, 4)) return PDEC_ERR_INVALID_ARG;
    if (dtype != PDEC_DTYPE_F32 && dtype != PDEC_DTYPE_BF16) return PDEC_ERR_UNSUPPORTED;
    if (num_tokens > kMostRows || num_q_heads > (1 << 20) || num_k_heads > (1 << 20)) return PDEC_ERR_UNSUPPORTED;
    auto rows = [&](int i, const void* in, int64_t in_stride, void* out, int64_t out_stride, int heads) {
        if (heads > 0 && (!aligned(in, 16) || !aligned(out, 16) || !row_stride(in_stride, (int64_t)heads * D, dtype) ||
                          !row_stride(out_stride, (int64_t)heads * D, dtype) || (in == out && in_stride != out_stride)))
            return false;
        a.in[i] = in;
        a.out[i] = out;
        a.in_stride[i] = in_stride;
        a.out_stride[i] = out_stride;
        a.heads[i] = heads;
        return true;
    };
    if (!rows(0, q, q_stride, q_out, q_out_stride, num_q_heads) || !rows(1, k, k_stride, k_out, k_out_stride, num_k_heads))
        return PDEC_ERR_INVALID_ARG;
    a.positions = positions;
    a.num_tokens = (int)num_tokens;
    const int per = 64 * 32 / (D * (dtype == PDEC_DTYPE_F32 ? 4 : 2));  // heads of a wave at a time
    a.split = rope_split(num_tokens, (num_q_heads + per - 1) / per + (num_k_heads + per - 1) / per);
    const dim3 grid = rope_grid(((int)num_tokens + 3) / 4, a.split), block(256);
    a.wide = (int)grid.x;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool f32 = dtype == PDEC_DTYPE_F32;
    if (D == 128) {
        if (f32) hipLaunchKernelGGL((rope_rows_kernel<128, float>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((rope_rows_kernel<128, uint16_t>), grid, block, 0, s, a);
    } else {
        if (f32) hipLaunchKernelGGL((rope_rows_kernel<64, float>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((rope_rows_kernel<64, uint16_t>), grid, block, 0, s, a);
    }
    return launched();
}

int pdec_paged_rope_kv_append(const pdec_paged_dims* d, const pdec_rope_spec* spec, const void* q, int64_t q_stride,
                              void* q_out, int64_t q_out_stride, const void* k_new, int64_t k_stride, const void* v_new,
                              int64_t v_stride, const int32_t* pos_base, const int32_t* cu_tokens,
                              const int32_t* block_table, const int32_t* lens_in, int32_t* lens_out, void* k_pages,
                              void* v_pages, uint8_t* k_scales, uint8_t* v_scales, void* stream)
{
    int rc = check_dims(d);
    if (rc != PDEC_OK) return rc;
    PagedRopeArgs a{};
    rc = rope_spec(spec, 0, a.spec);
    if (rc != PDEC_OK) return rc;
    const int64_t q_row = (int64_t)d->num_q_heads * d->head_dim, kv_row = (int64_t)d->num_kv_heads * d->head_dim;
    if (spec->head_dim != d->head_dim || !aligned(q, 16) || !aligned(q_out, 16) || !aligned(k_new, 16) || !aligned(v_new, 16) ||
        !row_stride(q_stride, q_row, d->dtype) || !row_stride(q_out_stride, q_row, d->dtype) ||
        (q == q_out && q_stride != q_out_stride) || !row_stride(k_stride, kv_row, d->dtype) ||
        !row_stride(v_stride, kv_row, d->dtype) || (pos_base && !aligned(pos_base, 4)) || !aligned(cu_tokens, 4) ||
        !aligned(block_table, 4) || !aligned(lens_in, 4) || !aligned(lens_out, 4) || lens_in == lens_out ||
        !cache_pointers(d, k_pages, v_pages, k_scales, v_scales))
        return PDEC_ERR_INVALID_ARG;
    if (debug_mode() && (rc = debug_check(d, cu_tokens, lens_in, 0, stream)) != PDEC_OK) return rc;
    a.io = io_args(d);
    a.io.k_rows = k_new;
    a.io.v_rows = v_new;
    a.io.k_pages = k_pages;
    a.io.v_pages = v_pages;
    a.io.k_scales = k_scales;
    a.io.v_scales = v_scales;
    a.io.block_table = block_table;
    a.io.cu = cu_tokens;
    a.io.lens = lens_in;
    a.io.lens_out = lens_out;
    a.q = q;
    a.q_out = q_out;
    a.pos_base = pos_base;
    a.q_stride = q_stride;
    a.q_out_stride = q_out_stride;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.H_q = d->num_q_heads;
    const int per = 64 * 32 / (d->head_dim * (d->dtype == PDEC_DTYPE_F32 ? 4 : 2));
    a.split = rope_split(d->num_tokens, (a.H_q + per - 1) / per + 2 * ((d->num_kv_heads + per - 1) / per));
    const dim3 grid = rope_grid(std::max((d->num_tokens + 3) / 4, (d->num_seqs + 63) / 64), a.split);
    a.wide = (int)grid.x;
    hipStream_t s = static_cast<hipStream_t>(stream);
    for_types(d, [&](auto dim, auto t, auto form) {
        hipLaunchKernelGGL((paged_rope_append_kernel<dim(), decltype(t), form()>), grid, dim3(256), 0, s, a);
    });
    return launched();
}

}  // extern "C"
