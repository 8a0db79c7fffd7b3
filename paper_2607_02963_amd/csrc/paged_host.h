// Host side of the paged calls: what their entry points share.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <memory>
#include <new>
#include <type_traits>

#include "pdec.h"

#include "kernel_paged_io.h"

namespace pdec {

inline bool aligned(const void* p, uintptr_t a) { return p && (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// Rows of a call, and sequences: the launches' threads stay within 32 bits.
constexpr int kMostRows = 1 << 27;

inline int check_dims(const pdec_paged_dims* d)
{
    if (!d) return PDEC_ERR_INVALID_ARG;
    if (d->num_seqs < 1 || d->num_tokens < 1 || d->num_q_heads < 1 || d->num_kv_heads < 1 ||
        d->num_q_heads % d->num_kv_heads != 0 || d->num_pages < 1 || d->max_pages < 1 || d->max_chunk < 0 ||
        d->max_len < 0 || d->causal < 0 || d->causal > 1 || d->page_size < 1)
        return PDEC_ERR_INVALID_ARG;
    if (std::isnan(d->softmax_scale) || std::isinf(d->softmax_scale)) return PDEC_ERR_INVALID_ARG;
    if (d->dtype != PDEC_DTYPE_F32 && d->dtype != PDEC_DTYPE_BF16) return PDEC_ERR_UNSUPPORTED;
    if (d->cache_dtype != d->dtype && d->cache_dtype != PDEC_DTYPE_E4M3 && d->cache_dtype != PDEC_DTYPE_E2M1)
        return PDEC_ERR_UNSUPPORTED;
    if (d->head_dim != 64 && d->head_dim != 128) return PDEC_ERR_UNSUPPORTED;
    if (d->page_size < 16 || d->page_size > 1024 || (d->page_size & (d->page_size - 1)) != 0)
        return PDEC_ERR_UNSUPPORTED;
    if (d->num_tokens > kMostRows || d->num_seqs > kMostRows) return PDEC_ERR_UNSUPPORTED;
    const int64_t most = (int64_t)d->max_pages * d->page_size;
    if (most > ((int64_t)1 << 30)) return PDEC_ERR_UNSUPPORTED;
    if (d->max_len > most) return PDEC_ERR_INVALID_ARG;
    // a token's keys, and a page, within 32-bit offsets (a pool may be larger)
    if ((int64_t)d->num_kv_heads * d->head_dim * d->page_size * 4 > INT32_MAX) return PDEC_ERR_UNSUPPORTED;
    return PDEC_OK;
}

inline int len_bound(const pdec_paged_dims* d) { return d->max_len > 0 ? d->max_len : d->max_pages * d->page_size; }
inline int shift_of(int page_size) { return __builtin_ctz((unsigned)page_size); }

// What the three cache calls share of their pointers' checks.
inline bool cache_pointers(const pdec_paged_dims* d, const void* k, const void* v, const uint8_t* ks, const uint8_t* vs)
{
    if (!aligned(k, 16) || !aligned(v, 16)) return false;
    if (d->cache_dtype == PDEC_DTYPE_E2M1) return aligned(ks, 16) && aligned(vs, 16);
    return d->cache_dtype != PDEC_DTYPE_E4M3 || (aligned(ks, 4) && aligned(vs, 4));
}

// PDEC_DEBUG=1: the lengths of a call, copied and checked (synchronises).
inline int debug_check(const pdec_paged_dims* d, const int32_t* cu, const int32_t* lens, int attn, void* stream)
{
    const size_t S = (size_t)d->num_seqs;
    const std::unique_ptr<int32_t[]> c(new (std::nothrow) int32_t[2 * S + 1]);  // no exception leaves a C entry
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (!c || hipMemcpyAsync(c.get(), cu, (S + 1) * 4, hipMemcpyDeviceToHost, s) != hipSuccess ||
        hipMemcpyAsync(c.get() + S + 1, lens, S * 4, hipMemcpyDeviceToHost, s) != hipSuccess ||
        hipStreamSynchronize(s) != hipSuccess)
        return PDEC_ERR_HIP;
    return pdec_check_paged_lengths(d, c.get(), c.get() + S + 1, attn);
}

inline PagedIoArgs io_args(const pdec_paged_dims* d)
{
    PagedIoArgs a{};
    a.num_seqs = d->num_seqs;
    a.num_tokens = d->num_tokens;
    a.H_kv = d->num_kv_heads;
    a.page_shift = shift_of(d->page_size);
    a.num_pages = d->num_pages;
    a.max_pages = d->max_pages;
    a.max_len = len_bound(d);
    return a;
}

// f(head dim, an element of the rows' type, the cache's form), as types
template <typename F>
void for_types(const pdec_paged_dims* d, F f)
{
    auto forms = [&](auto dim, auto t) {
        if (d->cache_dtype == PDEC_DTYPE_E2M1) f(dim, t, std::integral_constant<PagedForm, kE2m1Rows>{});
        else if (d->cache_dtype == PDEC_DTYPE_E4M3) f(dim, t, std::integral_constant<PagedForm, kE4m3Rows>{});
        else f(dim, t, std::integral_constant<PagedForm, kPlainRows>{});
    };
    auto types = [&](auto dim) { d->dtype == PDEC_DTYPE_F32 ? forms(dim, float{}) : forms(dim, uint16_t{}); };
    if (d->head_dim == 128) types(std::integral_constant<int, 128>{});
    else types(std::integral_constant<int, 64>{});
}

inline int launched() { return hipGetLastError() == hipSuccess ? PDEC_OK : PDEC_ERR_HIP; }

}  // namespace pdec
