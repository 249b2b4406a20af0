// What the kernels of the paged key/value cache share: the descriptor as kernels take it, its checks, and which
// sequence, slot and page a packed row belongs to.
#pragma once

#include "quant4.cuh"

#include <type_traits>

namespace coreinfer {

struct Paged {
    const uint8_t* pool[2];         // keys, values
    const int32_t* table;           // [B][max_pages]
    const int32_t* length;          // [B]
    const int32_t* start;           // [B + 1]
    long long page_stride, head_stride, token_stride;   // elements
    int n_pages, page_shift, H, D, B, max_pages;
    int cap;                        // positions that the table covers
    int tokens;                     // rows of the packed tensors
};

// Checks a descriptor and copies it out.
inline coreinfer_status paged_take(const coreinfer_paged_cache* c, Paged* out)
{
    if (!c) CI_FAIL(COREINFER_ERR_INVALID_ARG, "the cache descriptor is NULL");
    if (!dtype_known(c->dtype)) CI_FAIL(COREINFER_ERR_UNSUPPORTED, "dtype %d is not supported", (int)c->dtype);
    if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256)
        CI_FAIL(COREINFER_ERR_UNSUPPORTED, "head_dim %d: 64, 128 and 256 are built", c->head_dim);
    if (c->page_size < 16 || c->page_size > 256 || (c->page_size & (c->page_size - 1)))
        CI_FAIL(COREINFER_ERR_UNSUPPORTED, "page_size %d: 16, 32, 64, 128 or 256", c->page_size);
    if (c->batch < 1 || c->kv_heads < 1 || c->n_pages < 1 || c->max_pages < 1)
        CI_FAIL(COREINFER_ERR_INVALID_ARG, "batch, kv_heads, n_pages and max_pages must be >= 1");
    if (c->batch > COREINFER_PAGED_MAX_BATCH)
        CI_FAIL(COREINFER_ERR_UNSUPPORTED, "batch %d: at most %d", c->batch, COREINFER_PAGED_MAX_BATCH);
    if (c->kv_heads > 1024) CI_FAIL(COREINFER_ERR_UNSUPPORTED, "kv_heads %d: at most 1024", c->kv_heads);
    if (c->n_pages >= 1 << 27) CI_FAIL(COREINFER_ERR_UNSUPPORTED, "n_pages %d: below 2^27", c->n_pages);
    if ((long long)c->max_pages * c->page_size >= 1 << 30)
        CI_FAIL(COREINFER_ERR_UNSUPPORTED, "max_pages %d of %d slots: below 2^30 positions", c->max_pages, c->page_size);
    if (!c->k || !c->v || !aligned16(c->k) || !aligned16(c->v)) CI_FAIL(COREINFER_ERR_INVALID_ARG, "pools NULL or not 16-byte aligned");
    if (!c->table || !c->length || !aligned_to(c->table, 4) || !aligned_to(c->length, 4))
        CI_FAIL(COREINFER_ERR_INVALID_ARG, "table or length NULL or misaligned");
    const long long per16 = 16 / (long long)dtype_size(c->dtype);
    // slots of a head must not overlap: each stride covers a row at least, and a page what its heads and slots take
    if (c->token_stride < c->head_dim || (c->kv_heads > 1 && c->head_stride < c->head_dim) || c->head_stride < 0 ||
        (c->n_pages > 1 && c->page_stride < (long long)(c->kv_heads - 1) * c->head_stride + (c->page_size - 1) * c->token_stride + c->head_dim))
        CI_FAIL(COREINFER_ERR_INVALID_ARG, "strides (page %lld, head %lld, token %lld) let slots overlap", (long long)c->page_stride,
                (long long)c->head_stride, (long long)c->token_stride);
    if (c->kv_heads > 1 && c->head_stride < (long long)(c->page_size - 1) * c->token_stride + c->head_dim &&
        c->token_stride < (long long)(c->kv_heads - 1) * c->head_stride + c->head_dim)
        CI_FAIL(COREINFER_ERR_INVALID_ARG, "strides (head %lld, token %lld) let slots overlap", (long long)c->head_stride, (long long)c->token_stride);
    if (c->page_stride % per16 || c->head_stride % per16 || c->token_stride % per16 || c->page_stride < 0)
        CI_FAIL(COREINFER_ERR_INVALID_ARG, "strides must be multiples of 16 bytes");
    if (c->page_stride > (1LL << 40) / c->n_pages)
        CI_FAIL(COREINFER_ERR_UNSUPPORTED, "%d pages of stride %lld: at most 2^40 elements", c->n_pages, (long long)c->page_stride);
    if (c->page_stride >= 1LL << 36 || c->head_stride >= 1LL << 36 || c->token_stride >= 1LL << 36)
        CI_FAIL(COREINFER_ERR_UNSUPPORTED, "strides of 2^36 elements or more");
    out->pool[0] = (const uint8_t*)c->k;
    out->pool[1] = (const uint8_t*)c->v;
    out->table = c->table;
    out->length = c->length;
    out->page_stride = c->page_stride;
    out->head_stride = c->head_stride;
    out->token_stride = c->token_stride;
    out->n_pages = c->n_pages;
    out->page_shift = 0;
    while ((1 << out->page_shift) < c->page_size) ++out->page_shift;
    out->H = c->kv_heads;
    out->D = c->head_dim;
    out->B = c->batch;
    out->max_pages = c->max_pages;
    out->cap = c->max_pages * c->page_size;
    out->start = nullptr;
    out->tokens = 0;
    return COREINFER_OK;
}

// Rows of `heads` contiguous heads: alignment of the pointer and the stride.
static inline bool rows_fit(const void* p, long long ld, long long heads, int head_dim, coreinfer_dtype dtype)
{
    return p && aligned16(p) && ld >= heads * head_dim && (ld * (long long)dtype_size(dtype)) % 16 == 0;
}

#ifdef __CUDACC__

// Two values rounded to 16 bits, the first in the lower half.
template <typename T>
__device__ __forceinline__ uint32_t pack2(float lo, float hi)
{
    uint32_t r;
    if constexpr (sizeof(T) == 2 && std::is_same<T, __half>::value) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// A sequence's new rows first .. first + n - 1 and the position of the first of them (below 0 where length and
// start do not fit together).
struct PagedSeq {
    int first, n, position;
};
__device__ __forceinline__ int clamp_int(int x, int lo, int hi) { return x < lo ? lo : (x > hi ? hi : x); }
__device__ __forceinline__ PagedSeq paged_seq(const Paged& c, int b)
{
    PagedSeq s;
    s.first = clamp_int(c.start[b], 0, c.tokens);
    const int end = clamp_int(c.start[b + 1], 0, c.tokens);
    s.n = end > s.first ? end - s.first : 0;
    s.position = clamp_int(c.length[b], 0, 1 << 30) - s.n;
    return s;
}

// Page of a position, or -1 where the sequence has none there.  position < cap.
__device__ __forceinline__ int paged_page(const Paged& c, int b, int position)
{
    if (position < 0 || position >= c.cap) return -1;
    const int g = c.table[(long long)b * c.max_pages + (position >> c.page_shift)];
    return g >= 0 && g < c.n_pages ? g : -1;
}
// Element offset of a slot.
__device__ __forceinline__ long long paged_offset(const Paged& c, int page, int h, int position)
{
    return page * c.page_stride + h * c.head_stride + (position & ((1 << c.page_shift) - 1)) * c.token_stride;
}
#endif

}  // namespace coreinfer
