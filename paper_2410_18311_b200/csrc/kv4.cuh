// What the kernels of the 4-bit key/value cache share: the descriptor as kernels take it, and its checks.
#pragma once

#include "quant4.cuh"

namespace coreinfer {

struct Kv4 {
    uint8_t* codes[2];      // keys, values: [B][H][cap][D / 2]
    __half2* pairs[2];      // [B][H][cap][D / G]
    int32_t* state;         // [B][4]: slots in use, tokens ever appended, tokens refused, arrival ticket
    float* weight;          // [B][H][cap] or NULL
    int32_t* position;
    int B, H, cap, D, G;
};

enum { kStateLength = 0, kStateSeen = 1, kStateRefused = 2, kStateTicket = 3 };

// Checks a descriptor and copies it out.
inline coreinfer_status kv4_take(const coreinfer_kv4_cache* c, const char* what, Kv4* out)
{
    if (!c) CI_FAIL(COREINFER_ERR_INVALID_ARG, "%s cache descriptor is NULL", what);
    if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256)
        CI_FAIL(COREINFER_ERR_UNSUPPORTED, "%s cache: head_dim %d: 64, 128 and 256 are built", what, c->head_dim);
    if (!group_known(c->group) || c->group > c->head_dim)
        CI_FAIL(COREINFER_ERR_UNSUPPORTED, "%s cache: group %d: 32, 64 or 128, at most head_dim", what, c->group);
    if (c->batch < 1 || c->kv_heads < 1 || c->capacity < 16 || c->capacity % 16 != 0)
        CI_FAIL(COREINFER_ERR_INVALID_ARG, "%s cache: batch and kv_heads must be >= 1, capacity a positive multiple of 16", what);
    if (c->batch > COREINFER_KV4_MAX_BATCH)
        CI_FAIL(COREINFER_ERR_UNSUPPORTED, "%s cache: batch %d: at most %d", what, c->batch, COREINFER_KV4_MAX_BATCH);
    if (c->kv_heads > 1024) CI_FAIL(COREINFER_ERR_UNSUPPORTED, "%s cache: kv_heads %d: at most 1024", what, c->kv_heads);
    if (!c->k_codes || !c->v_codes || !c->k_pairs || !c->v_pairs || !aligned16(c->k_codes) || !aligned16(c->v_codes) ||
        !aligned16(c->k_pairs) || !aligned16(c->v_pairs))
        CI_FAIL(COREINFER_ERR_INVALID_ARG, "%s cache: codes / pairs NULL or not 16-byte aligned", what);
    if (!c->state || !aligned_to(c->state, 16)) CI_FAIL(COREINFER_ERR_INVALID_ARG, "%s cache: state NULL or not 16-byte aligned", what);
    if ((c->weight == nullptr) != (c->position == nullptr) || !aligned16(c->weight) || !aligned16(c->position))
        CI_FAIL(COREINFER_ERR_INVALID_ARG, "%s cache: weight and position come both (16-byte aligned) or neither", what);
    out->codes[0] = (uint8_t*)c->k_codes;
    out->codes[1] = (uint8_t*)c->v_codes;
    out->pairs[0] = (__half2*)c->k_pairs;
    out->pairs[1] = (__half2*)c->v_pairs;
    out->state = c->state;
    out->weight = c->weight;
    out->position = c->position;
    out->B = c->batch;
    out->H = c->kv_heads;
    out->cap = c->capacity;
    out->D = c->head_dim;
    out->G = c->group;
    return COREINFER_OK;
}

#ifdef __CUDACC__
// Slots in use, whatever the caller left in the state.
__device__ __forceinline__ int kv4_length(const Kv4& c, int b)
{
    const int n = c.state[b * 4 + kStateLength];
    return n < 0 ? 0 : (n > c.cap ? c.cap : n);
}

// Called by every thread of a CTA at its end; true in thread 0 of the last of the `ctas` CTAs that work on
// sequence b.  All of them have read the state by then, so that one may change it.
__device__ __forceinline__ bool kv4_last_of_sequence(const Kv4& c, int b, int ctas)
{
    __syncthreads();
    if (threadIdx.x != 0) return false;
    __threadfence();
    if (atomicAdd(&c.state[b * 4 + kStateTicket], 1) != ctas - 1) return false;
    c.state[b * 4 + kStateTicket] = 0;
    return true;
}
#endif

}  // namespace coreinfer
