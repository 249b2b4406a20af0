// Rotary positions with the norms of queries and keys, alone and on the way into a paged cache.
//
// Mathematics.  y = w x / sqrt(mean x^2 + eps) per head, then pairs of the first rot_dim values turned by position * f_i.
// The angle is position * (f_i / 2 pi mod 1) modulo a turn: with the fraction of a turn in 64 bits the product of integers
// wraps where the angle does, so nothing is lost however far the position is.  What is left after the nearest
// quarter of a turn goes to sincospif as an fp32 number of at most 1/4 (error 2e-8 in the angle, below fp32's rounding of
// cosine and sine).
//
// What bounds it: bytes (each value read and written once), and a launch's latency where the tokens are few.  Eight values a
// lane, so that a pair's other half is a shuffle away (or in the same lane) and a head's sum of squares stays in a warp; the
// lanes of a CTA share one table of cosines and sines per token, which would otherwise cost more instructions than all else.
// Few tokens: the heads of a token are spread over CTAs (grid y) until there is one for every SM.
#include "paged.cuh"

#include <math.h>

namespace coreinfer {

constexpr int kRopeThreads = 256;
constexpr int kRopeMaxTokens = 8;                    // tokens per CTA
constexpr int kRopeMaxPairs = 128;

struct RopeArgs {
    Paged c;                        // append only
    const uint64_t* turns;          // rot / 2
    const void* q_norm;
    const void* k_norm;
    const int32_t* positions;       // append: NULL means the slots' own
    const uint8_t* q;
    const uint8_t* k;
    const uint8_t* v;               // append only
    uint8_t* q_out;
    uint8_t* k_out;                 // apply only
    long long ld_q, ld_k, ld_v, ld_q_out, ld_k_out;
    float eps, magnitude;
    int rot, interleaved;
    int tokens, Hq, H;
    int units;                      // heads of a token, those of the values among them
    int per_token;                  // threads of a token
    int unit_step;                  // heads of a token per CTA
};

template <typename T>
__device__ __forceinline__ void load8(const uint8_t* p, uint4 (&raw)[sizeof(T) / 2])
{
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) raw[i] = reinterpret_cast<const uint4*>(p)[i];
}
template <typename T>
__device__ __forceinline__ void store8(uint8_t* p, const float (&x)[8])
{
    T v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = from_f32<T>(x[e]);
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(p)[i] = reinterpret_cast<const uint4*>(v)[i];
}

// The sequence that a packed row belongs to, or -1: every lane of the warp counts its share of the starts at or before the row.
__device__ __forceinline__ int row_sequence(const Paged& c, int row)
{
    const int lane = threadIdx.x & 31;
    int before = 0;
    for (int b = lane; b < c.B; b += 32) before += c.start[b + 1] <= row;
    before = __reduce_add_sync(0xffffffffu, before);
    return before < c.B && c.start[before] <= row ? before : -1;
}

template <typename T, int D, bool APPEND>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const __grid_constant__ RopeArgs a)
{
    constexpr int LPH = D / 8;                       // lanes per head
    constexpr int E = sizeof(T);
    __shared__ float2 table[kRopeMaxTokens][kRopeMaxPairs];
    __shared__ int at[kRopeMaxTokens];               // position a token is turned by
    const int tid = threadIdx.x;
    const int mine = tid / a.per_token;              // token of the CTA
    const int tokens = kRopeThreads / a.per_token;
    const int row = blockIdx.x * tokens + mine;
    const int slots = a.per_token / LPH;             // heads of a token at a time
    const int l = tid % LPH;
    const int first = blockIdx.y * a.unit_step;
    const int end = first + a.unit_step < a.units ? first + a.unit_step : a.units;
    const bool norms = a.q_norm != nullptr || a.k_norm != nullptr;
    wait_for_stream();

    // a token's place: the same in all its lanes, whole warps per token
    bool live = row < a.tokens;
    int page = -1, slot_position = 0;
    if (APPEND) {
        const int b = row_sequence(a.c, row);
        live = live && b >= 0;
        if (live) {
            const PagedSeq s = paged_seq(a.c, b);
            live = row - s.first < s.n;
            slot_position = s.position + row - s.first;
            if (live) page = paged_page(a.c, b, slot_position);
        }
    }
    auto source = [&](int u) -> const uint8_t* {
        if (u < a.Hq) return a.q + ((long long)row * a.ld_q + u * D + l * 8) * E;
        if (u < a.Hq + a.H) return a.k + ((long long)row * a.ld_k + (u - a.Hq) * D + l * 8) * E;
        return a.v + ((long long)row * a.ld_v + (u - a.Hq - a.H) * D + l * 8) * E;
    };
    int u = first + (tid % a.per_token) / LPH;
    uint4 raw[E / 2];
    if (live && u < end) load8<T>(source(u), raw);

    float wq[8], wk[8];
    if (norms) {
        uint4 w[E / 2];
        if (a.q_norm) { load8<T>((const uint8_t*)a.q_norm + l * 8 * E, w); unpack8<T>(w, wq); }
        if (a.k_norm) { load8<T>((const uint8_t*)a.k_norm + l * 8 * E, w); unpack8<T>(w, wk); }
    }
    if (a.rot) {
        if (tid % a.per_token == 0) at[mine] = !live ? 0 : (a.positions ? a.positions[row] : slot_position);
        __syncthreads();
        const int pairs = a.rot / 2;
        for (int i = tid; i < pairs * tokens; i += kRopeThreads) {
            const int t = i / pairs, j = i - t * pairs;
            const uint64_t turn = (uint64_t)(int64_t)at[t] * a.turns[j];
            const uint64_t quarter = (turn + (1ull << 61)) >> 62;
            float sine, cosine;
            sincospif((float)(int64_t)(turn - (quarter << 62)) * 0x1p-63f, &sine, &cosine);
            const float x = quarter & 1 ? sine : cosine, y = quarter & 1 ? cosine : sine;
            table[t][j] = make_float2(a.magnitude * (quarter == 1 || quarter == 2 ? -x : x), a.magnitude * (quarter & 2 ? -y : y));
        }
        __syncthreads();
    }
    if (!live) return;                               // whole warps: the shuffles below stay full

    // x' = c x + s (its partner's x)
    float c[8], s[8];
    const bool turned = l * 8 < a.rot;
    const int half = a.rot / 16;                     // lanes of the first halves
    const int partner = a.interleaved || !turned ? l : (l < half ? l + half : l - half);
    if (turned) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float2 t = table[mine][a.interleaved ? l * 4 + e / 2 : (l < half ? l : l - half) * 8 + e];
            c[e] = t.x;
            s[e] = (a.interleaved ? !(e & 1) : l < half) ? -t.y : t.y;
        }
    }
    // lanes of a warp may hold different heads: all of them go round as often as the first
    for (; u - (tid % a.per_token & 31) / LPH < end; u += slots) {
        const bool here = u < end;
        uint4 ahead[E / 2];
        if (u + slots < end) load8<T>(source(u + slots), ahead);
        float x[8];
        if (here) unpack8<T>(raw, x);
        else {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = 0.f;
        }
        const bool is_q = u < a.Hq, is_v = u >= a.Hq + a.H;
        if (norms) {
            float sum = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) sum = fmaf(x[e], x[e], sum);
#pragma unroll
            for (int d = 1; d < LPH; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
            const float r = __frsqrt_rn(sum * (1.f / D) + a.eps);
            if (is_q ? a.q_norm != nullptr : (!is_v && a.k_norm != nullptr)) {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = x[e] * r * (is_q ? wq[e] : wk[e]);
            }
        }
        if (a.rot) {
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = a.interleaved ? x[e ^ 1] : __shfl_sync(0xffffffffu, x[e], partner, LPH);
            if (turned && !is_v) {
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = fmaf(s[e], y[e], c[e] * x[e]);
            }
        }
        if (here) {
            if (is_q) store8<T>(a.q_out + ((long long)row * a.ld_q_out + u * D + l * 8) * E, x);
            else if (APPEND) {
                const int h = is_v ? u - a.Hq - a.H : u - a.Hq;
                if (page >= 0) {
                    uint8_t* to = const_cast<uint8_t*>(a.c.pool[is_v]) + (paged_offset(a.c, page, h, slot_position) + l * 8) * E;
                    if (is_v) {
#pragma unroll
                        for (int i = 0; i < E / 2; ++i) reinterpret_cast<uint4*>(to)[i] = raw[i];
                    } else store8<T>(to, x);
                }
            } else store8<T>(a.k_out + ((long long)row * a.ld_k_out + (u - a.Hq) * D + l * 8) * E, x);
        }
#pragma unroll
        for (int i = 0; i < E / 2; ++i) raw[i] = ahead[i];
    }
    let_next_start();
}

template <typename T, int D, bool APPEND>
static coreinfer_status launch_rope(RopeArgs& a, const DeviceInfo& di, cudaStream_t st)
{
    constexpr int LPH = D / 8;
    // several tokens per CTA where their heads leave room, but not fewer CTAs than two for every SM
    int tokens = 1;
    while (tokens < kRopeMaxTokens && 2 * tokens * a.units * LPH <= kRopeThreads && a.tokens / (2 * tokens) >= 2 * di.sm_count) tokens *= 2;
    a.per_token = kRopeThreads / tokens;
    const int slots = a.per_token / LPH;
    const int ctas = (a.tokens + tokens - 1) / tokens;
    // few tokens: their heads over several CTAs, one round of heads each at least
    const int rounds = (a.units + slots - 1) / slots;
    int split = (di.sm_count + ctas - 1) / ctas;
    if (split > rounds) split = rounds;
    a.unit_step = (rounds + split - 1) / split * slots;
    const int y = (a.units + a.unit_step - 1) / a.unit_step;
    CI_CUDA(launch_overlapped(rope_kernel<T, D, APPEND>, dim3(ctas, y), dim3(kRopeThreads), 0, st, a));
    return COREINFER_OK;
}

template <typename T, bool APPEND>
static coreinfer_status pick_rope(RopeArgs& a, int D, const DeviceInfo& di, cudaStream_t st)
{
    if (D == 64) return launch_rope<T, 64, APPEND>(a, di, st);
    return D == 128 ? launch_rope<T, 128, APPEND>(a, di, st) : launch_rope<T, 256, APPEND>(a, di, st);
}

template <bool APPEND>
static coreinfer_status launch_typed(RopeArgs& a, coreinfer_dtype dtype, int D, cudaStream_t st)
{
    DeviceInfo di;
    const coreinfer_status s = device_info(&di);
    if (s != COREINFER_OK) return s;
    if (dtype == COREINFER_F32) return pick_rope<float, APPEND>(a, D, di, st);
    if (dtype == COREINFER_BF16) return pick_rope<__nv_bfloat16, APPEND>(a, D, di, st);
    return pick_rope<__half, APPEND>(a, D, di, st);
}

static coreinfer_status take_rope(const coreinfer_rope* r, int head_dim, RopeArgs* a)
{
    if (!r->turns || !aligned_to(r->turns, 8)) CI_FAIL(COREINFER_ERR_INVALID_ARG, "turns NULL or not 8-byte aligned");
    if (r->rot_dim < 16 || r->rot_dim % 16 != 0 || r->rot_dim > head_dim)
        CI_FAIL(COREINFER_ERR_UNSUPPORTED, "rot_dim %d: a multiple of 16 up to head_dim %d", r->rot_dim, head_dim);
    if (!aligned16(r->q_norm) || !aligned16(r->k_norm)) CI_FAIL(COREINFER_ERR_INVALID_ARG, "norm weights not 16-byte aligned");
    if (!(r->eps >= 0.f)) CI_FAIL(COREINFER_ERR_INVALID_ARG, "eps must be >= 0");
    a->turns = r->turns;
    a->q_norm = r->q_norm;
    a->k_norm = r->k_norm;
    a->eps = r->eps;
    a->magnitude = r->magnitude;
    a->rot = r->rot_dim;
    a->interleaved = r->interleaved != 0;
    return COREINFER_OK;
}

static coreinfer_status check_sizes(int tokens, int q_heads, int kv_heads)
{
    if (tokens < 1 || q_heads < 0 || kv_heads < 0 || q_heads + (long long)kv_heads < 1)
        CI_FAIL(COREINFER_ERR_INVALID_ARG, "tokens and the number of heads must be >= 1");
    if (q_heads > 4096 || kv_heads > 1024) CI_FAIL(COREINFER_ERR_UNSUPPORTED, "q_heads %d, kv_heads %d: at most 4096 and 1024", q_heads, kv_heads);
    if ((long long)tokens * (q_heads + 2 * kv_heads) > 1LL << 29) CI_FAIL(COREINFER_ERR_UNSUPPORTED, "tokens %d: too many for one call", tokens);
    return COREINFER_OK;
}

}  // namespace coreinfer

using namespace coreinfer;

extern "C" {

coreinfer_status coreinfer_rope_frequencies(int32_t rot_dim, double base, coreinfer_rope_scaling scaling, double factor,
                                            int32_t original_context, double low, double high,
                                            uint64_t* turns, float* magnitude)
{
    if (!turns || !magnitude) CI_FAIL(COREINFER_ERR_INVALID_ARG, "turns or magnitude is NULL");
    if (rot_dim < 16 || rot_dim > 2 * kRopeMaxPairs || rot_dim % 16 != 0)
        CI_FAIL(COREINFER_ERR_UNSUPPORTED, "rot_dim %d: a multiple of 16 from 16 to 256", rot_dim);
    if (scaling < COREINFER_ROPE_PLAIN || scaling > COREINFER_ROPE_BANDS) CI_FAIL(COREINFER_ERR_UNSUPPORTED, "scaling %d is not known", (int)scaling);
    if (!(base > 1.0) || !isfinite(base)) CI_FAIL(COREINFER_ERR_INVALID_ARG, "base must be above 1");
    if (scaling != COREINFER_ROPE_PLAIN && (!(factor >= 1.0) || !isfinite(factor))) CI_FAIL(COREINFER_ERR_INVALID_ARG, "factor must be >= 1");
    const bool ranged = scaling == COREINFER_ROPE_YARN || scaling == COREINFER_ROPE_BANDS;
    if (ranged && (original_context < 1 || !(low > 0.0) || !(high > low) || !isfinite(high)))
        CI_FAIL(COREINFER_ERR_INVALID_ARG, "original_context >= 1 and 0 < low < high are needed");
    const double two_pi = 6.283185307179586476925;
    if (scaling == COREINFER_ROPE_NTK) base *= pow(factor, (double)rot_dim / (rot_dim - 2));
    double from = 0.0, to = 0.0;
    if (scaling == COREINFER_ROPE_YARN) {
        // the pair (as a real number) that turns n times within the context: 2 pi n = context * base^(-2 i / rot_dim)
        const double per = rot_dim / (2.0 * log(base));
        from = floor(per * log(original_context / (high * two_pi)));
        to = ceil(per * log(original_context / (low * two_pi)));
        if (from < 0.0) from = 0.0;
        if (to > rot_dim - 1.0) to = rot_dim - 1.0;
        if (to - from < 0.001) to = from + 0.001;
    }
    for (int i = 0; i < rot_dim / 2; ++i) {
        double f = pow(base, -2.0 * i / rot_dim);
        if (scaling == COREINFER_ROPE_LINEAR) f /= factor;
        if (scaling == COREINFER_ROPE_YARN) {
            double r = (i - from) / (to - from);
            r = r < 0.0 ? 0.0 : (r > 1.0 ? 1.0 : r);
            f = f / factor * r + f * (1.0 - r);
        }
        if (scaling == COREINFER_ROPE_BANDS) {
            double s = (original_context * f / two_pi - low) / (high - low);
            s = s < 0.0 ? 0.0 : (s > 1.0 ? 1.0 : s);
            f = f / factor * (1.0 - s) + f * s;
        }
        turns[i] = (uint64_t)ldexp(f / two_pi, 64);              // f <= 1: below a sixth of a turn
    }
    *magnitude = scaling == COREINFER_ROPE_YARN ? (float)(0.1 * log(factor) + 1.0) : 1.f;
    return COREINFER_OK;
}

coreinfer_status coreinfer_rope_apply(const coreinfer_rope* rope, const int32_t* positions, coreinfer_dtype dtype,
                                      int32_t tokens, int32_t q_heads, int32_t kv_heads, int32_t head_dim,
                                      const void* q, int64_t ld_q, const void* k, int64_t ld_k,
                                      void* q_out, int64_t ld_q_out, void* k_out, int64_t ld_k_out, void* cuda_stream)
{
    if (!rope) CI_FAIL(COREINFER_ERR_INVALID_ARG, "rope is NULL");
    if (!dtype_known(dtype)) CI_FAIL(COREINFER_ERR_UNSUPPORTED, "dtype %d is not supported", (int)dtype);
    if (head_dim != 64 && head_dim != 128 && head_dim != 256)
        CI_FAIL(COREINFER_ERR_UNSUPPORTED, "head_dim %d: 64, 128 and 256 are built", head_dim);
    RopeArgs a = {};
    coreinfer_status s = take_rope(rope, head_dim, &a);
    if (s != COREINFER_OK || (s = check_sizes(tokens, q_heads, kv_heads)) != COREINFER_OK) return s;
    if (!positions || !aligned_to(positions, 4)) CI_FAIL(COREINFER_ERR_INVALID_ARG, "positions NULL or misaligned");
    if (q_heads && (!rows_fit(q, ld_q, q_heads, head_dim, dtype) || !rows_fit(q_out, ld_q_out, q_heads, head_dim, dtype)))
        CI_FAIL(COREINFER_ERR_INVALID_ARG, "q / q_out NULL, not 16-byte aligned, or strides too small or not multiples of 16 bytes");
    if (kv_heads && (!rows_fit(k, ld_k, kv_heads, head_dim, dtype) || !rows_fit(k_out, ld_k_out, kv_heads, head_dim, dtype)))
        CI_FAIL(COREINFER_ERR_INVALID_ARG, "k / k_out NULL, not 16-byte aligned, or strides too small or not multiples of 16 bytes");
    a.positions = positions;
    a.q = (const uint8_t*)q;
    a.k = (const uint8_t*)k;
    a.q_out = (uint8_t*)q_out;
    a.k_out = (uint8_t*)k_out;
    a.ld_q = ld_q;
    a.ld_k = ld_k;
    a.ld_q_out = ld_q_out;
    a.ld_k_out = ld_k_out;
    a.tokens = tokens;
    a.Hq = q_heads;
    a.H = kv_heads;
    a.units = q_heads + kv_heads;
    return launch_typed<false>(a, dtype, head_dim, (cudaStream_t)cuda_stream);
}

coreinfer_status coreinfer_paged_append(const coreinfer_paged_cache* cache, const int32_t* start, int32_t tokens,
                                        const void* k, int64_t ld_k, const void* v, int64_t ld_v,
                                        const coreinfer_rope* rope, const int32_t* positions,
                                        const void* q, int64_t ld_q, int32_t q_heads, void* q_out, int64_t ld_q_out,
                                        void* cuda_stream)
{
    RopeArgs a = {};
    coreinfer_status s = paged_take(cache, &a.c);
    if (s != COREINFER_OK) return s;
    const coreinfer_dtype dtype = cache->dtype;
    const int D = a.c.D;
    if (rope && (s = take_rope(rope, D, &a)) != COREINFER_OK) return s;
    if ((s = check_sizes(tokens, q_heads, a.c.H)) != COREINFER_OK) return s;
    if (!start || !aligned_to(start, 4) || !aligned_to(positions, 4)) CI_FAIL(COREINFER_ERR_INVALID_ARG, "start NULL, or start or positions misaligned");
    if (!rows_fit(k, ld_k, a.c.H, D, dtype) || !rows_fit(v, ld_v, a.c.H, D, dtype))
        CI_FAIL(COREINFER_ERR_INVALID_ARG, "k / v NULL, not 16-byte aligned, or strides too small or not multiples of 16 bytes");
    if ((q != nullptr) != (q_out != nullptr) || (q != nullptr) != (q_heads > 0))
        CI_FAIL(COREINFER_ERR_INVALID_ARG, "q, q_out and q_heads come together or not at all");
    if (q && !rope) CI_FAIL(COREINFER_ERR_INVALID_ARG, "without rope there is nothing to do to q");
    if (q && (!rows_fit(q, ld_q, q_heads, D, dtype) || !rows_fit(q_out, ld_q_out, q_heads, D, dtype)))
        CI_FAIL(COREINFER_ERR_INVALID_ARG, "q / q_out not 16-byte aligned, or strides too small or not multiples of 16 bytes");
    a.c.start = start;
    a.c.tokens = tokens;
    a.positions = positions;
    a.q = (const uint8_t*)q;
    a.k = (const uint8_t*)k;
    a.v = (const uint8_t*)v;
    a.q_out = (uint8_t*)q_out;
    a.ld_q = ld_q;
    a.ld_k = ld_k;
    a.ld_v = ld_v;
    a.ld_q_out = ld_q_out;
    a.tokens = tokens;
    a.Hq = q_heads;
    a.H = a.c.H;
    a.units = q_heads + 2 * a.c.H;
    return launch_typed<true>(a, dtype, D, (cudaStream_t)cuda_stream);
}

}  // extern "C"
