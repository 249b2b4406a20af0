// Rotary positions with the norms of queries and keys, alone and on the way into a paged cache.
//
// Mathematics.  y = w x / sqrt(mean x^2 + eps) per head, then pairs of the first rot_dim values turned by position * f_i.
// The angle is position * (f_i / 2 pi mod 1) modulo a turn: with the fraction of a turn in 64 bits the product of integers
// wraps where the angle does, so nothing is lost however far the position is.  What is left after the nearest
// quarter of a turn goes to sincospif as an fp32 number of at most 1/4 (error 2e-8 in the angle, below fp32's rounding of
// cosine and sine).
//
// Measured from a graph, three sets of inputs: 8191 tokens x 40 heads of 128 fp16, norms 35.7 us, 4700 GB/s; 16000 x 64 bf16 92 us, 5670; 6000 x 40
// fp32, norms 45.8 us, 5370; 5000 tokens x 48 heads bf16 into pages 36 us, 3400 (a round of warps and a bit).
// Two loads ahead and 32 warps an SM: four loads and 24 warps 39.5, 89, 67, 35; eight at once and none ahead 47.6, 108, 46.7, 41.  At 64 registers
// ptxas spills 16 to 68 bytes a thread (fp32, at 80: up to 12).
//
// What bounds it: bytes (each value read and written once), and a launch's latency where the tokens are few.  A warp takes a token, or a
// part of its heads where the tokens are few, so that the cosines and sines are formed once per token (two pairs a lane, through
// shared memory) and no warp waits for another.  Eight values a lane: a pair's other half is a shuffle away (of packed words) or in the
// same lane.  Norm weights enter the table's factors, so that a value costs a product, a fused product and the product with 1 / root:
//   y = r (x (w c) + x' (w' s)),  r = 1 / sqrt(mean x^2 + eps),  x', w': the pair's other value and its weight.
#include "paged.cuh"

#include <math.h>

namespace coreinfer {

constexpr int kRopeWarps = 8;
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
    int split;                      // warps per token
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
    if constexpr (sizeof(T) == 4) {
        reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
        reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
    } else *reinterpret_cast<uint4*>(p) = make_uint4(pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3]), pack2<T>(x[4], x[5]), pack2<T>(x[6], x[7]));
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
__global__ void __launch_bounds__(32 * kRopeWarps, sizeof(T) == 2 ? 4 : 3) rope_kernel(const __grid_constant__ RopeArgs a)
{
    constexpr int LPH = D / 8;                       // lanes per head
    constexpr int HPW = 32 / LPH;                    // heads at a time
    constexpr int E = sizeof(T);
    constexpr int WORDS = E / 2;                     // 16-byte words of eight values
    constexpr int U = 2;                             // loads a lane makes ahead of those it works on
    __shared__ float2 tables[kRopeWarps][kRopeMaxPairs];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, l = lane % LPH;
    float2* table = tables[warp];
    const unsigned id = blockIdx.x * kRopeWarps + warp;
    const int row = id / (unsigned)a.split, part = id - row * a.split;
    const int rounds_q = (a.Hq + HPW - 1) / HPW, rounds_h = (a.H + HPW - 1) / HPW;
    const int total = rounds_q + (APPEND ? 2 : 1) * rounds_h;
    const int first = total * part / a.split, end = total * (part + 1) / a.split;
    wait_for_stream();
    if (row >= a.tokens) return;

    int page = -1, slot_position = 0;
    if (APPEND) {
        const int b = row_sequence(a.c, row);
        if (b < 0) return;
        const PagedSeq s = paged_seq(a.c, b);
        if (row - s.first >= s.n) return;
        slot_position = s.position + row - s.first;
        page = paged_page(a.c, b, slot_position);
    }
    if (a.rot && first < rounds_q + rounds_h) {
        const uint64_t at = (uint64_t)(int64_t)(a.positions ? a.positions[row] : slot_position);
        for (int j = lane; j < a.rot / 2; j += 32) {
            const uint64_t turn = at * a.turns[j];
            const uint64_t quarter = (turn + (1ull << 61)) >> 62 & 3;
            float sine, cosine;
            sincospif((float)(int64_t)(turn - (quarter << 62)) * 0x1p-63f, &sine, &cosine);
            const float x = quarter & 1 ? sine : cosine, y = quarter & 1 ? cosine : sine;
            table[j] = make_float2(a.magnitude * (quarter == 1 || quarter == 2 ? -x : x), a.magnitude * (quarter & 2 ? -y : y));
        }
        __syncwarp();
    }

    const bool turned = l * 8 < a.rot;
    const int half = a.rot / 16;                     // lanes of the first halves
    const int partner = a.interleaved || !turned ? l : (l < half ? l + half : l - half);

    // heads [from, to) of rounds of queries or keys; kind 0 queries, 1 keys
    auto turn_heads = [&](int kind, int from, int to) {
        const uint8_t* in = kind == 0 ? a.q : a.k;
        const long long ld = kind == 0 ? a.ld_q : a.ld_k;
        const int heads = kind == 0 ? a.Hq : a.H;
        const uint8_t* weight = (const uint8_t*)(kind == 0 ? a.q_norm : a.k_norm);
        const uint8_t* src = in + ((long long)row * ld + l * 8) * E;
        uint8_t* dst;
        long long step;                              // bytes between heads
        if (kind == 0) { dst = a.q_out + ((long long)row * a.ld_q_out + l * 8) * E; step = D * E; }
        else if (!APPEND) { dst = a.k_out + ((long long)row * a.ld_k_out + l * 8) * E; step = D * E; }
        else {
            if (page < 0) return;
            dst = const_cast<uint8_t*>(a.c.pool[0]) + (paged_offset(a.c, page, 0, slot_position) + l * 8) * E;
            step = a.c.head_stride * E;
        }
        float cw[8], sw[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) { cw[e] = 1.f; sw[e] = 0.f; }
        if (turned) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float2 t = table[a.interleaved ? l * 4 + e / 2 : (l < half ? l : l - half) * 8 + e];
                cw[e] = t.x;
                sw[e] = (a.interleaved ? !(e & 1) : l < half) ? -t.y : t.y;
            }
        }
        if (weight) {
            uint4 raw[WORDS];
            float w[8];
            load8<T>(weight + l * 8 * E, raw);
            unpack8<T>(raw, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float other = a.interleaved ? w[e ^ 1] : __shfl_sync(0xffffffffu, w[e], partner, LPH);
                cw[e] *= w[e];
                sw[e] *= other;
            }
        }
        uint4 raw[U][WORDS], ahead[U][WORDS];
        auto fetch = [&](int i, uint4 (&to_regs)[U][WORDS]) {
#pragma unroll
            for (int x = 0; x < U; ++x) {
                const int h = (i + x) * HPW + lane / LPH;
                if (i + x < to && h < heads) load8<T>(src + (long long)h * D * E, to_regs[x]);
            }
        };
        fetch(from, raw);
        for (int i = from; i < to; i += U) {
            fetch(i + U, ahead);
#pragma unroll
            for (int x = 0; x < U; ++x) {
                if (i + x >= to) break;
                const int h = (i + x) * HPW + lane / LPH;
                float v[8], o[8], r = 1.f;
                unpack8<T>(raw[x], v);
                if (a.interleaved) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) o[e] = v[e ^ 1];
                } else {
                    uint4 other[WORDS];
#pragma unroll
                    for (int y = 0; y < WORDS; ++y) {
                        other[y].x = __shfl_sync(0xffffffffu, raw[x][y].x, partner, LPH);
                        other[y].y = __shfl_sync(0xffffffffu, raw[x][y].y, partner, LPH);
                        other[y].z = __shfl_sync(0xffffffffu, raw[x][y].z, partner, LPH);
                        other[y].w = __shfl_sync(0xffffffffu, raw[x][y].w, partner, LPH);
                    }
                    unpack8<T>(other, o);
                }
                if (weight) {
                    float sum = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum = fmaf(v[e], v[e], sum);
#pragma unroll
                    for (int d = 1; d < LPH; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
                    r = __frsqrt_rn(sum * (1.f / D) + a.eps);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= cw[e];
                if (turned) {                        // what is not takes nothing from another value, be it infinite
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = fmaf(o[e], sw[e], v[e]);
                }
                if (weight) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] *= r;
                }
                if (h < heads) store8<T>(dst + h * step, v);
            }
#pragma unroll
            for (int x = 0; x < U; ++x)
#pragma unroll
                for (int y = 0; y < WORDS; ++y) raw[x][y] = ahead[x][y];
        }
    };
    // heads that are stored as they are
    auto copy_heads = [&](int which, int from, int to) {
        if (page < 0) return;
        const uint8_t* src = (which ? a.v : a.k) + ((long long)row * (which ? a.ld_v : a.ld_k) + l * 8) * E;
        uint8_t* dst = const_cast<uint8_t*>(a.c.pool[which]) + (paged_offset(a.c, page, 0, slot_position) + l * 8) * E;
        for (int i = from; i < to; i += U) {
            uint4 raw[U][WORDS];
#pragma unroll
            for (int x = 0; x < U; ++x) {
                const int h = (i + x) * HPW + lane / LPH;
                if (i + x < to && h < a.H) load8<T>(src + (long long)h * D * E, raw[x]);
            }
#pragma unroll
            for (int x = 0; x < U; ++x) {
                const int h = (i + x) * HPW + lane / LPH;
                if (i + x < to && h < a.H) {
#pragma unroll
                    for (int y = 0; y < WORDS; ++y) reinterpret_cast<uint4*>(dst + h * a.c.head_stride * E)[y] = raw[x][y];
                }
            }
        }
    };
    if (first < rounds_q) turn_heads(0, first, end < rounds_q ? end : rounds_q);
    const int k0 = first > rounds_q ? first - rounds_q : 0, k1 = end - rounds_q < rounds_h ? end - rounds_q : rounds_h;
    if (k0 < k1) {
        if (APPEND && !a.rot) copy_heads(0, k0, k1);
        else turn_heads(1, k0, k1);
    }
    if (APPEND) {
        const int v0 = first > rounds_q + rounds_h ? first - rounds_q - rounds_h : 0, v1 = end - rounds_q - rounds_h;
        if (v0 < v1) copy_heads(1, v0, v1);
    }
    let_next_start();
}

template <typename T, int D, bool APPEND>
static coreinfer_status launch_rope(RopeArgs& a, const DeviceInfo& di, cudaStream_t st)
{
    constexpr int HPW = 256 / D;
    // a warp per token, or as many as bring 16 to every SM, but not more than there are rounds of heads
    const int rounds = (a.Hq + HPW - 1) / HPW + (APPEND ? 2 : 1) * ((a.H + HPW - 1) / HPW);
    long long split = (16LL * di.sm_count + a.tokens - 1) / a.tokens;
    if (split > rounds) split = rounds;
    a.split = (int)split;
    const long long warps = a.tokens * split;
    CI_CUDA(launch_overlapped(rope_kernel<T, D, APPEND>, dim3((unsigned)((warps + kRopeWarps - 1) / kRopeWarps)), dim3(32 * kRopeWarps), 0, st, a));
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
    return launch_typed<true>(a, dtype, D, (cudaStream_t)cuda_stream);
}

}  // extern "C"
