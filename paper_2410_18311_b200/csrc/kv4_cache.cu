// Appending to and evicting from the 4-bit key/value cache.
#include "kv4.cuh"

namespace coreinfer {

// -------------------------------------------------------------------------------- append --
// One thread per four values of a head (one unit of codes); the lanes of a group agree on its range
// by shuffles.
template <typename T, int GROUP>
__global__ void __launch_bounds__(256)
kv4_append_kernel(Kv4 c, const T* __restrict__ k, const T* __restrict__ v, int tokens, long long ld,
                  T* __restrict__ k_stored, T* __restrict__ v_stored)
{
    const int b = blockIdx.y;
    const int n0 = kv4_length(c, b), seen = c.state[b * 4 + kStateSeen];
    const bool fits = tokens <= c.cap - n0;
    const int quads = c.D / 4;
    const long long per = (long long)tokens * c.H * quads;          // units of keys; as many of values follow
    const long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    if (i < 2 * per) {                                              // whole warps: 2 * H * D / 4 is a multiple of 32
        const int which = i >= per;
        const long long u = which ? i - per : i;
        const int quad = (int)(u % quads);
        const int h = (int)((u / quads) % c.H);
        const int t = (int)(u / quads / c.H);
        const T* src = (which ? v : k) + ((long long)b * tokens + t) * ld + (long long)h * c.D + quad * 4;
        T in[4];
        if (sizeof(T) == 4) *reinterpret_cast<uint4*>(in) = *reinterpret_cast<const uint4*>(src);
        else *reinterpret_cast<uint2*>(in) = *reinterpret_cast<const uint2*>(src);
        float x[4], lo = __int_as_float(0x7f800000), hi = -__int_as_float(0x7f800000);
        bool nan = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[e] = to_f32<T>(in[e]);
            lo = fminf(lo, x[e]);
            hi = fmaxf(hi, x[e]);
            nan |= x[e] != x[e];
        }
        group_range<GROUP / 4>(lo, hi, nan);
        const QuantPair p = quant_pair(lo, hi, nan);
        const float s = __half2float(p.s), o = __half2float(p.o);
        unsigned unit = 0;
        T back[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const unsigned q = quant_code(x[e], s, o);
            unit |= q << (4 * e);
            back[e] = from_f32<T>(fmaf(s, (float)q, o));
        }
        if (fits) {
            const size_t slot = ((size_t)b * c.H + h) * c.cap + n0 + t;
            *reinterpret_cast<uint16_t*>(c.codes[which] + slot * (c.D / 2) + unit_offset(quad * 4, c.D / 32)) = (uint16_t)unit;
            if (quad % (GROUP / 4) == 0) c.pairs[which][slot * (c.D / GROUP) + quad / (GROUP / 4)] = __halves2half2(p.s, p.o);
            if (!which && quad == 0 && c.weight) {
                c.weight[slot] = 0.f;
                c.position[slot] = seen + t;
            }
        }
        T* out = which ? v_stored : k_stored;
        if (out) {
            out += (((long long)b * tokens + t) * c.H + h) * c.D + quad * 4;
            if (sizeof(T) == 4) *reinterpret_cast<uint4*>(out) = *reinterpret_cast<uint4*>(back);
            else *reinterpret_cast<uint2*>(out) = *reinterpret_cast<uint2*>(back);
        }
    }
    if (kv4_last_of_sequence(c, b, gridDim.x)) {
        if (fits) {
            c.state[b * 4 + kStateLength] = n0 + tokens;
            c.state[b * 4 + kStateSeen] = seen + tokens;
        } else {
            c.state[b * 4 + kStateRefused] += tokens;
        }
    }
}

template <typename T>
static coreinfer_status launch_append(const Kv4& c, const void* k, const void* v, int tokens, long long ld, void* ks, void* vs, cudaStream_t st)
{
    const long long units = 2LL * tokens * c.H * (c.D / 4);
    const dim3 grid((unsigned)((units + 255) / 256), (unsigned)c.B);
    auto go = [&](auto kernel) { kernel<<<grid, 256, 0, st>>>(c, (const T*)k, (const T*)v, tokens, ld, (T*)ks, (T*)vs); };
    if (c.G == 32) go(kv4_append_kernel<T, 32>);
    else if (c.G == 64) go(kv4_append_kernel<T, 64>);
    else go(kv4_append_kernel<T, 128>);
    CI_CUDA(cudaGetLastError());
    return COREINFER_OK;
}

// --------------------------------------------------------------------------------- evict --
constexpr int kEvictThreads = 1024;

// Order of eviction as an unsigned number: kept for certain > larger weight > smaller weight > NaN.
__device__ __forceinline__ unsigned evict_key(float w, int pos, int seen, int recent, int first)
{
    if (pos >= seen - recent || pos < first) return 0xffffffffu;
    if (w != w) return 0u;
    const unsigned u = __float_as_uint(w + 0.f);                    // -0 counts as 0
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ int block_scan_excl(int v, int* warp_tot, int* total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int incl = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += t;
    }
    if (lane == 31) warp_tot[warp] = incl;
    __syncthreads();
    if (warp == 0) {
        int w = warp_tot[lane];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int t = __shfl_up_sync(0xffffffffu, w, o);
            if (lane >= o) w += t;
        }
        warp_tot[lane] = w;
    }
    __syncthreads();
    const int base = warp > 0 ? warp_tot[warp - 1] : 0;
    *total = warp_tot[31];
    __syncthreads();
    return base + incl - v;
}

// Copies one slot, `lane` of 32.
__device__ __forceinline__ void move_slot(const Kv4& a, size_t from, const Kv4& z, size_t to, int lane)
{
    const int words = a.D / 8, groups = a.D / a.G;                  // of codes per row
    for (int w = 0; w < 2; ++w) {
        const unsigned* s = reinterpret_cast<const unsigned*>(a.codes[w] + from * (a.D / 2));
        unsigned* d = reinterpret_cast<unsigned*>(z.codes[w] + to * (a.D / 2));
        for (int i = lane; i < words; i += 32) d[i] = s[i];
        for (int i = lane; i < groups; i += 32) z.pairs[w][to * groups + i] = a.pairs[w][from * groups + i];
    }
    if (lane == 0) {
        z.weight[to] = a.weight[from];
        z.position[to] = a.position[from];
    }
}

// One CTA per sequence and head: the key of the last slot that stays by four 8-bit digits, then the lists
// of slots that move, then the moves.
__global__ void __launch_bounds__(kEvictThreads)
kv4_evict_kernel(Kv4 a, Kv4 z, int in_place, int budget, int recent, int first, int32_t* lists)
{
    __shared__ unsigned hist[256];
    __shared__ int warp_tot[32];
    __shared__ unsigned prefix_s;
    __shared__ int left_s;
    const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
    const int n = kv4_length(a, b), seen = a.state[b * 4 + kStateSeen];
    const int keep = n < budget ? n : budget;
    const size_t base = ((size_t)b * a.H + h) * a.cap, zbase = ((size_t)b * a.H + h) * z.cap;
    int32_t* list = lists + base;
    auto key = [&](int i) { return evict_key(a.weight[base + i], a.position[base + i], seen, recent, first); };

    unsigned prefix = 0;
    int left = keep;                                                // slots still to be taken among those that match the prefix
    if (keep > 0 && keep < n) {
        for (int shift = 24; shift >= 0; shift -= 8) {
            if (tid < 256) hist[tid] = 0;
            __syncthreads();
            const unsigned mask = shift == 24 ? 0u : 0xffffffffu << (shift + 8);
            for (int i = tid; i < n; i += blockDim.x) {
                const unsigned u = key(i);
                if ((u & mask) == prefix) atomicAdd(&hist[(u >> shift) & 255u], 1u);
            }
            __syncthreads();
            if (tid == 0) {
                int d = 255, acc = 0;
                while (d > 0 && acc + (int)hist[d] < left) acc += hist[d--];
                prefix_s = prefix | ((unsigned)d << shift);
                left_s = left - acc;
            }
            __syncthreads();
            prefix = prefix_s;
            left = left_s;
        }
    }
    // the slots with a larger key stay, and the first `left` of those with this key
    int ties = 0, movers = 0, holes = 0;
    for (int i0 = 0; i0 < n; i0 += blockDim.x) {
        const int i = i0 + tid;
        const unsigned u = i < n ? key(i) : 0u;
        const bool all = keep == n;
        const int tie = i < n && !all && u == prefix;
        int tot;
        const int rank = ties + block_scan_excl(tie, warp_tot, &tot);
        ties += tot;
        const bool stays = i < n && keep > 0 && (all || u > prefix || (tie && rank < left));
        const int mover = in_place ? stays && i >= keep : stays;
        const int m = movers + block_scan_excl(mover, warp_tot, &tot);
        movers += tot;
        const int hole = in_place && i < keep && !stays;
        const int e = holes + block_scan_excl(hole, warp_tot, &tot);
        holes += tot;
        if (mover) list[in_place ? a.cap / 2 + m : m] = i;
        if (hole) list[e] = i;
    }
    __syncthreads();
    for (int m = tid >> 5; m < movers; m += blockDim.x >> 5) {
        const int from = list[in_place ? a.cap / 2 + m : m], to = in_place ? list[m] : m;
        move_slot(a, base + from, z, zbase + to, tid & 31);
    }
    if (kv4_last_of_sequence(a, b, gridDim.x)) {
        z.state[b * 4 + kStateLength] = keep;
        z.state[b * 4 + kStateSeen] = seen;
    }
}

}  // namespace coreinfer

using namespace coreinfer;

extern "C" {

coreinfer_status coreinfer_kv4_append(const coreinfer_kv4_cache* cache, const void* k, const void* v,
                                      coreinfer_dtype dtype, int32_t T, int64_t ld_token,
                                      void* k_stored, void* v_stored, void* cuda_stream)
{
    Kv4 c;
    coreinfer_status s = kv4_take(cache, "the", &c);
    if (s != COREINFER_OK) return s;
    if (!dtype_known(dtype)) CI_FAIL(COREINFER_ERR_UNSUPPORTED, "dtype %d is not supported", (int)dtype);
    if (T < 1) CI_FAIL(COREINFER_ERR_INVALID_ARG, "T must be >= 1");
    if (!k || !v || !aligned16(k) || !aligned16(v)) CI_FAIL(COREINFER_ERR_INVALID_ARG, "k / v NULL or not 16-byte aligned");
    if (ld_token < (int64_t)c.H * c.D || (ld_token * (int64_t)dtype_size(dtype)) % 16 != 0)
        CI_FAIL(COREINFER_ERR_INVALID_ARG, "ld_token must cover kv_heads * head_dim elements and be a multiple of 16 bytes");
    if ((k_stored == nullptr) != (v_stored == nullptr) || !aligned16(k_stored) || !aligned16(v_stored))
        CI_FAIL(COREINFER_ERR_INVALID_ARG, "k_stored and v_stored come both (16-byte aligned) or neither");
    if ((long long)T * c.H > (1LL << 30)) CI_FAIL(COREINFER_ERR_UNSUPPORTED, "T %d: too many tokens for one call", T);
    DeviceInfo di;
    if ((s = device_info(&di)) != COREINFER_OK) return s;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (dtype == COREINFER_F32) return launch_append<float>(c, k, v, T, ld_token, k_stored, v_stored, st);
    if (dtype == COREINFER_BF16) return launch_append<__nv_bfloat16>(c, k, v, T, ld_token, k_stored, v_stored, st);
    return launch_append<__half>(c, k, v, T, ld_token, k_stored, v_stored, st);
}

size_t coreinfer_kv4_evict_workspace_bytes(const coreinfer_kv4_cache* src)
{
    Kv4 c;
    if (kv4_take(src, "the source", &c) != COREINFER_OK) return 0;
    return (size_t)c.B * c.H * c.cap * sizeof(int32_t);
}

coreinfer_status coreinfer_kv4_evict(const coreinfer_kv4_cache* src, const coreinfer_kv4_cache* dst,
                                     int32_t budget, int32_t recent, int32_t first,
                                     void* workspace, size_t workspace_bytes, void* cuda_stream)
{
    Kv4 a, z;
    coreinfer_status s = kv4_take(src, "the source", &a);
    if (s != COREINFER_OK || (s = kv4_take(dst, "the destination", &z)) != COREINFER_OK) return s;
    if (!a.weight || !z.weight) CI_FAIL(COREINFER_ERR_INVALID_ARG, "eviction needs caches with weight and position");
    if (budget < 1 || recent < 0 || first < 0 || (long long)recent + first > budget)
        CI_FAIL(COREINFER_ERR_INVALID_ARG, "budget %d must be >= 1 and hold recent %d + first %d", budget, recent, first);
    if (a.B != z.B || a.H != z.H || a.D != z.D || a.G != z.G)
        CI_FAIL(COREINFER_ERR_INVALID_ARG, "the two caches differ in batch, kv_heads, head_dim or group");
    int same = 0;
    for (int w = 0; w < 2; ++w) same += (a.codes[w] == z.codes[w]) + (a.pairs[w] == z.pairs[w]);
    same += (a.state == z.state) + (a.weight == z.weight) + (a.position == z.position);
    if (same != 0 && (same != 7 || a.cap != z.cap))
        CI_FAIL(COREINFER_ERR_INVALID_ARG, "the two caches share some buffers: all (in place) or none");
    if (z.cap < (budget < a.cap ? budget : a.cap))
        CI_FAIL(COREINFER_ERR_INVALID_ARG, "the destination holds %d slots, %d may be kept", z.cap, budget < a.cap ? budget : a.cap);
    if (!workspace || !aligned16(workspace)) CI_FAIL(COREINFER_ERR_WORKSPACE, "workspace is NULL or misaligned");
    const size_t need = coreinfer_kv4_evict_workspace_bytes(src);
    if (workspace_bytes < need) CI_FAIL(COREINFER_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", workspace_bytes, need);
    DeviceInfo di;
    if ((s = device_info(&di)) != COREINFER_OK) return s;
    kv4_evict_kernel<<<dim3(a.H, a.B), kEvictThreads, 0, (cudaStream_t)cuda_stream>>>(a, z, same == 7, budget, recent, first,
                                                                                      (int32_t*)workspace);
    CI_CUDA(cudaGetLastError());
    return COREINFER_OK;
}

}  // extern "C"
