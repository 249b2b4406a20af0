// The 4-bit storage format shared by the weight matrices and the key/value cache (include/coreinfer.h
// section (7)): codes in units of two bytes, one fp16 pair (s, o) per group, x^ = s c + o.
#pragma once

#include "common.cuh"

#include <atomic>

namespace coreinfer {

constexpr float kHalfMax = 65504.f;

static inline bool group_known(int g) { return g == 32 || g == 64 || g == 128; }
static inline bool aligned_to(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

#ifdef __CUDACC__

// Dynamic shared memory that a kernel may ask for beside `fixed` bytes (1 KB unless said) for its static part.
static inline size_t smem_room(const DeviceInfo& di, int fixed = 1024) { return (size_t)di.smem_optin - fixed; }
// Lets a kernel use that much; once per kernel and device, since the call costs about a microsecond of host time.
template <auto Kernel>
static coreinfer_status allow_smem(const DeviceInfo& di, int fixed = 1024)
{
    static std::atomic<unsigned long long> done{0};
    const unsigned long long bit = di.device >= 0 && di.device < 64 ? 1ull << di.device : 0ull;
    if (done.load(std::memory_order_relaxed) & bit) return COREINFER_OK;
    CI_CUDA(cudaFuncSetAttribute(Kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_room(di, fixed)));
    done.fetch_or(bit, std::memory_order_relaxed);
    return COREINFER_OK;
}

// A launch that may begin while the kernel before it on the stream still runs: its blocks get ready and wait
// (griddepcontrol.wait) before they touch global memory, so the order of results is that of the stream.  `cluster`: CTAs
// per cluster along x.
template <typename Args>
static cudaError_t launch_overlapped(void (*kernel)(const Args), dim3 grid, dim3 block, size_t smem, cudaStream_t st, const Args& args, int cluster = 1)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, args);
}
__device__ __forceinline__ void wait_for_stream() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// The next kernel of the stream may get its blocks ready.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// Typed views of the three storage types.
template <typename T> __device__ __forceinline__ float to_f32(T v);
template <> __device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f32<__half>(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// The eight values of one (16-bit types) or two 16-byte words.
template <typename T>
__device__ __forceinline__ void unpack8(const uint4* raw, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
        const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if constexpr (sizeof(T) == 4) v[4 * i + e] = __uint_as_float(w[e]);
            else {
                v[2 * e] = to_f32<T>(*reinterpret_cast<const T*>(&w[e]));
                const uint32_t high = w[e] >> 16;
                v[2 * e + 1] = to_f32<T>(*reinterpret_cast<const T*>(&high));
            }
        }
    }
}

// Byte of the unit that holds values v .. v + 3 (v a multiple of 4) of a row piece of 32 H values.
__device__ __forceinline__ int unit_offset(int v, int H) { return 2 * (((v & 31) >> 2) * H + (v >> 5)); }

// Minimum and maximum that hand a NaN on.
__device__ __forceinline__ float min_nan(float a, float b)
{
    float r;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
// Over the `lanes` consecutive lanes (a power of two) of a group.
__device__ __forceinline__ void group_range(float& lo, float& hi, int lanes)
{
    for (int d = 1; d < lanes; d <<= 1) {
        lo = min_nan(lo, __shfl_xor_sync(0xffffffffu, lo, d));
        hi = max_nan(hi, __shfl_xor_sync(0xffffffffu, hi, d));
    }
}

// The pair of a group from its range (NaN both where the group holds one).  Every step is one correctly
// rounded operation, so the format is a function of the values alone, whoever computes it.
struct QuantPair {
    __half s, o;
};
__device__ __forceinline__ QuantPair quant_pair(float lo, float hi)
{
    QuantPair p;
    p.o = __float2half_rn(fminf(fmaxf(lo, -kHalfMax), kHalfMax));
    p.s = __float2half_rn(min_nan(__fmul_rn(__fsub_rn(hi, lo), 1.f / 15.f), kHalfMax));
    if (lo != lo) p.s = p.o = __ushort_as_half((unsigned short)0x7fff);
    return p;
}
// Codes of N values in one unit or several: clamp(round((x - o) / s), 0, 15), 0 where s is 0 or NaN.  The quotients
// come from a reciprocal, good to 2^-22 of at most 15.5 (4e-6); adding 3 * 2^22 rounds them, ties to even, and leaves
// the code in the low bits.  A quotient within 1e-5 of a tie between two codes could round to the other one, so the
// values then go through the division.  units[i] gets four codes; c the codes as numbers.
constexpr float kRoundMagic = 12582912.f;
__device__ __forceinline__ float clamp15(float q) { return fminf(fmaxf(q, 0.f), 15.f); }
template <int N>
__device__ __forceinline__ void quant_codes(const float (&x)[N], float s, float o, unsigned (&units)[N / 4], float (&c)[N])
{
    float r = 0.f;
    if (s > 0.f) asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(s));
    unsigned bits[N];
    bool close = false;
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const float q = clamp15(__fsub_rn(x[e], o) * r), t = q + kRoundMagic;
        bits[e] = __float_as_uint(t);
        c[e] = t - kRoundMagic;
        close |= fabsf(q - c[e]) > 0.49999f;
    }
    if (close) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float t = clamp15(__fdiv_rn(__fsub_rn(x[e], o), s)) + kRoundMagic;
            bits[e] = __float_as_uint(t);
            c[e] = t - kRoundMagic;
        }
    }
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
        unsigned u = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) u |= (bits[4 * i + e] & 15u) << (4 * e);
        units[i] = u;
    }
}

// ---- codes as matrix operands ----
// Four bits masked into the low end of a 16-bit lane ARE an fp16 number: the subnormal c * 2^-24 (bits 0-3)
// or c * 2^-20 (bits 4-7), exact, and mma takes fp16 subnormals at their value.  One AND therefore turns
// two codes into a pair of operands; the factor 2^24 (2^20) is applied to the fp32 sums.  The MMA lines products up by exponent
// fields, a subnormal's being that of 2^-14, and cuts off some 2^-24 below the largest: products of a code are cut at about 2^-18
// of the largest one's size unless they are multiples of a step above that (round_to).
constexpr float kCodeScaleLow = 16777216.f;     // 2^24
constexpr float kCodeScaleHigh = 1048576.f;     // 2^20

__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// The same with C = 0.
__device__ __forceinline__ void mma_16816_zero(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}

__device__ __forceinline__ uint32_t pack_half2(float lo, float hi)
{
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
// v rounded to a multiple of `step` (a power of two; |v| < 2^22 steps).  Sums of products of such numbers with codes
// stay whole multiples of the step, which an fp32 accumulator holds exactly up to 2^24 of them; the MMA cuts off, and
// does not round, what lies below its last place.
__device__ __forceinline__ float round_to(float v, float step)
{
    const float middle = 12582912.f * step;
    return __fadd_rn(__fadd_rn(v, middle), -middle);
}
// The two fp16 parts of a v below 2048 steps, together 22 bits of the largest such v.
__device__ __forceinline__ float half_part(float v, float step, int low)
{
    const float high = round_to(v, step);
    return low ? v - high : high;
}
// Exponent x with m = max |v| in [2^(x-1), 2^x), at least -100; 14 where no scaling can help (m = 0, infinite or NaN).
__device__ __forceinline__ int range_exponent(float m)
{
    const int e = (int)(__float_as_uint(m) >> 23) - 126;
    return m == 0.f || e > 128 ? 14 : (e < -100 ? -100 : e);
}
// 2^e for -126 <= e <= 127.
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }
__device__ __forceinline__ float exp2_fast(float v)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ float log2_fast(float v)
{
    float r;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

// The word of the j-th step over a row piece of 32 H values, from the words a lane loads (units 2 tig and 2 tig + 1: H / 2
// words each).  Steps 2 p and 2 p + 1 cover blocks 2 p and 2 p + 1 of 32 values.  In groups of 64 or 128 the words serve as
// they are, a word's two halves being the two blocks: step 2 p takes unit 2 tig, step 2 p + 1 unit 2 tig + 1, and code e of a
// half-word stands for value 8 tig + e (4 more in the second step).  In groups of 32 the two blocks have to stay
// apart: step j takes block j of both units, and code e stands for values 8 tig + e and 8 tig + 4 + e.
template <int G, int H>
__device__ __forceinline__ uint32_t code_word(const uint32_t (&w)[H], int j)
{
    if (G == 32) return __byte_perm(w[j / 2], w[H / 2 + j / 2], j & 1 ? 0x7632 : 0x5410);
    return w[(j & 1) * (H / 2) + j / 2];
}

// ---- copies into shared memory, 16 bytes a thread, complete in groups ----
__device__ __forceinline__ void copy16(uint32_t dst, const void* src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
// The same where `on` is not 0.
__device__ __forceinline__ void copy16_if(uint32_t dst, const void* src, int on)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.s32 p, %2, 0;\n\t@p cp.async.cg.shared.global [%0], [%1], 16;\n\t}" ::"r"(dst), "l"(src), "r"(on)
                 : "memory");
}
// The warp's number, in a form that the compiler knows to be the same for the warp.
__device__ __forceinline__ int warp_number() { return __shfl_sync(0xffffffffu, (int)(threadIdx.x >> 5), 0); }
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Loads by 32-bit shared address (running addresses in one register, offsets in the instruction).
__device__ __forceinline__ uint4 lds128(uint32_t at)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
    return v;
}
__device__ __forceinline__ float2 lds_f32x2(uint32_t at)
{
    float2 v;
    asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(at));
    return v;
}
__device__ __forceinline__ float2 lds_half2(uint32_t at)
{
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(at));
    return __half22float2(*reinterpret_cast<const __half2*>(&v));
}

// ---- the CTAs of a cluster; with one CTA all of this is the block's own ----
__device__ __forceinline__ unsigned cluster_size()
{
    unsigned v;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(v));
    return v;
}
__device__ __forceinline__ unsigned cluster_rank()
{
    unsigned v;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(v));
    return v;
}
__device__ __forceinline__ void cluster_sync(unsigned size)
{
    if (size == 1) {
        __syncthreads();
        return;
    }
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t cluster_address(const void* p, unsigned rank)
{
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(p)), "r"(rank));
    return r;
}
__device__ __forceinline__ void cluster_store(uint32_t at, int v) { asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(at), "r"(v) : "memory"); }
__device__ __forceinline__ void cluster_add(uint32_t at, unsigned v) { asm volatile("red.shared::cluster.add.u32 [%0], %1;" ::"r"(at), "r"(v) : "memory"); }
__device__ __forceinline__ float cluster_load(uint32_t at)
{
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
    return v;
}

#endif  // __CUDACC__

}  // namespace coreinfer
