// Matrix-vector products with 4-bit weights and group scales, and the one-time layout of such weights.
#include "quant4.cuh"

namespace coreinfer {

static inline long long w4_rows16(int N) { return ((long long)N + 15) / 16; }
static inline long long w4_blocks128(int K) { return ((long long)K + 127) / 128; }

// ------------------------------------------------------------------------------ quantise --
// One CTA per 16 rows x 128 columns.  The tile goes through shared memory so that the source is read
// along whichever of its strides is 1; then 32 lanes hold a row's 128 values, four each, and the
// lanes of a group agree on its range by shuffles.
template <typename T>
__global__ void __launch_bounds__(256)
w4_quantize_kernel(const T* __restrict__ w, int N, int K, long long sn, long long sk, int group,
                   uint8_t* __restrict__ codes, __half2* __restrict__ pairs)
{
    __shared__ float tile[16][129];
    const long long kb = blockIdx.x, rt = blockIdx.y;
    const long long KB = gridDim.x;
    const int k0 = (int)(kb * 128), n0 = (int)(rt * 16);
    for (int i = threadIdx.x; i < 16 * 128; i += blockDim.x) {
        const int r = sk == 1 ? i >> 7 : i & 15, c = sk == 1 ? i & 127 : i >> 4;
        const bool in = n0 + r < N && k0 + c < K;
        tile[r][c] = in ? to_f32<T>(w[(long long)(n0 + r) * sn + (long long)(k0 + c) * sk]) : 0.f;
    }
    __syncthreads();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int r = warp; r < 16; r += 8) {
        float x[4], lo = __int_as_float(0x7f800000), hi = -__int_as_float(0x7f800000);
        bool nan = false, any = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[e] = tile[r][lane * 4 + e];
            if (n0 + r < N && k0 + lane * 4 + e < K) {
                lo = fminf(lo, x[e]);
                hi = fmaxf(hi, x[e]);
                nan |= x[e] != x[e];
                any = true;
            }
        }
        const int lanes = group / 4;
        for (int d = 1; d < lanes; d <<= 1) {
            lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, d));
            hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, d));
            nan |= __shfl_xor_sync(0xffffffffu, (int)nan, d) != 0;
            any |= __shfl_xor_sync(0xffffffffu, (int)any, d) != 0;
        }
        QuantPair p = quant_pair(lo, hi, nan);
        if (!any) p.s = p.o = __ushort_as_half((unsigned short)0);      // wholly beyond the matrix
        const float s = __half2float(p.s), o = __half2float(p.o);
        unsigned unit = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (k0 + lane * 4 + e < K && n0 + r < N) unit |= quant_code(x[e], s, o) << (4 * e);
        uint8_t* row = codes + (((size_t)rt * KB + kb) * 16 + r) * 64;
        *reinterpret_cast<uint16_t*>(row + unit_offset(lane * 4, 4)) = (uint16_t)unit;
        if ((lane & (lanes - 1)) == 0) {
            const size_t per = 128 / group;
            pairs[(((size_t)rt * KB + kb) * per + lane / lanes) * 16 + r] = __halves2half2(p.s, p.o);
        }
    }
}

// -------------------------------------------------------------------------------- matvec --
struct W4Args {
    const uint8_t* codes;
    const __half2* pairs;
    int N, K, group, batch, act;
    const void* x;
    const void* bias;
    const void* mul;
    void* y;
    long long ld_x, ld_mul, ld_y;
};

__device__ __forceinline__ float w4_act(float v, int act)
{
    if (act == COREINFER_ACT_RELU) return fmaxf(v, 0.f);
    if (act == COREINFER_ACT_SILU) return v / (1.f + __expf(-v));
    return v;
}

// One warp per output and row of x.
template <typename T, typename Y>
__global__ void __launch_bounds__(256) w4_matvec_kernel(W4Args a)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int n = blockIdx.x * 8 + warp, b = blockIdx.y;
    if (n >= a.N) return;
    const int KB = (a.K + 127) / 128, per = 128 / a.group;
    const T* x = (const T*)a.x + (long long)b * a.ld_x;
    float acc = 0.f;
    for (int kb = 0; kb < KB; ++kb) {
        const size_t tile = (size_t)(n >> 4) * KB + kb;
        const uint8_t* row = a.codes + (tile * 16 + (n & 15)) * 64;
        const unsigned unit = *reinterpret_cast<const uint16_t*>(row + unit_offset(lane * 4, 4));
        const __half2 p = a.pairs[(tile * per + lane * 4 / a.group) * 16 + (n & 15)];
        const float s = __low2float(p), o = __high2float(p);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int k = kb * 128 + lane * 4 + e;
            if (k < a.K) acc = fmaf(to_f32<T>(x[k]), fmaf(s, (float)((unit >> (4 * e)) & 15u), o), acc);
        }
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, d);
    if (lane == 0) {
        if (a.bias) acc += to_f32<T>(((const T*)a.bias)[n]);
        acc = w4_act(acc, a.act);
        if (a.mul) acc *= to_f32<Y>(((const Y*)a.mul)[(long long)b * a.ld_mul + n]);
        ((Y*)a.y)[(long long)b * a.ld_y + n] = from_f32<Y>(acc);
    }
}

template <typename T, typename Y>
static void launch_matvec(const W4Args& a, cudaStream_t st)
{
    w4_matvec_kernel<T, Y><<<dim3((a.N + 7) / 8, a.batch), 256, 0, st>>>(a);
}

}  // namespace coreinfer

using namespace coreinfer;

extern "C" {

size_t coreinfer_w4_codes_bytes(int32_t N, int32_t K)
{
    if (N < 1 || K < 1) return 0;
    return (size_t)w4_rows16(N) * (size_t)w4_blocks128(K) * 1024;
}

size_t coreinfer_w4_pairs_bytes(int32_t N, int32_t K, int32_t group)
{
    if (N < 1 || K < 1 || !group_known(group)) return 0;
    return (size_t)w4_rows16(N) * (size_t)w4_blocks128(K) * (size_t)(128 / group) * 64;
}

coreinfer_status coreinfer_w4_quantize(const void* w, coreinfer_dtype dtype, int32_t N, int32_t K,
                                       int64_t stride_n, int64_t stride_k, int32_t group,
                                       void* codes, void* pairs, void* cuda_stream)
{
    if (!dtype_known(dtype)) CI_FAIL(COREINFER_ERR_UNSUPPORTED, "dtype %d is not supported", (int)dtype);
    if (!group_known(group)) CI_FAIL(COREINFER_ERR_UNSUPPORTED, "group %d: 32, 64 and 128 are built", group);
    if (N < 1 || K < 1) CI_FAIL(COREINFER_ERR_INVALID_ARG, "N and K must be >= 1");
    if (w4_rows16(N) > 65535) CI_FAIL(COREINFER_ERR_UNSUPPORTED, "N %d: at most %d rows", N, 65535 * 16);
    if (!w || !codes || !pairs || !aligned_to(w, dtype_size(dtype)) || !aligned16(codes) || !aligned16(pairs))
        CI_FAIL(COREINFER_ERR_INVALID_ARG, "w / codes / pairs NULL or misaligned");
    DeviceInfo di;
    const coreinfer_status s = device_info(&di);
    if (s != COREINFER_OK) return s;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const dim3 grid((unsigned)w4_blocks128(K), (unsigned)w4_rows16(N));
    if (dtype == COREINFER_F32)
        w4_quantize_kernel<float><<<grid, 256, 0, st>>>((const float*)w, N, K, stride_n, stride_k, group, (uint8_t*)codes, (__half2*)pairs);
    else if (dtype == COREINFER_BF16)
        w4_quantize_kernel<__nv_bfloat16><<<grid, 256, 0, st>>>((const __nv_bfloat16*)w, N, K, stride_n, stride_k, group, (uint8_t*)codes, (__half2*)pairs);
    else
        w4_quantize_kernel<__half><<<grid, 256, 0, st>>>((const __half*)w, N, K, stride_n, stride_k, group, (uint8_t*)codes, (__half2*)pairs);
    CI_CUDA(cudaGetLastError());
    return COREINFER_OK;
}

coreinfer_status coreinfer_w4_matvec(const coreinfer_w4_matrix* w, const void* x, int32_t batch, int64_t ld_x,
                                     coreinfer_dtype dtype, coreinfer_act act,
                                     const void* bias, const void* mul, int64_t ld_mul,
                                     void* y, coreinfer_dtype y_dtype, int64_t ld_y, void* cuda_stream)
{
    if (!w) CI_FAIL(COREINFER_ERR_INVALID_ARG, "matrix descriptor is NULL");
    if (!dtype_known(dtype)) CI_FAIL(COREINFER_ERR_UNSUPPORTED, "dtype %d is not supported", (int)dtype);
    if (y_dtype != COREINFER_F32 && y_dtype != dtype)
        CI_FAIL(COREINFER_ERR_UNSUPPORTED, "y_dtype %d: fp32 or the type of x", (int)y_dtype);
    if (!group_known(w->group)) CI_FAIL(COREINFER_ERR_UNSUPPORTED, "group %d: 32, 64 and 128 are built", w->group);
    if (act != COREINFER_ACT_NONE && act != COREINFER_ACT_RELU && act != COREINFER_ACT_SILU)
        CI_FAIL(COREINFER_ERR_UNSUPPORTED, "act %d is not supported", (int)act);
    if (batch < 1 || batch > COREINFER_MAX_BATCH)
        CI_FAIL(COREINFER_ERR_UNSUPPORTED, "batch %d: 1..%d are built", batch, COREINFER_MAX_BATCH);
    if (w->N < 1 || w->K < 1) CI_FAIL(COREINFER_ERR_INVALID_ARG, "N and K must be >= 1");
    if (!w->codes || !w->pairs || !aligned16(w->codes) || !aligned16(w->pairs))
        CI_FAIL(COREINFER_ERR_INVALID_ARG, "codes / pairs NULL or not 16-byte aligned");
    const size_t xe = dtype_size(dtype), ye = dtype_size(y_dtype);
    if (!x || !y || !aligned_to(x, xe) || !aligned_to(y, ye) || !aligned_to(bias, xe) || !aligned_to(mul, ye))
        CI_FAIL(COREINFER_ERR_INVALID_ARG, "x or y NULL, or x / y / bias / mul not aligned to their elements");
    if (ld_x < w->K || ld_y < w->N || (mul && ld_mul < w->N))
        CI_FAIL(COREINFER_ERR_INVALID_ARG, "ld_x, ld_y and ld_mul must be at least a row's length");
    DeviceInfo di;
    const coreinfer_status s = device_info(&di);
    if (s != COREINFER_OK) return s;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    W4Args a;
    a.codes = (const uint8_t*)w->codes;
    a.pairs = (const __half2*)w->pairs;
    a.N = w->N;
    a.K = w->K;
    a.group = w->group;
    a.batch = batch;
    a.act = (int)act;
    a.x = x;
    a.bias = bias;
    a.mul = mul;
    a.y = y;
    a.ld_x = ld_x;
    a.ld_mul = ld_mul;
    a.ld_y = ld_y;
    if (dtype == COREINFER_F32) launch_matvec<float, float>(a, st);
    else if (dtype == COREINFER_BF16) {
        if (y_dtype == COREINFER_F32) launch_matvec<__nv_bfloat16, float>(a, st);
        else launch_matvec<__nv_bfloat16, __nv_bfloat16>(a, st);
    } else {
        if (y_dtype == COREINFER_F32) launch_matvec<__half, float>(a, st);
        else launch_matvec<__half, __half>(a, st);
    }
    CI_CUDA(cudaGetLastError());
    return COREINFER_OK;
}

}  // extern "C"
