// Attention of a few new tokens over the 4-bit key/value cache.
#include "kv4.cuh"

namespace coreinfer {

struct AttnArgs {
    Kv4 c;
    const void* q;
    void* out;
    long long ld_q, ld_out;
    int Hq, T;
    float scale;
    float* logits;          // [B][T][Hq][cap]
};

__device__ __forceinline__ float kv4_value(const Kv4& c, int which, size_t slot, int d)
{
    const unsigned unit = *reinterpret_cast<const uint16_t*>(c.codes[which] + slot * (c.D / 2) + unit_offset(d & ~3, c.D / 32));
    const __half2 p = c.pairs[which][slot * (c.D / c.G) + d / c.G];
    return fmaf(__low2float(p), (float)((unit >> (4 * (d & 3))) & 15u), __high2float(p));
}

// One CTA per token and query head.
template <typename T>
__global__ void __launch_bounds__(256) kv4_attention_kernel(AttnArgs a)
{
    __shared__ float q[256], red[8];
    const int qh = blockIdx.x, t = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const Kv4& c = a.c;
    const int h = qh / (a.Hq / c.H);
    const int n = kv4_length(c, b) - (a.T - 1 - t);
    const size_t base = ((size_t)b * c.H + h) * c.cap;
    float* lg = a.logits + (((size_t)b * a.T + t) * a.Hq + qh) * c.cap;
    if (tid < c.D) q[tid] = to_f32<T>(((const T*)a.q)[((long long)b * a.T + t) * a.ld_q + (long long)qh * c.D + tid]) * a.scale;
    __syncthreads();
    float top = -__int_as_float(0x7f800000);
    for (int i = warp; i < n; i += 8) {
        float s = 0.f;
        for (int d = lane; d < c.D; d += 32) s = fmaf(q[d], kv4_value(c, 0, base + i, d), s);
#pragma unroll
        for (int e = 16; e; e >>= 1) s += __shfl_xor_sync(0xffffffffu, s, e);
        if (lane == 0) lg[i] = s;
        top = fmaxf(top, s);
    }
    if (lane == 0) red[warp] = top;
    __syncthreads();
    for (int i = 0; i < 8; ++i) top = fmaxf(top, red[i]);
    __syncthreads();
    float sum = 0.f;
    for (int i = tid; i < n; i += 256) {
        const float p = expf(lg[i] - top);
        lg[i] = p;
        sum += p;
    }
#pragma unroll
    for (int e = 16; e; e >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, e);
    if (lane == 0) red[warp] = sum;
    __syncthreads();
    sum = 0.f;
    for (int i = 0; i < 8; ++i) sum += red[i];
    for (int i = tid; i < c.cap; i += 256) lg[i] = i < n ? lg[i] / sum : 0.f;
    __syncthreads();
    if (tid < c.D) {
        float o = 0.f;
        for (int i = 0; i < n; ++i) o = fmaf(lg[i], kv4_value(c, 1, base + i, tid), o);
        ((T*)a.out)[((long long)b * a.T + t) * a.ld_out + (long long)qh * c.D + tid] = from_f32<T>(o);
    }
}

__global__ void kv4_accumulate_kernel(AttnArgs a)
{
    const Kv4& c = a.c;
    const int i = blockIdx.x * blockDim.x + threadIdx.x, h = blockIdx.y, b = blockIdx.z, share = a.Hq / c.H;
    if (i >= kv4_length(c, b)) return;
    float w = 0.f;
    for (int t = 0; t < a.T; ++t)
        for (int g = 0; g < share; ++g) w += a.logits[(((size_t)b * a.T + t) * a.Hq + h * share + g) * c.cap + i];
    c.weight[((size_t)b * c.H + h) * c.cap + i] += w;
}

}  // namespace coreinfer

using namespace coreinfer;

extern "C" {

size_t coreinfer_kv4_attention_workspace_bytes(const coreinfer_kv4_cache* cache, int32_t q_heads, int32_t T)
{
    Kv4 c;
    if (kv4_take(cache, "the", &c) != COREINFER_OK) return 0;
    if (q_heads < 1 || T < 1 || q_heads % c.H != 0 || T > COREINFER_KV4_MAX_QUERIES) return 0;
    return (size_t)c.B * T * q_heads * c.cap * sizeof(float);
}

coreinfer_status coreinfer_kv4_attention(const coreinfer_kv4_cache* cache, const void* q, coreinfer_dtype dtype,
                                         int32_t q_heads, int32_t T, int64_t ld_q, float scale,
                                         void* out, int64_t ld_out, int32_t accumulate,
                                         void* workspace, size_t workspace_bytes, void* cuda_stream)
{
    AttnArgs a;
    coreinfer_status s = kv4_take(cache, "the", &a.c);
    if (s != COREINFER_OK) return s;
    if (!dtype_known(dtype)) CI_FAIL(COREINFER_ERR_UNSUPPORTED, "dtype %d is not supported", (int)dtype);
    if (T < 1 || T > COREINFER_KV4_MAX_QUERIES)
        CI_FAIL(COREINFER_ERR_UNSUPPORTED, "T %d: 1..%d tokens a sequence", T, COREINFER_KV4_MAX_QUERIES);
    if (q_heads < 1 || q_heads % a.c.H != 0)
        CI_FAIL(COREINFER_ERR_INVALID_ARG, "q_heads %d is not a multiple of kv_heads %d", q_heads, a.c.H);
    if (q_heads > 65535) CI_FAIL(COREINFER_ERR_UNSUPPORTED, "q_heads %d: at most 65535", q_heads);
    if (!q || !out || !aligned16(q) || !aligned16(out)) CI_FAIL(COREINFER_ERR_INVALID_ARG, "q / out NULL or not 16-byte aligned");
    const int64_t row = (int64_t)q_heads * a.c.D, e = (int64_t)dtype_size(dtype);
    if (ld_q < row || ld_out < row || (ld_q * e) % 16 != 0 || (ld_out * e) % 16 != 0)
        CI_FAIL(COREINFER_ERR_INVALID_ARG, "ld_q and ld_out must cover q_heads * head_dim elements and be multiples of 16 bytes");
    if (accumulate && !a.c.weight) CI_FAIL(COREINFER_ERR_INVALID_ARG, "accumulate needs a cache with weight and position");
    if (!(scale == scale) || scale - scale != 0.f) CI_FAIL(COREINFER_ERR_INVALID_ARG, "scale is not a finite number");
    if (!workspace || !aligned16(workspace)) CI_FAIL(COREINFER_ERR_WORKSPACE, "workspace is NULL or misaligned");
    const size_t need = coreinfer_kv4_attention_workspace_bytes(cache, q_heads, T);
    if (workspace_bytes < need) CI_FAIL(COREINFER_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", workspace_bytes, need);
    DeviceInfo di;
    if ((s = device_info(&di)) != COREINFER_OK) return s;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    a.q = q;
    a.out = out;
    a.ld_q = ld_q;
    a.ld_out = ld_out;
    a.Hq = q_heads;
    a.T = T;
    a.scale = scale;
    a.logits = (float*)workspace;
    const dim3 grid(q_heads, T, a.c.B);
    if (dtype == COREINFER_F32) kv4_attention_kernel<float><<<grid, 256, 0, st>>>(a);
    else if (dtype == COREINFER_BF16) kv4_attention_kernel<__nv_bfloat16><<<grid, 256, 0, st>>>(a);
    else kv4_attention_kernel<__half><<<grid, 256, 0, st>>>(a);
    CI_CUDA(cudaGetLastError());
    if (accumulate) {
        kv4_accumulate_kernel<<<dim3((a.c.cap + 255) / 256, a.c.H, a.c.B), 256, 0, st>>>(a);
        CI_CUDA(cudaGetLastError());
    }
    return COREINFER_OK;
}

}  // extern "C"
