// Matrix-vector products with 4-bit weights and group scales, and the one-time layout of such weights.
#include "quant4.cuh"

#include <type_traits>

namespace coreinfer {

static inline long long w4_rows16(int N) { return ((long long)N + 15) / 16; }
static inline long long w4_blocks128(int K) { return ((long long)K + 127) / 128; }

// Eight entries of a row from column k on as they are in memory, zeros beyond K.
template <typename T>
__device__ __forceinline__ void load_x8(const T* row, int k, int K, int vec, uint4 (&raw)[sizeof(T) / 2])
{
    if (vec && k + 8 <= K) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) raw[i] = reinterpret_cast<const uint4*>(row + k)[i];
    } else {
        T v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = k + e < K ? row[k + e] : from_f32<T>(0.f);
        uint32_t w[2 * sizeof(T)];
#pragma unroll
        for (int i = 0; i < (int)(2 * sizeof(T)); ++i) {
            if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(to_f32<T>(v[i]));
            else w[i] = *reinterpret_cast<uint16_t*>(&v[2 * i]) | (uint32_t)*reinterpret_cast<uint16_t*>(&v[2 * i + 1]) << 16;
        }
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) raw[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    }
}

// ------------------------------------------------------------------------------ quantise --
// A lane holds eight consecutive columns of a row, 16 lanes a row's block of 128; the lanes of a group agree on its range
// by shuffles, and neighbouring blocks of 32 exchange a unit so that codes are stored in words.  Work is done once per
// matrix (per sentence for the core neurons' weights); it is bound by instructions (36864 x 9216 bf16 290 us, 2960 GB/s; with
// four values a lane, read one by one through shared memory, 1008 us).  ROWS: columns are contiguous and a CTA walks kQuantSteps column blocks of 16 rows.  Otherwise (a transposed
// view, the compacted down projection) a CTA brings 64 rows x 128 columns through shared memory, reading along the rows.
constexpr int kQuantSteps = 4;

template <typename T, int G>
__device__ __forceinline__ void w4_quantize_lane(float (&x)[8], int n, int k, int N, int K, long long block, int r, int l,
                                                 uint8_t* __restrict__ codes, __half2* __restrict__ pairs)
{
    constexpr int GL = G / 8;
    const int have = n < N ? K - k : 0;                      // columns of this lane and beyond that the matrix has
    float lo = x[0], hi = x[0];
    if (have >= 8) {
#pragma unroll
        for (int e = 1; e < 8; ++e) {
            lo = min_nan(lo, x[e]);
            hi = max_nan(hi, x[e]);
        }
    } else {
        lo = __int_as_float(0x7f800000);
        hi = -lo;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < have) {
                lo = min_nan(lo, x[e]);
                hi = max_nan(hi, x[e]);
            }
    }
    group_range(lo, hi, GL);
    QuantPair p = quant_pair(lo, hi);
    if (have + (l & (GL - 1)) * 8 <= 0 || n >= N) p.s = p.o = __ushort_as_half((unsigned short)0);       // a group wholly beyond the matrix
    unsigned unit[2];
    float c[8];
    quant_codes<8>(x, __half2float(p.s), __half2float(p.o), unit, c);
    if (have < 8) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e >= have) unit[e >> 2] &= ~(15u << (4 * (e & 3)));
    }
    const int h = l >> 2, odd = h & 1;
    const unsigned got = __shfl_xor_sync(0xffffffffu, odd ? unit[0] : unit[1], 4);
    const unsigned word = odd ? got | unit[1] << 16 : unit[0] | got << 16;
    *reinterpret_cast<unsigned*>(codes + (block * 16 + r) * 64 + 2 * ((2 * (l & 3) + odd) * 4 + (h & ~1))) = word;
    if ((l & (GL - 1)) == 0) pairs[(block * (128 / G) + l / GL) * 16 + r] = __halves2half2(p.s, p.o);
}

struct W4QuantArgs {
    const void* w;
    int N, K;
    long long sn, sk;       // strides of a row and of a column
    int vec;                // rows are 16-byte aligned
    uint8_t* codes;
    __half2* pairs;
};

template <typename T, int G, bool ROWS>
__global__ void __launch_bounds__(256) w4_quantize_kernel(const __grid_constant__ W4QuantArgs a)
{
    const int N = a.N, K = a.K, KB = (K + 127) / 128, l = threadIdx.x & 15;
    const T* const w = (const T*)a.w;
    wait_for_stream();
    let_next_start();
    if constexpr (ROWS) {
        const int r = threadIdx.x >> 4, rt = blockIdx.y, n = rt * 16 + r;
        const T* row = w + (long long)(n < N ? n : N - 1) * a.sn;
        const int kb0 = blockIdx.x * kQuantSteps, kb1 = kb0 + kQuantSteps < KB ? kb0 + kQuantSteps : KB;
        uint4 raw[sizeof(T) / 2];
        load_x8<T>(row, kb0 * 128 + l * 8, K, a.vec, raw);
        for (int kb = kb0; kb < kb1; ++kb) {
            float x[8];
            unpack8<T>(raw, x);
            if (kb + 1 < kb1) load_x8<T>(row, (kb + 1) * 128 + l * 8, K, a.vec, raw);
            w4_quantize_lane<T, G>(x, n, kb * 128 + l * 8, N, K, (long long)rt * KB + kb, r, l, a.codes, a.pairs);
        }
    } else {
        constexpr int PITCH = 128 + 4 / sizeof(T);           // an odd number of words
        __shared__ T tile[64 * PITCH];
        const int k0 = blockIdx.x * 128, n0 = blockIdx.y * 64, tn = threadIdx.x & 63, tk = threadIdx.x >> 6;
        const T* src = w + (long long)(n0 + tn < N ? n0 + tn : N - 1) * a.sn;
#pragma unroll 8
        for (int k = tk; k < 128; k += 4) tile[tn * PITCH + k] = src[(long long)(k0 + k < K ? k0 + k : K - 1) * a.sk];
        __syncthreads();
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int r = threadIdx.x >> 4, n = n0 + q * 16 + r;
            if (n0 + q * 16 >= N) break;
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = to_f32<T>(tile[(q * 16 + r) * PITCH + l * 8 + e]);
            w4_quantize_lane<T, G>(x, n, k0 + l * 8, N, K, (long long)(blockIdx.y * 4 + q) * KB + blockIdx.x, r, l, a.codes, a.pairs);
        }
    }
}

template <typename T, int G>
static cudaError_t launch_quantize(W4QuantArgs& a, cudaStream_t st)
{
    const unsigned blocks = (unsigned)w4_blocks128(a.K), rows = (unsigned)w4_rows16(a.N);
    a.vec = aligned16(a.w) && a.sn * (long long)sizeof(T) % 16 == 0;
    if (a.sk == 1) return launch_overlapped(w4_quantize_kernel<T, G, true>, dim3((blocks + kQuantSteps - 1) / kQuantSteps, rows), dim3(256), 0, st, a);
    return launch_overlapped(w4_quantize_kernel<T, G, false>, dim3(blocks, (rows + 3) / 4), dim3(256), 0, st, a);
}
template <typename T>
static cudaError_t pick_quantize(W4QuantArgs& a, int group, cudaStream_t st)
{
    if (group == 32) return launch_quantize<T, 32>(a, st);
    if (group == 64) return launch_quantize<T, 64>(a, st);
    return launch_quantize<T, 128>(a, st);
}

// -------------------------------------------------------------------------------- matvec --
// y[b, n] = sum over groups g of  s[n, g] sum_k x c + o[n, g] sum_k x : the inner sums run over the codes themselves on
// mma.sync.m16n8k16 (16 output rows on the M side, up to 8 rows of x on the N side, codes as fp16
// subnormals: quant4.cuh), the scales are factors of fp32 sums.  Bound by the bytes of the weights,
// read once.  x enters as fp16 after a power-of-two scaling per row and group that puts the group's largest
// entry into [2^13, 2^14) - exact for bf16 and fp16 x but for what lies 2^-25 below it, two parts of 22 bits for fp32 (the high
// ones multiples of one step, whose sums lose nothing) - so that no value of x is out of fp16's range.
// What an MMA cuts off beside a subnormal's largest product (quant4.cuh) shows in fp32 outputs of 16-bit x only: error 3 to
// 5e-7 of the output with normal x (bf16; fp16 up to 1.1e-6), 1e-5 where x has entries 200 times the others, far below the
// rounding of such an x (torch's fp32 product 3e-7).  Codes shifted up to where the loss ends (3e-7) cost two shifts per four operands: 30.8 ->
// 32.2 us at 36864 x 9216, 1 row, 18.7 -> 20.1 at 5120 x 20480.
// Each of a CTA's 16 warps streams its own blocks of 32 rows (two row tiles: the fragments of x are read once for both) x
// 128 columns through a ring of its own (cp.async, 16 bytes a lane; refilled as soon as it is read), so no warp waits for
// another inside a pair of row tiles.  A pair's columns are split over `split` warps where pairs are few, and over
// the two or four CTAs of a cluster where the fragments of x, laid out in shared memory, would not fit one (4 only then:
// such clusters leave SMs empty, 57.6 against 36.7 us at 36864 x 9216 and 8 rows).  What does not fit four goes over
// two in chunks of columns, laid out again for every pair.  The partial sums meet in shared memory, in a fixed
// order, after every pair.
// Measured back to back from a graph over three sets of inputs: 36864 x 9216, 8 rows of bf16 36.9 us, 4910 GB/s (1 row 30.8 us,
// 5880; what 8 rows cost more is laying x out, about 4 us in which only the rings fill, and the MMAs' instructions), 40.1 with
// a bias, whose loads begin after the join of a pair; 4096 x 4096, 1 row 5.2 us and 768 x 768, fp32 3.7 us (5.5 and 4.1 with a
// bias): launch, x, the first blocks' latency and the join, one after the other.  On a stream 1 us more each.
constexpr int kW4Warps = 16;
constexpr int kW4Threads = 32 * kW4Warps;
constexpr int kW4Join = 3;                  // what the join of a pair costs, in column blocks (16384 x 4096 over clusters of two: 28.7 us without it)
constexpr int kW4Stages = 3;                // of two column blocks

struct W4Args {
    const uint8_t* codes;
    const uint8_t* pairs;
    int N, K, batch, act;
    int KB;                 // column blocks of 128
    int share;              // column blocks per CTA of a cluster
    int chunk;              // column blocks whose x is in shared memory at once
    int tiles;              // row tiles
    int split;              // warps that share a pair of row tiles
    int vec;                // rows of x are 16-byte aligned
    const void* x;
    const void* bias;
    const void* mul;
    void* y;
    long long ld_x, ld_mul, ld_y;
};

__device__ __forceinline__ float w4_act(float v, int act)
{
    if (act == COREINFER_ACT_RELU) return max_nan(v, 0.f);    // a NaN stays one, as in the other activations
    if (act == COREINFER_ACT_SILU) return v / (1.f + __expf(-v));
    return v;
}

// Lays columns [kb0, kb0 + nkb) x 128 of x out as B fragments: xs[block][step (code_word)][column of the MMA][4 lanes] of
// 16 bytes, and xg[group][row] = (2^(x - 14), sum of the group's entries).  A half-warp per block and row of x; a round
// of kXLoads tasks is loaded at once, and the first round before the caller fills the memory system with weights.
constexpr int kXLoads = 5;
template <typename T, int G>
struct XStage {
    static constexpr bool SPLIT = sizeof(T) == 4;
    static constexpr int PER = 128 / G;
    const W4Args& a;
    const int kb0, nkb, l16, h, tig;
    int b, kb, base;                                        // the next task: block kb of row b; a half-warp's next is 32 further on
    uint4 raw[kXLoads][sizeof(T) / 2];
    int bs[kXLoads], ks[kXLoads];

    __device__ __forceinline__ XStage(const W4Args& args, int first, int count, int tid)
        : a(args), kb0(first), nkb(count), l16(tid & 15), h((tid & 15) >> 2), tig(tid & 3), b(0), kb(tid >> 4), base((tid >> 4) & ~1)
    {
        settle();
    }
    __device__ __forceinline__ void settle()
    {
        if (nkb == 0) b = a.batch;
        while (b < a.batch && kb >= nkb) {
            kb -= nkb;
            ++b;
        }
    }
    // Whether there is a round left; the same for both halves of a warp.
    __device__ __forceinline__ bool more() const { return base < nkb * a.batch; }
    __device__ __forceinline__ void load()
    {
#pragma unroll
        for (int u = 0; u < kXLoads; ++u) {
            bs[u] = b;
            ks[u] = kb;
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; ++i) raw[u][i] = make_uint4(0u, 0u, 0u, 0u);
            if (b < a.batch) load_x8<T>((const T*)a.x + (long long)b * a.ld_x, (kb0 + kb) * 128 + h * 32 + tig * 8, a.K, a.vec, raw[u]);
            kb += 2 * kW4Warps;
            settle();
        }
        base += 2 * kW4Warps * kXLoads;
    }
    __device__ __forceinline__ void rest(uint4* xs, float2* xg)
    {
        while (more()) {
            load();
            store(xs, xg);
        }
    }
    __device__ __forceinline__ void store(uint4* xs, float2* xg)
    {
        const int slots = a.batch * (SPLIT ? 2 : 1);
#pragma unroll
        for (int u = 0; u < kXLoads; ++u) {
            if (__all_sync(0xffffffffu, bs[u] >= a.batch)) break;
            float v[8], m = 0.f, sum = 0.f;
            unpack8<T>(raw[u], v);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                m = fmaxf(m, fabsf(v[e]));
                sum += v[e];
            }
#pragma unroll
            for (int d = 1; d < G / 8; d <<= 1) {            // within the half-warp: both halves take part
                m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
                sum += __shfl_xor_sync(0xffffffffu, sum, d);
            }
            // p[e], q[e]: the two entries that code e of a lane's word stands beside (code_word)
            float p[4], q[4];
            if (G == 32) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    p[e] = v[e];
                    q[e] = v[4 + e];
                }
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float other = __shfl_xor_sync(0xffffffffu, h & 1 ? v[e] : v[4 + e], 4);
                    p[e] = h & 1 ? other : v[e];
                    q[e] = h & 1 ? v[4 + e] : other;
                }
            }
            if (bs[u] >= a.batch) continue;
            const int x = range_exponent(m);
            const float up = pow2(14 - x), up16 = up * (1.f / 16.f);          // odd codes stand 16 times higher
#pragma unroll
            for (int part = 0; part < (SPLIT ? 2 : 1); ++part) {
                auto x_part = [part](float x, float step) { return SPLIT ? half_part(x, step, part) : x; };
                uint4 f;
                f.x = pack_half2(x_part(p[0] * up, 8.f), x_part(q[0] * up, 8.f));
                f.y = pack_half2(x_part(p[2] * up, 8.f), x_part(q[2] * up, 8.f));
                f.z = pack_half2(x_part(p[1] * up16, .5f), x_part(q[1] * up16, .5f));
                f.w = pack_half2(x_part(p[3] * up16, .5f), x_part(q[3] * up16, .5f));
                xs[((ks[u] * 4 + h) * slots + (SPLIT ? 2 * bs[u] + part : bs[u])) * 4 + tig] = f;
            }
            if ((l16 & (G / 8 - 1)) == 0) xg[(ks[u] * PER + l16 / (G / 8)) * a.batch + bs[u]] = make_float2(pow2(x - 14), sum);
        }
    }
};

// CHUNKED: x does not fit the shared memory of its CTAs (a kernel of its own: the code for it costs the others 0.5 us).
template <typename T, typename Y, int G, bool CHUNKED>
__global__ void __launch_bounds__(kW4Threads, 1) w4_matvec_kernel(const __grid_constant__ W4Args a)
{
    constexpr bool SPLIT = sizeof(T) == 4;
    constexpr int PER = 128 / G, STAGES = kW4Stages, MM = SPLIT ? 2 : 1;          // MMAs of 8 columns: two for fp32 x of over 4 rows
    constexpr uint32_t BLOCK = 1024 + PER * 64, STAGE = 2 * BLOCK;           // a column block of two row tiles
    const int slots = a.batch * (SPLIT ? 2 : 1);
    const bool both = SPLIT && a.batch > 4;

    extern __shared__ __align__(128) uint8_t smem[];
    uint4* xs = reinterpret_cast<uint4*>(smem + (size_t)kW4Warps * STAGES * STAGE);
    float2* xg = reinterpret_cast<float2*>(xs + (size_t)a.chunk * 16 * slots);
    float* part = reinterpret_cast<float*>(xg + (size_t)a.chunk * PER * a.batch);           // [16 warps][2][8][16]
    const int tid = threadIdx.x, warp = warp_number(), lane = tid & 31, gid = lane >> 2, tig = lane & 3;
    const unsigned size = cluster_size(), rank = cluster_rank();

    // this CTA's column blocks [c0, c1) in chunks, and this warp's share of a chunk, counted from the chunk's start
    const int c0 = (int)rank * a.share < a.KB ? (int)rank * a.share : a.KB, c1 = c0 + a.share < a.KB ? c0 + a.share : a.KB;
    const int part_of = warp % a.split, group = warp / a.split, groups = kW4Warps / a.split;
    const int clusters = gridDim.x / size, cluster = blockIdx.x / size;
    const int chunks = CHUNKED ? (c1 - c0 + a.chunk - 1) / a.chunk : 1;
    auto chunk_len = [&](int ch) { return !CHUNKED ? c1 - c0 : c1 - c0 - ch * a.chunk < a.chunk ? c1 - c0 - ch * a.chunk : a.chunk; };
    auto first_of = [&](int ch) { return part_of * ((chunk_len(ch) + a.split - 1) / a.split); };
    auto count_of = [&](int ch) {
        const int len = chunk_len(ch), each = (len + a.split - 1) / a.split, left = len - part_of * each;
        return left < each ? (left < 0 ? 0 : left) : each;
    };
    // a group's i-th pair: consecutive pairs go to different clusters
    const int pairs = (a.tiles + 1) / 2;
    auto pair_of = [&](int i) { return (i * groups + group) * clusters + cluster; };

    wait_for_stream();
    let_next_start();
    XStage<T, G> stage_x(a, c0, c1 > c0 ? chunk_len(0) : 0, tid);
    stage_x.load();
    const uint32_t ring = smem_u32(smem) + (uint32_t)(warp * STAGES) * STAGE;
    int f_i = 0, f_ch = -1, f_left = 0;                      // the pair and chunk that are copied, the blocks still to copy
    const uint8_t *f_codes = nullptr, *f_pairs = nullptr;    // this lane's part of the next block of its first row tile
    bool f_two = false;                                      // it has a second one
    const size_t codes_row = (size_t)a.KB * 1024, pairs_row = (size_t)a.KB * (PER * 64);
    auto feed_open = [&]() {                                 // the next chunk, or the first of the next pair, with blocks of this warp
        while (pair_of(f_i) < pairs) {
            if (CHUNKED ? ++f_ch >= chunks : ++f_ch > 0) {
                f_ch = -1;
                ++f_i;
                continue;
            }
            f_left = count_of(f_ch);
            if (f_left == 0) {
                if (!CHUNKED) break;
                continue;
            }
            const int pair = pair_of(f_i);
            f_two = 2 * pair + 1 < a.tiles;
            const size_t block = (size_t)(2 * pair) * a.KB + c0 + f_ch * a.chunk + first_of(f_ch);
            f_codes = a.codes + block * 1024 + lane * 16;
            f_pairs = a.pairs + block * (PER * 64) + lane * 16;
            break;
        }
    };
    feed_open();
    auto feed = [&](uint32_t at) {
        if (f_left > 0) {
            copy16(at, f_codes);
            copy16(at + 512, f_codes + 512);
            copy16_if(at + 1024, f_pairs, lane < PER * 4);
            copy16_if(at + BLOCK, f_codes + codes_row, f_two);
            copy16_if(at + BLOCK + 512, f_codes + codes_row + 512, f_two);
            copy16_if(at + BLOCK + 1024, f_pairs + pairs_row, f_two && lane < PER * 4);
            f_codes += 1024;
            f_pairs += PER * 64;
            if (--f_left == 0) feed_open();
        }
        copy_commit();                                       // one group per stage, empty ones too
    };
#pragma unroll 1
    for (int s = 0; s < STAGES; ++s) feed(ring + lane * 16 + s * STAGE);
    stage_x.store(xs, xg);
    stage_x.rest(xs, xg);
    __syncthreads();

    uint32_t stage = 0;
    // columns beyond the rows of x repeat the first one; nobody reads their sums
    const uint32_t xcol0 = ((gid < slots ? gid : 0) * 4 + tig) * 16, xcol1 = ((8 + gid < slots ? 8 + gid : 0) * 4 + tig) * 16 - xcol0;
    const uint32_t xstep = slots * 64, gstep = a.batch * sizeof(float2);      // bytes between pieces of 32 columns, between groups
    uint32_t gx[MM][SPLIT ? 1 : 2];                               // rows of x of this lane's columns
#pragma unroll
    for (int m = 0; m < MM; ++m)
#pragma unroll
        for (int i = 0; i < (SPLIT ? 1 : 2); ++i) {
            const int b = SPLIT ? m * 4 + tig : 2 * tig + i;
            gx[m][i] = (b < a.batch ? b : 0) * sizeof(float2);
        }
    for (int round = 0; round * groups * clusters + cluster < pairs; ++round) {              // the same rounds for a whole cluster
        const bool mine = pair_of(round) < pairs;
        float y[2][MM][4];                                   // [row tile][MMA][rows gid, gid + 8 x two columns]
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int m = 0; m < MM; ++m)
#pragma unroll
                for (int e = 0; e < 4; ++e) y[r][m][e] = 0.f;
#pragma unroll 1
        for (int ch = 0; ch < (CHUNKED ? chunks : 1); ++ch) {
            if (CHUNKED && (round > 0 || ch > 0)) {       // the chunk before is no longer read
                __syncthreads();
                XStage<T, G> next(a, c0 + ch * a.chunk, chunk_len(ch), tid);
                next.rest(xs, xg);
                __syncthreads();
            }
            if (!mine) continue;
            const int k0 = first_of(ch), n = count_of(ch);
            uint32_t xa = smem_u32(xs) + k0 * 4 * xstep + xcol0, ga = smem_u32(xg) + k0 * PER * gstep;
#pragma unroll 1
            for (int k = 0; k < n; ++k) {
                copy_wait<STAGES - 1>();
                __syncwarp();
                const uint32_t st = ring + stage;            // a lane's 16 bytes of the codes of rows gid and gid + 8 stand at lane * 16
                uint32_t w[2][2][4];
#pragma unroll
                for (int r = 0; r < 2; ++r)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint4 v = lds128(st + r * BLOCK + i * 512 + lane * 16);
                        w[r][i][0] = v.x; w[r][i][1] = v.y; w[r][i][2] = v.z; w[r][i][3] = v.w;
                    }
#pragma unroll
                for (int g = 0; g < PER; ++g) {
                    float acc[2][MM][4];
#pragma unroll
                    for (int q = g * G / 32; q < (g + 1) * G / 32; ++q) {
                        uint4 f[MM];
                        f[0] = lds128(xa + q * xstep);
                        if (SPLIT && both) f[MM - 1] = lds128(xa + xcol1 + q * xstep);
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            const uint32_t x0 = code_word<G, 4>(w[r][0], q), x1 = code_word<G, 4>(w[r][1], q);
                            const uint32_t y0 = x0 >> 8, y1 = x1 >> 8;
                            const uint32_t a0 = x0 & 0x000f000fu, a1 = x1 & 0x000f000fu, a2 = y0 & 0x000f000fu, a3 = y1 & 0x000f000fu;
                            const uint32_t b0 = x0 & 0x00f000f0u, b1 = x1 & 0x00f000f0u, b2 = y0 & 0x00f000f0u, b3 = y1 & 0x00f000f0u;
#pragma unroll
                            for (int m = 0; m < MM; ++m) {
                                if (m == 1 && !both) break;
                                if (q == g * G / 32) mma_16816_zero(acc[r][m], a0, a1, a2, a3, f[m].x, f[m].y);
                                else mma_16816(acc[r][m], a0, a1, a2, a3, f[m].x, f[m].y);
                                mma_16816(acc[r][m], b0, b1, b2, b3, f[m].z, f[m].w);
                            }
                        }
                    }
                    float2 e[MM][SPLIT ? 1 : 2];             // (scale, sum) of the group of this lane's rows of x
#pragma unroll
                    for (int m = 0; m < MM; ++m) {
                        if (m == 1 && !both) break;
#pragma unroll
                        for (int i = 0; i < (SPLIT ? 1 : 2); ++i) e[m][i] = lds_f32x2(ga + g * gstep + gx[m][i]);
                    }
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const uint32_t pr = st + r * BLOCK + 1024 + g * 64 + gid * 4;
                        const float2 p0 = lds_half2(pr), p1 = lds_half2(pr + 32);
                        const float s0 = p0.x * kCodeScaleLow, s1 = p1.x * kCodeScaleLow;
#pragma unroll
                        for (int m = 0; m < MM; ++m) {
                            if (m == 1 && !both) break;
                            if (SPLIT) {                     // the two parts of a row of x stand in neighbouring columns
                                y[r][m][0] = fmaf(s0 * (acc[r][m][0] + acc[r][m][1]), e[m][0].x, fmaf(p0.y, e[m][0].y, y[r][m][0]));
                                y[r][m][2] = fmaf(s1 * (acc[r][m][2] + acc[r][m][3]), e[m][0].x, fmaf(p1.y, e[m][0].y, y[r][m][2]));
                            } else {
#pragma unroll
                                for (int i = 0; i < 2; ++i) {
                                    const float2 x = e[m][SPLIT ? 0 : i];
                                    y[r][m][i] = fmaf(s0 * acc[r][m][i], x.x, fmaf(p0.y, x.y, y[r][m][i]));
                                    y[r][m][2 + i] = fmaf(s1 * acc[r][m][2 + i], x.x, fmaf(p1.y, x.y, y[r][m][2 + i]));
                                }
                            }
                        }
                    }
                }
                __syncwarp();                                // all lanes have read the stage
                feed(ring + lane * 16 + stage);
                xa += 4 * xstep;
                ga += PER * gstep;
                stage = stage + STAGE == STAGES * STAGE ? 0 : stage + STAGE;
            }
        }
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            float* buf = part + (warp * 2 + r) * 128;        // [row of x][output row]
#pragma unroll
            for (int m = 0; m < MM; ++m)
#pragma unroll
                for (int i = 0; i < (SPLIT ? 1 : 2); ++i) {
                    const int b = SPLIT ? m * 4 + tig : 2 * tig + i;
                    buf[b * 16 + gid] = y[r][m][i];
                    buf[b * 16 + gid + 8] = y[r][m][2 + i];
                }
        }
        cluster_sync(size);
        // the outputs of the round: the row tiles go round the cluster's CTAs
        const int i = tid & 127, b = i >> 4;                 // row of x and output row
        for (int at = tid >> 7; at < groups * 2; at += kW4Threads >> 7) {
            const int g = at >> 1, r = at & 1, n = ((((round * groups + g) * clusters + cluster) * 2 + r) << 4) + (i & 15);
            if ((at & (size - 1)) != rank || b >= a.batch || n >= a.N) continue;
            float v = 0.f;
            for (unsigned c = 0; c < size; ++c)
                for (int q = 0; q < a.split; ++q) {
                    const float* from = part + ((g * a.split + q) * 2 + r) * 128 + i;
                    v += size == 1 ? *from : cluster_load(cluster_address(from, c));
                }
            if (a.bias) v += to_f32<T>(((const T*)a.bias)[n]);
            v = w4_act(v, a.act);
            if (a.mul) v *= to_f32<Y>(((const Y*)a.mul)[(long long)b * a.ld_mul + n]);
            ((Y*)a.y)[(long long)b * a.ld_y + n] = from_f32<Y>(v);
        }
        cluster_sync(size);                                  // the sums may be overwritten; in the end, no CTA leaves while another reads its
    }
}

// Clusters of `cluster` CTAs of a kernel that the GPU holds at once; asked once per kernel and device: whatever x takes,
// the rings and the sums of a CTA are over half of an SM's shared memory, so the answer is that for one CTA per SM.
template <auto Kernel>
static int clusters_at_once(const DeviceInfo& di, int cluster, size_t smem)
{
    static std::atomic<int> known[64];
    std::atomic<int>& slot = known[di.device & 63];
    int n = slot.load(std::memory_order_relaxed);
    if (n > 0) return n;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(cluster * di.sm_count);
    cfg.blockDim = dim3(kW4Threads);
    cfg.dynamicSmemBytes = smem;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = cluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaOccupancyMaxActiveClusters(&n, Kernel, &cfg) != cudaSuccess || n < 1) n = di.sm_count / (2 * cluster);
    slot.store(n, std::memory_order_relaxed);
    return n;
}

template <typename T, typename Y, int G>
static coreinfer_status launch_group(W4Args& a, const DeviceInfo& di, cudaStream_t st)
{
    constexpr int PER = 128 / G;
    constexpr size_t RING = (size_t)kW4Warps * kW4Stages * 2 * (1024 + PER * 64), PART = (size_t)kW4Warps * 2 * 128 * sizeof(float);
    const int slots = a.batch * (sizeof(T) == 4 ? 2 : 1);
    const size_t per_block = (size_t)slots * 256 + (size_t)PER * a.batch * sizeof(float2);
    const size_t most = smem_room(di) - RING - PART;         // bytes of x fragments and group factors in a CTA
    coreinfer_status s = allow_smem<w4_matvec_kernel<T, Y, G, false>>(di);
    if (s != COREINFER_OK) return s;
    int cluster = a.KB * per_block > most ? 2 : 1;
    if (a.KB * per_block > 2 * most && a.KB * per_block <= 4 * most) cluster = 4;
    a.share = (a.KB + cluster - 1) / cluster;
    a.chunk = a.share * per_block > most ? (int)(most / per_block) : a.share;
    const size_t smem = RING + PART + a.chunk * per_block;
    // pairs of SMs share a TPC, so clusters of two leave none empty
    int clusters = cluster == 4 ? clusters_at_once<w4_matvec_kernel<T, Y, G, false>>(di, 4, smem) : di.sm_count / cluster;
    const int pairs = (a.tiles + 1) / 2;
    if (clusters > pairs) clusters = pairs;
    // Warps per pair: as many as make the longest warp's list of blocks shortest, a join counting as kW4Join blocks.
    long long best = 0;
    for (int split = 1; split <= kW4Warps; split *= 2) {
        const long long groups = (long long)clusters * (kW4Warps / split);
        const long long cost = ((pairs + groups - 1) / groups) * ((a.share + split - 1) / split + kW4Join);
        if (split == 1 || cost < best) {
            best = cost;
            a.split = split;
        }
    }
    auto go = [&](auto chunked) -> coreinfer_status {
        constexpr bool CHUNKED = decltype(chunked)::value;
        if (CHUNKED && (s = allow_smem<w4_matvec_kernel<T, Y, G, CHUNKED>>(di)) != COREINFER_OK) return s;
        CI_CUDA(launch_overlapped(w4_matvec_kernel<T, Y, G, CHUNKED>, dim3(clusters * cluster), dim3(kW4Threads), smem, st, a, cluster));
        return COREINFER_OK;
    };
    return a.chunk < a.share ? go(std::true_type()) : go(std::false_type());
}

template <typename T, typename Y>
static coreinfer_status launch_matvec(W4Args& a, int group, const DeviceInfo& di, cudaStream_t st)
{
    if (group == 32) return launch_group<T, Y, 32>(a, di, st);
    if (group == 64) return launch_group<T, Y, 64>(a, di, st);
    return launch_group<T, Y, 128>(a, di, st);
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
    W4QuantArgs a = {w, N, K, stride_n, stride_k, 0, (uint8_t*)codes, (__half2*)pairs};
    if (dtype == COREINFER_F32) CI_CUDA(pick_quantize<float>(a, group, st));
    else if (dtype == COREINFER_BF16) CI_CUDA(pick_quantize<__nv_bfloat16>(a, group, st));
    else CI_CUDA(pick_quantize<__half>(a, group, st));
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
    a.pairs = (const uint8_t*)w->pairs;
    a.N = w->N;
    a.K = w->K;
    a.KB = (int)w4_blocks128(w->K);
    a.tiles = (int)w4_rows16(w->N);
    a.batch = batch;
    a.act = (int)act;
    a.vec = aligned16(x) && (ld_x * (int64_t)xe) % 16 == 0;
    a.x = x;
    a.bias = bias;
    a.mul = mul;
    a.y = y;
    a.ld_x = ld_x;
    a.ld_mul = ld_mul;
    a.ld_y = ld_y;
    if (dtype == COREINFER_F32) return launch_matvec<float, float>(a, w->group, di, st);
    if (dtype == COREINFER_BF16)
        return y_dtype == COREINFER_F32 ? launch_matvec<__nv_bfloat16, float>(a, w->group, di, st)
                                        : launch_matvec<__nv_bfloat16, __nv_bfloat16>(a, w->group, di, st);
    return y_dtype == COREINFER_F32 ? launch_matvec<__half, float>(a, w->group, di, st)
                                    : launch_matvec<__half, __half>(a, w->group, di, st);
}

}  // extern "C"
