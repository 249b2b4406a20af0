// Attention of a few new tokens per sequence over the 4-bit key/value cache.
//
// Mathematics.  With x^ = s c + o per group, a logit is  sum_g [ s_g sum_{d in g} q_d c_d + o_g sum_{d in g} q_d ]
// and an output  sum_n (p_n s_n) c_nd + sum_n p_n o_n : both products run over the codes themselves, scales enter
// as factors of fp32 sums (keys) or of the fp32 weights p (values).  One pass over the cache with a running
// maximum per query row; rows = new tokens x query heads that share a key head.
//
// What bounds it: the bytes of the cache (codes and pairs of keys and values, each read once).  The work per
// byte is what has to be kept small, so the codes go to mma.sync.m16n8k16 as fp16 subnormals (quant4.cuh: one AND
// per two codes), 16 slots on the M side and 8 query rows on the N side: S^T = K Q^T, then O^T = V^T P^T with
// P^T made from the accumulators of S^T by movmatrix.  tcgen05 would leave most of its 128 rows empty, and its
// operands would have to be widened in shared memory first.
//
// kv4_attention_kernel: persistent CTAs of 8 warps over a ring of stages, each the keys or the values of a tile of up to
// 256 slots of one sequence and head (two bulk copies, contiguous).  Keys and values are stages of their own so
// that the keys' buffer is on its way again while the values are worked on.  The warps take turns at
// refilling the stage used two steps before: a ninth warp for
// the copies would cut the registers of a thread from 128 to 96 at two CTAs per SM.  The tiles of all (sequence, head)
// units form one list, cut into equal pieces, one per CTA, whatever the lengths are; a unit that is cut leaves
// partial results (maximum, sum, output) in the workspace.  kv4_finish_kernel joins those, and turns the
// logits into weights that it adds to the cache's where that is asked for.
// fp32 and fp16 calls carry query rows and p s as two fp16 parts in neighbouring columns (22 bits; four rows per
// tile instead of eight): with one part the rounding of p s (2^-12, times the ratio of s c to the centred
// value, about 3) would exceed fp16's own rounding.
#include "kv4.cuh"

#include <type_traits>

namespace coreinfer {

// Slots per tile: two pieces of 16 per warp, so that waits, votes and addresses are paid once per 32 slots; one piece
// where registers (head_dim 128 in groups of 32) or shared memory (256) do not carry two.
template <int D, int G> constexpr int kAttnTile = D == 256 || (D == 128 && G == 32) ? 128 : 256;
constexpr int kAttnWarps = 8;
constexpr int kAttnThreads = 32 * kAttnWarps;
constexpr int kAttnMaxStages = 10;
constexpr int kAttnMaxCtas = 320;
constexpr float kNoLogit = -1e30f;

struct AttnArgs {
    Kv4 c;
    const void* q;
    void* out;
    long long ld_q, ld_out;
    int Hq, T, share;
    int R;                  // query rows per key head: T * share, row r = t * share + head
    int RT;                 // row tiles (of 8 or 4 rows) per CTA, dividing the warps
    int RU;                 // rows per unit: RT * 8 or RT * 4
    int RB;                 // units per (sequence, key head)
    int n_ctas;             // CTAs of the main kernel
    int stages;
    int tile;               // slots per tile
    float scale;
    int accumulate;
    unsigned* status;
    float2* part_ml;        // [n_ctas][2][RU]: reference exponent and sum of a cut unit's piece
    float* part_o;          // [n_ctas][2][RU][D]
    float2* stats;          // [B][H][RB][RU]: the same of whole units, for the weights
    float* logits;          // [B][H][R][cap], base-2 logits; only with accumulate
};

__device__ __forceinline__ int attn_tiles(int len, int tile) { return (len + tile - 1) / tile; }
// The list of tiles in n equal pieces, the first `more` of them one longer; every CTA that works has one tile at least.
struct AttnCut {
    int n, each, more;
    __device__ __forceinline__ AttnCut(int n_ctas, int total)
    {
        n = total < n_ctas ? total : n_ctas;
        each = n ? total / n : 0;
        more = total - each * n;
    }
    __device__ __forceinline__ int start(int i) const { return i * each + (i < more ? i : more); }
    __device__ __forceinline__ int owner(int t) const
    {
        const int head = more * (each + 1);
        return t < head ? t / (each + 1) : more + (t - head) / each;
    }
};

__device__ __forceinline__ uint32_t movmatrix_trans(uint32_t a)
{
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}

// N consecutive 32-bit words of shared memory.
template <int N>
__device__ __forceinline__ void ld_words(uint32_t (&w)[N], const uint8_t* p)
{
    if constexpr (N == 1) w[0] = *reinterpret_cast<const uint32_t*>(p);
    else if constexpr (N == 2) {
        const uint2 v = *reinterpret_cast<const uint2*>(p);
        w[0] = v.x; w[1] = v.y;
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const uint4 v = *reinterpret_cast<const uint4*>(p + 4 * i);
            w[i] = v.x; w[i + 1] = v.y; w[i + 2] = v.z; w[i + 3] = v.w;
        }
    }
}
__device__ __forceinline__ float2 pair_f32(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }

// Four neighbouring outputs; the address is a multiple of four elements.
template <typename T>
__device__ __forceinline__ void store4(T* dst, float x, float y, float z, float w)
{
    T v[4] = {from_f32<T>(x), from_f32<T>(y), from_f32<T>(z), from_f32<T>(w)};
    if (sizeof(T) == 4) *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<uint4*>(v);
    else *reinterpret_cast<uint2*>(dst) = *reinterpret_cast<uint2*>(v);
}

// Position in the list of tiles.
struct Cursor {
    int b, hr, tile, nt;
};

// How query rows sit in the 8 columns of an MMA: a row per column; a row per two columns with the second empty
// (up to 4 rows: half the softmax work per lane); a row per two columns, the second for the low part.
enum { kRows8 = 0, kRows4 = 1, kRows4Parts = 2 };

template <typename T, int D, int G, int MODE>
__global__ void __launch_bounds__(kAttnThreads, D <= 128 ? 2 : 1)
kv4_attention_kernel(const __grid_constant__ AttnArgs a)
{
    constexpr bool PARTS = MODE == kRows4Parts, WIDE = MODE != kRows8;
    constexpr int H32 = D / 32, NG = D / G, RPT = WIDE ? 4 : 8, NV = WIDE ? 1 : 2, TILE = kAttnTile<D, G>;
    constexpr int UN = TILE / (16 * kAttnWarps);             // pieces of 16 slots per step of a warp
    constexpr uint32_t CODE_ROW = D / 2, PAIR_ROW = NG * 4;
    constexpr uint32_t CODE_TILE = TILE * CODE_ROW, PAIR_TILE = TILE * PAIR_ROW;
    constexpr uint32_t STAGE = CODE_TILE + PAIR_TILE;
    const Kv4& c = a.c;

    extern __shared__ __align__(128) uint8_t smem[];
    float* obuf = reinterpret_cast<float*>(smem + (size_t)a.stages * STAGE);                // [8 warps][RPT][D]
    float2* mlbuf = reinterpret_cast<float2*>(obuf + kAttnWarps * RPT * D);                  // [8 warps][RPT]
    int* pre = reinterpret_cast<int*>(mlbuf + kAttnWarps * RPT);                             // [B + 1] tiles of a head before sequence b
    int* lens = pre + c.B + 1;                                                               // [B]
    __shared__ uint64_t full_bar[kAttnMaxStages], empty_bar[kAttnMaxStages];
    __shared__ int abort_s;
    volatile int* abort_flag = &abort_s;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int s = 0; s < a.stages; ++s) {
            mbar_init(smem_u32(&full_bar[s]), 1);
            mbar_init(smem_u32(&empty_bar[s]), kAttnWarps);
        }
        abort_s = 0;
        mbar_fence_init();
        if (blockIdx.x == 0) *a.status = kStatusOk;          // a wait gives up seconds later at the earliest
    }
    if (warp == 0) {
        int run = 0;
        for (int b0 = 0; b0 < c.B; b0 += 32) {
            const int b = b0 + lane;
            const int len = b < c.B ? kv4_length(c, b) : 0;
            const int v = attn_tiles(len, TILE);
            int incl = v;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int u = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += u;
            }
            if (b < c.B) {
                lens[b] = len;
                pre[b] = run + incl - v;
            }
            run += __shfl_sync(0xffffffffu, incl, 31);
        }
        if (lane == 0) pre[c.B] = run;
    }
    __syncthreads();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    const int HR = c.H * a.RB;
    const int total = pre[c.B] * HR;
    const AttnCut cut(a.n_ctas, total);
    const int me = blockIdx.x;
    const int begin = me < cut.n ? cut.start(me) : 0, end = me < cut.n ? cut.start(me + 1) : 0;
    auto token_of = [&](int r) { return a.T == 1 ? 0 : r / a.share; };       // of a query row
    auto seek = [&](int t) {
        Cursor k;
        int lo = 0, hi = c.B - 1;                           // last b with pre[b] * HR <= t: it has tiles
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (pre[mid] * HR <= t) lo = mid; else hi = mid - 1;
        }
        k.b = lo;
        k.nt = attn_tiles(lens[lo], TILE);
        const unsigned rem = (unsigned)(t - pre[lo] * HR);
        k.hr = (int)(rem / (unsigned)k.nt);
        k.tile = (int)(rem % (unsigned)k.nt);
        return k;
    };
    // One thread: the copies of a tile's keys (which = 0) or values into stage s.
    auto fetch = [&](int b, int hr, int tile, int which, int s) {
        const int t0 = tile * TILE;
        // whole 16-slot pieces: the capacity is a multiple of 16, so they lie within the buffers
        const int left = (lens[b] - t0 + 15) & ~15;
        const uint32_t rows = left < TILE ? left : TILE;
        const size_t slot = ((size_t)b * c.H + hr / a.RB) * c.cap + t0;
        const uint32_t bar = smem_u32(&full_bar[s]), dst = smem_u32(smem + (size_t)s * STAGE);
        mbar_arrive_expect_tx(bar, rows * (CODE_ROW + PAIR_ROW));
        bulk_g2s(dst, c.codes[which] + slot * CODE_ROW, rows * CODE_ROW, bar);
        bulk_g2s(dst + CODE_TILE, reinterpret_cast<const uint8_t*>(c.pairs[which]) + slot * PAIR_ROW, rows * PAIR_ROW, bar);
    };

    if (begin < end) {
        for (int s = warp; s < a.stages && s < 2 * (end - begin); s += kAttnWarps)       // the first stages, one warp each
            if (lane == 0) {
                const Cursor p = seek(begin + s / 2);
                fetch(p.b, p.hr, p.tile, s & 1, s);
            }
        __syncwarp();
        const int rt = warp % a.RT, sg = warp / a.RT, nsg = kAttnWarps / a.RT;
        const int gid = lane >> 2, tig = lane & 3;
        const int tok0 = (gid >> 1) + (gid & 1) * 4;         // slot of accumulator row gid within 8; row gid + 8: tok0 + 8
        Cursor k = seek(begin);
        int s = 0;
        uint32_t ph = 0;
        int t = begin, step = 0;                             // step 2 i: keys of the CTA's tile i, 2 i + 1: its values
        while (t < end) {
            const int first_tile = k.tile, b = k.b, len = lens[b], h = a.RB == 1 ? k.hr : k.hr / a.RB, rb = k.hr - h * a.RB;
            const int n_tiles = end - t < k.nt - first_tile ? end - t : k.nt - first_tile;
            const int row0 = rb * a.RU + rt * RPT;           // first query row of this warp's tile

            // query rows as the B operand: column gid = row gid (or part gid & 1 of row gid >> 1), 8 values per 32
            uint32_t qf[H32][4];
            float qsum[NG][NV], f[NV];
            int lim[NV];                                     // slots this lane's columns see
            {
                const int r = row0 + (WIDE ? gid >> 1 : gid);
                const bool valid = r < a.R && (MODE != kRows4 || (gid & 1) == 0);
                const int rt_ = valid ? token_of(r) : 0, rh = valid ? r - rt_ * a.share : 0;
                const T* src = (const T*)a.q + ((long long)b * a.T + rt_) * a.ld_q + (long long)(h * a.share + rh) * D + 8 * tig;
                float v[H32][8], m = 0.f;
#pragma unroll
                for (int j = 0; j < H32; ++j) {
                    T in[8];
                    const uint4* p = reinterpret_cast<const uint4*>(src + j * 32);
                    *reinterpret_cast<uint4*>(in) = p[0];
                    if (sizeof(T) == 4) reinterpret_cast<uint4*>(in)[1] = p[1];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        v[j][e] = valid ? to_f32<T>(in[e]) : 0.f;
                        m = fmaxf(m, fabsf(v[j][e]));
                    }
                }
                m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
                m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
                const int x = range_exponent(m);             // the largest value goes to [2^13, 2^14)
                const float up = pow2(14 - x);
                float gs[NG];
#pragma unroll
                for (int g = 0; g < NG; ++g) gs[g] = 0.f;
#pragma unroll
                for (int j = 0; j < H32; ++j) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        v[j][e] *= up;
                        gs[j * 32 / G] += v[j][e];
                    }
                }
                const int low = PARTS ? gid & 1 : 0;
                const float lo16 = 1.f / 16.f;               // odd codes stand 16 times higher
#pragma unroll
                for (int j = 0; j < H32; ++j) {
                    // the two entries beside each other in step j (code_word)
                    const float *p = G == 32 ? &v[j][0] : &v[j & ~1][(j & 1) * 4], *q = G == 32 ? &v[j][4] : &v[j | 1][(j & 1) * 4];
                    qf[j][0] = pack_half2(half_part(p[0], low), half_part(q[0], low));
                    qf[j][1] = pack_half2(half_part(p[2], low), half_part(q[2], low));
                    qf[j][2] = pack_half2(half_part(p[1] * lo16, low), half_part(q[1] * lo16, low));
                    qf[j][3] = pack_half2(half_part(p[3] * lo16, low), half_part(q[3] * lo16, low));
                }
                // sums of c q carry 2^-24, so the sums of q do too; f undoes both scalings
                const float ff = ldexpf(a.scale * 1.44269504088896341f, x - 14 + 24);
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    gs[g] += __shfl_xor_sync(0xffffffffu, gs[g], 1);
                    gs[g] += __shfl_xor_sync(0xffffffffu, gs[g], 2);
                    gs[g] *= 1.f / kCodeScaleLow;
                }
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int from = (2 * tig + i) * 4;      // a lane of column 2 tig + i
#pragma unroll
                    for (int g = 0; g < NG; ++g) qsum[g][i] = __shfl_sync(0xffffffffu, gs[g], from);
                    f[i] = __shfl_sync(0xffffffffu, ff, from);
                    const int rr = row0 + (WIDE ? tig : 2 * tig + i);
                    lim[i] = rr < a.R ? len - (a.T - 1 - token_of(rr)) : 0;
                }
            }
            float* lg[NV];                                   // this lane's logits, NULL where none are kept
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int rr = row0 + (WIDE ? tig : 2 * tig + i);
                lg[i] = a.accumulate && rr < a.R ? a.logits + (((size_t)b * c.H + h) * a.R + rr) * c.cap + tok0 : nullptr;
            }
            const int all_see = len - (a.T - 1);             // slots below this are seen by every row

            float o[H32][2][4], om[NG][NV], l[NV], mx[NV];
            // The weights enter the second product as p s 2^E in fp16: E keeps the largest s near 2^9, so
            // that p s neither overflows nor loses bits to fp16's bottom for p down to about 2^-20.
            float E = 0.f, s_most = -1.f;
#pragma unroll
            for (int j = 0; j < H32; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[j][0][e] = o[j][1][e] = 0.f;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                l[i] = 0.f;
                mx[i] = kNoLogit;
#pragma unroll
                for (int g = 0; g < NG; ++g) om[g][i] = 0.f;
            }

            // Into a step: refill the stage of two steps before (every warp has left it, or will without this one), then
            // wait for this step's stage.
            auto enter = [&]() {
                const int refill = step - 2 + a.stages;
                if (warp == (step & (kAttnWarps - 1)) && lane == 0 && step >= 2 && refill < 2 * (end - begin)) {
                    const int was = s >= 2 ? s - 2 : s - 2 + a.stages;
                    bounded_wait(smem_u32(&empty_bar[was]), s >= 2 ? ph : ph ^ 1u, abort_flag, a.status);
                    if (!*abort_flag) {
                        const int tile = begin + (refill >> 1) - t + first_tile;
                        if (tile < k.nt) {
                            fetch(b, k.hr, tile, refill & 1, was);
                        } else {
                            const Cursor p = seek(begin + (refill >> 1));
                            fetch(p.b, p.hr, p.tile, refill & 1, was);
                        }
                    }
                }
                __syncwarp();
                bounded_wait(smem_u32(&full_bar[s]), ph, abort_flag, a.status);
                const int here = s;
                ++step;
                if (++s == a.stages) { s = 0; ph ^= 1u; }
                return here;
            };
            auto leave = [&](int stage) {
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&empty_bar[stage]));
            };

            for (int it = 0; it < n_tiles; ++it) {
                const int t0 = (first_tile + it) * TILE;
                const int ks = enter();
                int vs = -1;
                bool keys_left = false;
                const uint8_t* kst = smem + (size_t)ks * STAGE;
                const uint8_t* vst = nullptr;
                for (int sub = UN * sg; sub < TILE / 16; sub += UN * nsg) {
                    const int n0 = t0 + sub * 16;
                    if (n0 >= len) break;
                    // ---- logits: S^T [UN][16 slots][8 columns]; lo[u][v]: slot n0 + 16 u + 8 v + tok0 ----
                    float lo[UN][2][NV];
#pragma unroll
                    for (int u = 0; u < UN; ++u) {
                        const uint8_t* krow = kst + (sub * 16 + u * 16 + tok0) * CODE_ROW + tig * (D / 8);
                        uint32_t w0[D / 32], w1[D / 32], kp0[NG], kp1[NG];
                        ld_words<D / 32>(w0, krow);
                        ld_words<D / 32>(w1, krow + 8 * CODE_ROW);
                        const uint8_t* kpr = kst + CODE_TILE + (sub * 16 + u * 16 + tok0) * PAIR_ROW;
                        ld_words<NG>(kp0, kpr);
                        ld_words<NG>(kp1, kpr + 8 * PAIR_ROW);
#pragma unroll
                        for (int g = 0; g < NG; ++g) {
                            float acc[4];
#pragma unroll
                            for (int j = g * G / 32; j < (g + 1) * G / 32; ++j) {
                                const uint32_t x0 = code_word<G, H32>(w0, j), x1 = code_word<G, H32>(w1, j);
                                const uint32_t y0 = x0 >> 8, y1 = x1 >> 8;
                                if (j == g * G / 32)
                                    mma_16816_zero(acc, x0 & 0x000f000fu, x1 & 0x000f000fu, y0 & 0x000f000fu, y1 & 0x000f000fu, qf[j][0], qf[j][1]);
                                else
                                    mma_16816(acc, x0 & 0x000f000fu, x1 & 0x000f000fu, y0 & 0x000f000fu, y1 & 0x000f000fu, qf[j][0], qf[j][1]);
                                mma_16816(acc, x0 & 0x00f000f0u, x1 & 0x00f000f0u, y0 & 0x00f000f0u, y1 & 0x00f000f0u, qf[j][2], qf[j][3]);
                            }
                            const float2 p0 = pair_f32(kp0[g]), p1 = pair_f32(kp1[g]);
#pragma unroll
                            for (int i = 0; i < NV; ++i) {
                                const float a0 = PARTS ? acc[0] + acc[1] : acc[i], a1 = PARTS ? acc[2] + acc[3] : acc[2 + i];
                                const float o0 = p0.y * qsum[g][i], o1 = p1.y * qsum[g][i];
                                lo[u][0][i] = fmaf(p0.x, a0, g ? lo[u][0][i] + o0 : o0);
                                lo[u][1][i] = fmaf(p1.x, a1, g ? lo[u][1][i] + o1 : o1);
                            }
                        }
                    }
                    const int na = n0 + tok0;
                    const bool edge = n0 + 16 * UN > all_see;     // some row does not see some slot
                    float most[NV];
#pragma unroll
                    for (int i = 0; i < NV; ++i) {
#pragma unroll
                        for (int u = 0; u < UN; ++u)
#pragma unroll
                            for (int v = 0; v < 2; ++v) lo[u][v][i] *= f[i];
                        if (edge) [[unlikely]] {
#pragma unroll
                            for (int u = 0; u < UN; ++u)
#pragma unroll
                                for (int v = 0; v < 2; ++v)
                                    if (na + 16 * u + 8 * v >= lim[i]) lo[u][v][i] = -__int_as_float(0x7f800000);
                        }
                        most[i] = fmaxf(lo[0][0][i], lo[0][1][i]);
#pragma unroll
                        for (int u = 1; u < UN; ++u) most[i] = fmaxf(most[i], fmaxf(lo[u][0][i], lo[u][1][i]));
                        if (lg[i]) {
                            // what a row does not see may be written too: it lies within the capacity and is never read
                            float* to = lg[i] + n0;
#pragma unroll
                            for (int u = 0; u < UN; ++u)
                                if (UN == 1 || u == 0 || n0 + 16 < len) {
                                    to[16 * u] = lo[u][0][i];
                                    to[16 * u + 8] = lo[u][1][i];
                                }
                        }
                    }
                    if (n0 + 16 * UN * nsg >= len || sub + UN * nsg >= TILE / 16) {      // this warp's last step of the tile
                        leave(ks);
                        keys_left = true;
                    }
                    if (!vst) {
                        vs = enter();
                        vst = smem + (size_t)vs * STAGE;
                    }
                    // ---- value pairs, running maximum ----
                    uint32_t vp[UN][2][NG];
                    __half2 smax = __float2half2_rn(0.f);
#pragma unroll
                    for (int u = 0; u < UN; ++u)
#pragma unroll
                        for (int v = 0; v < 2; ++v) {
                            ld_words<NG>(vp[u][v], vst + CODE_TILE + (sub * 16 + 16 * u + 8 * v + tok0) * PAIR_ROW);
                            if (edge && na + 16 * u + 8 * v >= len) [[unlikely]] {                        // never used
#pragma unroll
                                for (int g = 0; g < NG; ++g) vp[u][v][g] = 0u;
                            }
#pragma unroll
                            for (int g = 0; g < NG; ++g) {
                                smax = __hmax2(smax, *reinterpret_cast<const __half2*>(&vp[u][v][g]));
                            }
                        }
                    float s_here = __low2float(smax);
                    bool change = s_here > s_most;
#pragma unroll
                    for (int i = 0; i < NV; ++i) change |= most[i] > mx[i];
                    if (__any_sync(0xffffffffu, change)) {
                        float e_new = E;
                        if (__any_sync(0xffffffffu, s_here > s_most)) {
#pragma unroll
                            for (int d = 1; d < 32; d <<= 1) s_here = fmaxf(s_here, __shfl_xor_sync(0xffffffffu, s_here, d));
                            int x;
                            frexpf(s_here, &x);
                            x = s_here > 0.f ? (x < -15 ? -15 : x) : -15;
                            e_new = (float)(9 - x);
                            s_most = ldexpf(1.f, x + 5);     // room for scales up to 32 times larger before E moves
                        }
#pragma unroll
                        for (int i = 0; i < NV; ++i) {
                            float m = most[i];
                            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 4));
                            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
                            m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
                            m = fmaxf(m, mx[i]);
                            const float corr = exp2_fast((mx[i] - E) - (m - e_new));
                            mx[i] = m;
                            l[i] *= corr;
#pragma unroll
                            for (int g = 0; g < NG; ++g) om[g][i] *= corr;
#pragma unroll
                            for (int j = 0; j < H32; ++j)
#pragma unroll
                                for (int e = 0; e < 2; ++e) {
                                    o[j][e][i] *= corr;
                                    o[j][e][2 + i] *= corr;
                                    if (PARTS) {
                                        o[j][e][1] *= corr;
                                        o[j][e][3] *= corr;
                                    }
                                }
                        }
                        E = e_new;
                    }
#pragma unroll
                    for (int i = 0; i < NV; ++i) {
                        const float ref = mx[i] - E;
#pragma unroll
                        for (int u = 0; u < UN; ++u)
#pragma unroll
                            for (int v = 0; v < 2; ++v) {
                                lo[u][v][i] = exp2_fast(lo[u][v][i] - ref);          // p from here on
                                l[i] += lo[u][v][i];
                            }
                    }
                    // ---- O^T += V^T P^T, per group of scales ----
#pragma unroll
                    for (int u = 0; u < UN; ++u) {
                        const uint8_t* vrow = vst + (sub * 16 + u * 16 + tig) * CODE_ROW + gid * (D / 16);
                        uint32_t va[H32 / 2], vb[H32 / 2], vc[H32 / 2], vd[H32 / 2];
                        ld_words<H32 / 2>(va, vrow);
                        ld_words<H32 / 2>(vb, vrow + 4 * CODE_ROW);
                        ld_words<H32 / 2>(vc, vrow + 8 * CODE_ROW);
                        ld_words<H32 / 2>(vd, vrow + 12 * CODE_ROW);
#pragma unroll
                        for (int g = 0; g < NG; ++g) {
                            uint32_t bf[2];
#pragma unroll
                            for (int v = 0; v < 2; ++v) {
                                const float2 so = pair_f32(vp[u][v][g]);
                                float ps[NV];
                                float om_was[NV];
#pragma unroll
                                for (int i = 0; i < NV; ++i) {
                                    om_was[i] = om[g][i];
                                    ps[i] = lo[u][v][i] * so.x;
                                    om[g][i] = fmaf(lo[u][v][i], so.y, om[g][i]);
                                }
                                if (edge) [[unlikely]] {     // a slot that a row does not see adds nothing, whatever it holds
#pragma unroll
                                    for (int i = 0; i < NV; ++i)
                                        if (na + 16 * u + 8 * v >= lim[i]) {
                                            ps[i] = 0.f;
                                            om[g][i] = om_was[i];
                                        }
                                }
                                if (PARTS) {
                                    const float high = __half2float(__float2half_rn(ps[0]));
                                    bf[v] = movmatrix_trans(pack_half2(high, ps[0] - high));
                                } else {
                                    bf[v] = movmatrix_trans(pack_half2(ps[0], WIDE ? 0.f : ps[NV - 1]));
                                }
                            }
#pragma unroll
                            for (int j = g * G / 32; j < (g + 1) * G / 32; ++j) {
                                const uint32_t x = __byte_perm(va[j / 2], vb[j / 2], j & 1 ? 0x7632 : 0x5410);
                                const uint32_t y = __byte_perm(vc[j / 2], vd[j / 2], j & 1 ? 0x7632 : 0x5410);
                                const uint32_t x8 = x >> 8, y8 = y >> 8;
                                mma_16816(o[j][0], x & 0x000f000fu, x8 & 0x000f000fu, y & 0x000f000fu, y8 & 0x000f000fu, bf[0], bf[1]);
                                mma_16816(o[j][1], x & 0x00f000f0u, x8 & 0x00f000f0u, y & 0x00f000f0u, y8 & 0x00f000f0u, bf[0], bf[1]);
                            }
                        }
                    }
                }
                if (!keys_left) leave(ks);                   // the tile ends before this warp's slots
                if (!vst) vs = enter();
                leave(vs);
            }

            // ---- join the warps of a row tile ----
            __syncthreads();                                 // the buffer's last use is over
#pragma unroll
            for (int i = 0; i < NV; ++i) {
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) {
                    l[i] += __shfl_xor_sync(0xffffffffu, l[i], d);
#pragma unroll
                    for (int g = 0; g < NG; ++g) om[g][i] += __shfl_xor_sync(0xffffffffu, om[g][i], d);
                }
                const int r = WIDE ? tig : 2 * tig + i;
                if (gid == 0) mlbuf[warp * RPT + r] = make_float2(mx[i] - E, l[i]);
#pragma unroll
                for (int j = 0; j < H32; ++j) {
                    const float add = om[j * 32 / G][i];
                    float4 v;
                    if (PARTS) {
                        v.x = o[j][0][0] + o[j][0][1];
                        v.y = o[j][1][0] + o[j][1][1];
                        v.z = o[j][0][2] + o[j][0][3];
                        v.w = o[j][1][2] + o[j][1][3];
                    } else {
                        v.x = o[j][0][i];
                        v.y = o[j][1][i];
                        v.z = o[j][0][2 + i];
                        v.w = o[j][1][2 + i];
                    }
                    v.x = fmaf(v.x, kCodeScaleLow, add);
                    v.y = fmaf(v.y, kCodeScaleHigh, add);
                    v.z = fmaf(v.z, kCodeScaleLow, add);
                    v.w = fmaf(v.w, kCodeScaleHigh, add);
                    *reinterpret_cast<float4*>(obuf + ((size_t)warp * RPT + r) * D + j * 32 + gid * 4) = v;
                }
            }
            __syncthreads();
            const bool whole = n_tiles == k.nt;
            const int piece = blockIdx.x * 2 + (first_tile == 0 ? 1 : 0);
            // nsg neighbouring lanes take the parts of one quad of outputs and add them up by shuffles
            const int rows_here = a.R - rb * a.RU < a.RU ? a.R - rb * a.RU : a.RU, items = rows_here * (D / 4);
            const int part = tid % nsg, per_round = 32 * kAttnWarps / nsg;
            for (int i0 = 0; i0 < items; i0 += per_round) {
                const int item = i0 + tid / nsg, ru = item < items ? item / (D / 4) : 0, d4 = item % (D / 4);
                const int from = (part * a.RT + ru / RPT) * RPT + ru % RPT;      // row of the part's warp
                const float2 ml = mlbuf[from];
                const float4 x = *reinterpret_cast<const float4*>(obuf + (size_t)from * D + d4 * 4);
                float top = ml.x;
                for (int d = 1; d < nsg; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                const float e = exp2_fast(ml.x - top);
                float sum = ml.y * e;
                float4 v = make_float4(x.x * e, x.y * e, x.z * e, x.w * e);
                for (int d = 1; d < nsg; d <<= 1) {
                    sum += __shfl_xor_sync(0xffffffffu, sum, d);
                    v.x += __shfl_xor_sync(0xffffffffu, v.x, d);
                    v.y += __shfl_xor_sync(0xffffffffu, v.y, d);
                    v.z += __shfl_xor_sync(0xffffffffu, v.z, d);
                    v.w += __shfl_xor_sync(0xffffffffu, v.w, d);
                }
                if (part != 0 || item >= items) continue;
                if (whole) {
                    const float inv = sum == 0.f ? 0.f : 1.f / sum;
                    const int r = rb * a.RU + ru, rt_ = token_of(r);
                    T* dst = (T*)a.out + ((long long)b * a.T + rt_) * a.ld_out + (long long)(h * a.share + r - rt_ * a.share) * D + d4 * 4;
                    store4(dst, v.x * inv, v.y * inv, v.z * inv, v.w * inv);
                    if (d4 == 0 && a.accumulate) a.stats[(((size_t)b * c.H + h) * a.RB + rb) * a.RU + ru] = make_float2(top, sum);
                } else {
                    *reinterpret_cast<float4*>(a.part_o + ((size_t)piece * a.RU + ru) * D + d4 * 4) = v;
                    if (d4 == 0) a.part_ml[(size_t)piece * a.RU + ru] = make_float2(top, sum);
                }
            }
            t += n_tiles;
            if (t < end) k = seek(t);
        }
    }
    __syncthreads();
    if (tid == 0 && *abort_flag) {
        // after a wait that gave up copies may be in flight: give them a bounded time to land
        const long long t0 = clock64();
        while (clock64() - t0 < 20000000LL) __nanosleep(1000);
    }
    __syncthreads();
}

// ------------------------------------------------------------------------------ finish --
// Blocks x < R of a (sequence, head): query row x, joined from the pieces of its unit where that was cut
// (zeros where the sequence is empty).  Blocks beyond: 1024 slots each, whose weights get the
// sum over rows of 2^(logit - maximum) / sum.
constexpr int kFinishThreads = 256;
constexpr int kFinishSlots = 1024;

template <typename V, typename Op>
__device__ __forceinline__ V finish_reduce(V v, V* buf, Op op)
{
#pragma unroll
    for (int d = 16; d; d >>= 1) v = op(v, __shfl_xor_sync(0xffffffffu, v, d));
    if ((threadIdx.x & 31) == 0) buf[threadIdx.x >> 5] = v;
    __syncthreads();
    v = buf[0];
#pragma unroll
    for (int i = 1; i < kFinishThreads / 32; ++i) v = op(v, buf[i]);
    __syncthreads();
    return v;
}

template <typename T>
__global__ void __launch_bounds__(kFinishThreads) kv4_finish_kernel(const __grid_constant__ AttnArgs a)
{
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ float redf[8];
    const Kv4& c = a.c;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int b = blockIdx.y / c.H, h = blockIdx.y % c.H, D = c.D;
    const int len = kv4_length(c, b);
    if ((int)blockIdx.x >= a.R && ((int)blockIdx.x - a.R) * kFinishSlots >= len) return;
    int before = 0, all = 0;                                 // tiles of a head, before this sequence and in all; every warp for itself
    for (int i = lane; i < c.B; i += 32) {
        const int n = attn_tiles(kv4_length(c, i), a.tile);
        all += n;
        if (i < b) before += n;
    }
    before = __reduce_add_sync(0xffffffffu, before);
    all = __reduce_add_sync(0xffffffffu, all);
    const int HR = c.H * a.RB, nt = attn_tiles(len, a.tile), total = all * HR;
    const AttnCut cut(a.n_ctas, total);
    asm volatile("griddepcontrol.wait;" ::: "memory");

    if ((int)blockIdx.x < a.R) {
        const int r = blockIdx.x, rb = r / a.RU, ru = r % a.RU;
        const int rt_ = a.T == 1 ? 0 : r / a.share;
        T* dst = (T*)a.out + ((long long)b * a.T + rt_) * a.ld_out + (long long)(h * a.share + r - rt_ * a.share) * D;
        if (nt == 0) {
            for (int d = tid; d < D; d += kFinishThreads) dst[d] = from_f32<T>(0.f);
            return;
        }
        const int u0 = before * HR + (h * a.RB + rb) * nt;
        const int i0 = cut.owner(u0), i1 = cut.owner(u0 + nt - 1);
        if (i0 == i1) return;
        float* wgt = reinterpret_cast<float*>(smem);                     // [pieces]
        const int n = i1 - i0 + 1;
        auto piece = [&](int i) { return (size_t)(i0 + i) * 2 + (i == 0 ? 1 : 0); };
        float top = kNoLogit * 2.f;
        for (int i = tid; i < n; i += kFinishThreads) top = fmaxf(top, a.part_ml[piece(i) * a.RU + ru].x);
        top = finish_reduce(top, redf, [](float x, float y) { return fmaxf(x, y); });
        float sum = 0.f;
        for (int i = tid; i < n; i += kFinishThreads) {
            const float2 ml = a.part_ml[piece(i) * a.RU + ru];
            const float e = exp2_fast(ml.x - top);
            wgt[i] = e;
            sum = fmaf(ml.y, e, sum);
        }
        sum = finish_reduce(sum, redf, [](float x, float y) { return x + y; });
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        // D / 4 threads cover the row, 256 / (D / 4) of such groups take the pieces in turn
        const int quads = D / 4, groups = kFinishThreads / quads, d4 = tid % quads, g = tid / quads;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int i = g; i < n; i += groups) {
            const float4 x = *reinterpret_cast<const float4*>(a.part_o + (piece(i) * a.RU + ru) * D + d4 * 4);
            const float e = wgt[i];
            v.x = fmaf(x.x, e, v.x);
            v.y = fmaf(x.y, e, v.y);
            v.z = fmaf(x.z, e, v.z);
            v.w = fmaf(x.w, e, v.w);
        }
        float4* buf = reinterpret_cast<float4*>(smem + kAttnMaxCtas * sizeof(float));
        buf[tid] = v;
        __syncthreads();
        if (g == 0) {
            for (int j = 1; j < groups; ++j) {
                const float4 x = buf[j * quads + d4];
                v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
            }
            store4(dst + d4 * 4, v.x * inv, v.y * inv, v.z * inv, v.w * inv);
        }
        return;
    }

    // weights: maximum and 1 / sum of every row, one warp per row
    float2* rows = reinterpret_cast<float2*>(smem);                      // [R]
    int* sees = reinterpret_cast<int*>(rows + a.R);                      // [R] slots that the row sees
    for (int r = warp; r < a.R; r += kFinishThreads / 32) {
        const int rb = r / a.RU, ru = r % a.RU;
        const int u0 = before * HR + (h * a.RB + rb) * nt;
        const int i0 = cut.owner(u0), i1 = cut.owner(u0 + nt - 1);
        float top, sum;
        if (i0 == i1) {
            const float2 ml = a.stats[(((size_t)b * c.H + h) * a.RB + rb) * a.RU + ru];
            top = ml.x;
            sum = ml.y;
        } else {
            top = kNoLogit * 2.f;
            for (int i = i0 + lane; i <= i1; i += 32) top = fmaxf(top, a.part_ml[((size_t)i * 2 + (i == i0)) * a.RU + ru].x);
#pragma unroll
            for (int d = 16; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
            sum = 0.f;
            for (int i = i0 + lane; i <= i1; i += 32) {
                const float2 ml = a.part_ml[((size_t)i * 2 + (i == i0)) * a.RU + ru];
                sum = fmaf(ml.y, exp2_fast(ml.x - top), sum);
            }
#pragma unroll
            for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        }
        if (lane == 0) {
            rows[r] = make_float2(top, sum == 0.f ? 0.f : 1.f / sum);
            sees[r] = len - (a.T - 1 - r / a.share);
        }
    }
    __syncthreads();
    // four slots a thread: the capacity is a multiple of 16, so they lie within a row of logits
    const int n = ((int)blockIdx.x - a.R) * kFinishSlots + tid * 4;
    if (n >= len) return;
    const float* lg = a.logits + ((size_t)b * c.H + h) * a.R * c.cap + n;
    float4* weight = reinterpret_cast<float4*>(c.weight + ((size_t)b * c.H + h) * c.cap + n);
    float4 w = *weight;
#pragma unroll 8
    for (int r = 0; r < a.R; ++r) {
        const float4 x = *reinterpret_cast<const float4*>(lg + (size_t)r * c.cap);
        const float2 ml = rows[r];
        const int see = sees[r] - n;                        // slots of the four that the row sees
        if (see > 0) w.x = fmaf(exp2_fast(x.x - ml.x), ml.y, w.x);
        if (see > 1) w.y = fmaf(exp2_fast(x.y - ml.x), ml.y, w.y);
        if (see > 2) w.z = fmaf(exp2_fast(x.z - ml.x), ml.y, w.z);
        if (see > 3) w.w = fmaf(exp2_fast(x.w - ml.x), ml.y, w.w);
    }
    *weight = w;
}

// -------------------------------------------------------------------------------- host --
static inline size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

// Rows per unit and units per key head for R query rows.
static void attn_rows(int R, int rpt, int* RT, int* RU, int* RB)
{
    const int tiles = (R + rpt - 1) / rpt;
    *RT = tiles > 4 ? 8 : (tiles > 2 ? 4 : tiles);
    *RU = *RT * rpt;
    *RB = (R + *RU - 1) / *RU;
}

struct AttnLayout {
    size_t ml, o, stats, logits, total;
};
static AttnLayout attn_layout(const Kv4& c, int R, int rpt)
{
    int RT, RU, RB;
    attn_rows(R, rpt, &RT, &RU, &RB);
    AttnLayout w;
    w.ml = 256;
    w.o = w.ml + up256((size_t)kAttnMaxCtas * 2 * RU * sizeof(float2));
    w.stats = w.o + up256((size_t)kAttnMaxCtas * 2 * RU * c.D * sizeof(float));
    w.logits = w.stats + up256((size_t)c.B * c.H * RB * RU * sizeof(float2));
    w.total = w.logits + (c.weight ? up256((size_t)c.B * c.H * R * c.cap * sizeof(float)) : 0);
    return w;
}

template <typename T, int D, int G, int MODE>
static coreinfer_status launch_mode(AttnArgs& a, const DeviceInfo& di, cudaStream_t st)
{
    constexpr int RPT = MODE == kRows8 ? 8 : 4, NG = D / G, TILE = kAttnTile<D, G>;
    constexpr size_t STAGE = (size_t)TILE * (D / 2 + NG * 4);
    const size_t fixed = (size_t)kAttnWarps * RPT * (D * sizeof(float) + sizeof(float2)) + (2 * a.c.B + 1) * sizeof(int);
    // two CTAs per SM where registers (head_dim up to 128) and four stages each allow it
    int per_sm = D <= 128 ? 2 : 1, stages = 0;
    for (;; --per_sm) {
        const size_t room = (smem_room(di) - (per_sm - 1) * 1024) / per_sm;
        stages = room > fixed ? (int)((room - fixed) / STAGE) : 0;
        if (stages >= 4 || per_sm == 1) break;
    }
    if (stages < 4) CI_FAIL(COREINFER_ERR_UNSUPPORTED, "not enough shared memory for four pipeline stages");
    if (stages > kAttnMaxStages) stages = kAttnMaxStages;
    a.stages = stages;
    a.tile = TILE;
    const size_t smem = fixed + stages * STAGE;
    const long long tiles = (long long)a.c.B * a.c.H * a.RB * ((a.c.cap + TILE - 1) / TILE);
    if (tiles > (1LL << 30)) CI_FAIL(COREINFER_ERR_UNSUPPORTED, "the cache has %lld tiles of %d slots: too many for one call", tiles, TILE);
    long long ctas = (long long)di.sm_count * per_sm;
    if (ctas > kAttnMaxCtas) ctas = kAttnMaxCtas;
    if (ctas > tiles) ctas = tiles;
    a.n_ctas = (int)ctas;
    const coreinfer_status s = allow_smem<kv4_attention_kernel<T, D, G, MODE>>(di);
    if (s != COREINFER_OK) return s;
    kv4_attention_kernel<T, D, G, MODE><<<a.n_ctas, kAttnThreads, smem, st>>>(a);
    CI_CUDA(cudaGetLastError());

    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(a.R + (a.accumulate ? (a.c.cap + kFinishSlots - 1) / kFinishSlots : 0), a.c.B * a.c.H);
    cfg.blockDim = dim3(kFinishThreads);
    const size_t join = kAttnMaxCtas * sizeof(float) + kFinishThreads * sizeof(float4), rows = (size_t)a.R * (sizeof(float2) + sizeof(int));
    cfg.dynamicSmemBytes = join > rows ? join : rows;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    CI_CUDA(cudaLaunchKernelEx(&cfg, kv4_finish_kernel<T>, a));
    return COREINFER_OK;
}

// Rows per MMA tile for R query rows: fp32 and fp16 always carry two parts; bf16 takes the form with four rows where that
// is enough.
static inline int attn_rpt(coreinfer_dtype dtype, long long R) { return dtype != COREINFER_BF16 || R <= 4 ? 4 : 8; }

template <typename T, int D, int G>
static coreinfer_status launch_attention(AttnArgs& a, const DeviceInfo& di, cudaStream_t st)
{
    if constexpr (std::is_same<T, __nv_bfloat16>::value)
        return a.R <= 4 ? launch_mode<T, D, G, kRows4>(a, di, st) : launch_mode<T, D, G, kRows8>(a, di, st);
    else
        return launch_mode<T, D, G, kRows4Parts>(a, di, st);
}

template <typename T>
static coreinfer_status pick_attention(AttnArgs& a, const DeviceInfo& di, cudaStream_t st)
{
    const int D = a.c.D, G = a.c.G;
    if (D == 64) return G == 32 ? launch_attention<T, 64, 32>(a, di, st) : launch_attention<T, 64, 64>(a, di, st);
    if (D == 128)
        return G == 32 ? launch_attention<T, 128, 32>(a, di, st)
                       : (G == 64 ? launch_attention<T, 128, 64>(a, di, st) : launch_attention<T, 128, 128>(a, di, st));
    return G == 32 ? launch_attention<T, 256, 32>(a, di, st)
                   : (G == 64 ? launch_attention<T, 256, 64>(a, di, st) : launch_attention<T, 256, 128>(a, di, st));
}

constexpr int kAttnMaxRows = 2048;          // query rows per key head (they sit in shared memory of the finishing kernel)

}  // namespace coreinfer

using namespace coreinfer;

extern "C" {

size_t coreinfer_kv4_attention_workspace_bytes(const coreinfer_kv4_cache* cache, int32_t q_heads, int32_t T)
{
    Kv4 c;
    if (kv4_take(cache, "the", &c) != COREINFER_OK) return 0;
    if (q_heads < 1 || T < 1 || q_heads % c.H != 0 || T > COREINFER_KV4_MAX_QUERIES) return 0;
    const long long R = (long long)(q_heads / c.H) * T;
    if (R > kAttnMaxRows) return 0;
    const size_t x = attn_layout(c, (int)R, 8).total, y = attn_layout(c, (int)R, 4).total;
    return x > y ? x : y;
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
    const long long R = (long long)(q_heads / a.c.H) * T;
    if (R > kAttnMaxRows) CI_FAIL(COREINFER_ERR_UNSUPPORTED, "%lld query rows per key head: at most %d", R, kAttnMaxRows);
    if ((long long)a.c.B * a.c.H > 65535) CI_FAIL(COREINFER_ERR_UNSUPPORTED, "batch * kv_heads: at most 65535");
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
    const int rpt = attn_rpt(dtype, R);
    const AttnLayout w = attn_layout(a.c, (int)R, rpt);
    uint8_t* ws = (uint8_t*)workspace;
    a.q = q;
    a.out = out;
    a.ld_q = ld_q;
    a.ld_out = ld_out;
    a.Hq = q_heads;
    a.T = T;
    a.share = q_heads / a.c.H;
    a.R = (int)R;
    attn_rows(a.R, rpt, &a.RT, &a.RU, &a.RB);
    a.scale = scale;
    a.accumulate = accumulate ? 1 : 0;
    a.status = (unsigned*)ws;
    a.part_ml = (float2*)(ws + w.ml);
    a.part_o = (float*)(ws + w.o);
    a.stats = (float2*)(ws + w.stats);
    a.logits = (float*)(ws + w.logits);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (dtype == COREINFER_F32) return pick_attention<float>(a, di, st);
    if (dtype == COREINFER_BF16) return pick_attention<__nv_bfloat16>(a, di, st);
    return pick_attention<__half>(a, di, st);
}

}  // extern "C"
