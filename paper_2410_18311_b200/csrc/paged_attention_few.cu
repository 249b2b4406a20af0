// Attention of few query rows over a paged cache: 16-bit caches, one token a sequence or a few, split over their positions.
//
// What bounds it: the bytes of the slots that are seen, each read once.  tcgen05 would leave most of its 128 rows empty, so the
// products run on mma.sync.m16n8k16 with 16 positions on the M side and 8 query rows on the N side:  S^T = K Q^T, then
// O^T = V^T P^T, P^T made from the accumulators of S^T by movmatrix.  Weights enter as two parts (the value in 16 bits
// and what that leaves), so their rounding is below the output's: 16 bits of a weight for bf16, 22 for fp16.
//
// Persistent CTAs of 8 warps over the common list, two an SM or, where the outputs and queries of a warp's rows fill 255 registers (head_dim 128
// with 16 rows, 256), one.  A tile is 8 pieces of 16 positions (32 where head_dim is 64), one per warp.  Each
// warp brings its own pieces through a ring of three stages of its own, six where 128 leaves room (keys or values of a piece; cp.async, 16 bytes a
// lane) and keeps its own maximum, sum and output: no warp waits for another before the end of a unit.  Page numbers are loaded by
// the lanes 16 or 32 tiles ahead.  The maximum is moved only when a logit exceeds it by 2^8, which one vote finds out; fp16 weights are raised by
// 2^7 as in the form for chunks.  Slots that no row sees, or that lie in pages that are none, are not read but set to 0; values that only
// some rows see are looked through, and what is not finite is set to 0 and added at the end to the rows that see it.
//
// Measured from a graph, three sets of inputs, ragged lengths: 8 sequences x 32 heads x up to 4001 positions bf16 73 us, 5710 GB/s (under the
// profiler 74.7 us, 417 MB read, issue 49 %); 2 x 8 heads x 4 rows x up to 130000 fp16 152 us, 5920 GB/s; 16 x 8 heads x 8 rows x 4000 44 us;
// 4 x 32 heads x 200 12.4 us; 2 x 4 heads x 16 rows x 100000 71 us, 6 x 8 heads x 15 rows x 4096 of 9000 33 us (issue 37 %; twelve warps and rings
// of four take 78 and 38.7 where eight took 78 and 34.4).  Some 10 to 12 us do not grow with the length: launch and list 2 us, a unit's start (page, first slots) 3,
// its end (the warps' results) 3, the join.
#include "paged_attention.cuh"

namespace coreinfer {

constexpr int kFewWarps = 8;
constexpr int kFewThreads = 32 * kFewWarps;

template <int D> constexpr int kFewPiece = D == 64 ? 32 : 16;                       // positions of a piece
template <int D> constexpr int kFewStageBytes = kFewPiece<D> * D * 2;
template <int D, int NT> constexpr int kFewCtas = D * NT >= 256 ? 1 : 2;              // per SM
template <int D, int NT> constexpr int kFewStages = D == 128 && NT == 2 ? 6 : 3;

template <typename T>
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    if constexpr (std::is_same<T, __half>::value)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void load_matrices(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void load_matrices_trans(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t turn_matrix(uint32_t a)
{
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}
// The two values of a packed pair.
template <typename T>
__device__ __forceinline__ float2 unpack2(uint32_t w)
{
    const uint32_t high = w >> 16;
    return make_float2(to_f32<T>(*reinterpret_cast<const T*>(&w)), to_f32<T>(*reinterpret_cast<const T*>(&high)));
}

template <typename T, int D, int NT>
__global__ void __launch_bounds__(kFewThreads, kFewCtas<D, NT>) paged_few_kernel(const __grid_constant__ PagedAttnArgs a)
{
    constexpr int KW = kFewPiece<D>, KT = KW * kFewWarps, RU = 8 * NT;
    constexpr int STAGE = kFewStageBytes<D>, STAGES = kFewStages<D, NT>, RING = STAGES * STAGE;
    constexpr int CPR = D / 8;                       // 16-byte pieces of a slot
    constexpr int SPI = 32 / CPR;                    // slots that a warp copies at once
    constexpr int KS = D / 16;
    constexpr int HALVES = KW / 16;                  // pages a piece can touch
    constexpr int OP = D + 4;                        // row of the outputs in shared memory: lanes of a store hit 32 banks
    constexpr float LIFT = std::is_same<T, __half>::value ? 7.f : 0.f;
    static_assert(RU * OP * 4 <= RING, "a warp's outputs take its ring's place");
    extern __shared__ __align__(128) uint8_t smem[];
    float2* stats = reinterpret_cast<float2*>(smem + kFewWarps * RING);              // [warps][RU]
    int* found = reinterpret_cast<int*>(stats + kFewWarps * RU);
    int* at = reinterpret_cast<int*>(found + 2);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    uint8_t* ring = smem + warp * RING;
    const uint32_t ring_at = smem_u32(ring);
    if (tid == 0) found[0] = 0;                      // the plan's barriers stand between this and who sets it
    wait_for_stream();
    const int total = paged_plan(a, at);
    if (tid == 0) paged_first_words(a);
    int unit = 0;
    const long long page_bytes = a.c.page_stride * 2, head_bytes = a.c.head_stride * 2, slot_bytes = a.c.token_stride * 2;

    PagedWalk w;
    for (w.begin(a, at, total, blockIdx.x); w.more(); w.next(a, at)) {
        const int from = w.from(a), to = w.to(a);
        if (w.t.count > 0 && from >= to) continue;
        const int rows = paged_unit_rows(a, w), r0 = w.tile * RU;
        const PagedRow low = paged_row(a, w.s, r0), high = paged_row(a, w.s, r0 + rows - 1);
        const bool one_token = low.hi == high.hi && low.lo == high.lo;
        const int steps = 2 * (to - from);
        // pages of the next 32 / HALVES tiles, a lane each
        int pages = 0;
        auto fetch_pages = [&](int i0) {
            const int i = i0 + lane / HALVES;
            pages = i < to ? paged_page(a.c, w.b, paged_tile_at(w.t, i) * KT + warp * KW + lane % HALVES * 16) : -1;
        };
        auto issue = [&](int step, int stage) {
            if (step < steps) {
                const int i = from + step / 2;
                if ((step & 1) == 0 && (step / 2) % (32 / HALVES) == 0) fetch_pages(i);
                const int j0 = paged_tile_at(w.t, i) * KT + warp * KW;
                const bool all = j0 + KW <= high.hi && (j0 >= low.lo || j0 + KW <= a.sinks);
                const uint32_t dst = ring_at + stage * STAGE;
#pragma unroll
                for (int h = 0; h < HALVES; ++h) {
                    const int page = __shfl_sync(0xffffffffu, pages, (step / 2) % (32 / HALVES) * HALVES + h);
                    const uint8_t* src = a.c.pool[step & 1] + (page < 0 ? 0 : page) * page_bytes + w.h * head_bytes +
                                         ((j0 + 16 * h) & ((1 << a.c.page_shift) - 1)) * slot_bytes + lane % CPR * 16;
#pragma unroll
                    for (int x = 0; x < 16 / SPI; ++x) {
                        const int r = h * 16 + x * SPI + lane / CPR;
                        const int j = j0 + r;
                        const bool read = page >= 0 && (all || (j < high.hi && (j >= low.lo || j < a.sinks)));
                        const uint8_t* p = src + (x * SPI + lane / CPR) * slot_bytes;
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + r * (D * 2) + (((lane % CPR) ^ (r & 7)) << 4)),
                                     "l"(read ? p : a.c.pool[0]), "r"(read ? 16 : 0) : "memory");
                    }
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
#pragma unroll
        for (int x = 0; x < STAGES - 1; ++x) issue(x, x);
        // while the first slots are on their way:
        // queries as the second operand: row lane / 4 (of each group of eight), values 2 (lane % 4) and the next, and 8 further
        uint32_t q[NT][KS][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int r = n * 8 + lane / 4;
            const T* src = reinterpret_cast<const T*>(a.q) + (r < rows ? paged_row_offset(a, w.s, w.h, r0 + r, a.ld_q) : 0) + 2 * (lane & 3);
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                q[n][k][0] = r < rows ? *reinterpret_cast<const uint32_t*>(src + k * 16) : 0u;
                q[n][k][1] = r < rows ? *reinterpret_cast<const uint32_t*>(src + k * 16 + 8) : 0u;
            }
        }
        // a lane's rows: 2 (lane % 4) and the next of each group
        PagedRow see[NT][2];
        float m[NT][2], l[NT][2], o[NT][KS][4];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int r = n * 8 + 2 * (lane & 3) + e;
                see[n][e] = paged_row(a, w.s, r0 + (r < rows ? r : rows - 1));
                m[n][e] = -INFINITY;
                l[n][e] = 0.f;
            }
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[n][k][e] = 0.f;
        }

        int stage = 0;
        bool odd = false;
        for (int i = from; i < to; ++i) {
            const int j0 = paged_tile_at(w.t, i) * KT + warp * KW;
            const int step = 2 * (i - from);
            float s[NT][HALVES][4];
            // ---- keys
            asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
            __syncwarp();
            issue(step + STAGES - 1, stage == 0 ? STAGES - 1 : stage - 1);
            const uint32_t key_at = ring_at + stage * STAGE;
#pragma unroll
            for (int h = 0; h < HALVES; ++h) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[n][h][e] = 0.f;
                const int r = h * 16 + (lane & 15);
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    uint32_t f[4];
                    load_matrices(f, key_at + r * (D * 2) + (((2 * k + (lane >> 4)) ^ (r & 7)) << 4));
#pragma unroll
                    for (int n = 0; n < NT; ++n) mma16816<T>(s[n][h], f, q[n][k][0], q[n][k][1]);
                }
            }
            if (++stage == STAGES) stage = 0;
            // ---- weights: element e of a half is position lane / 4 (+ 8 for e >= 2), row 2 (lane % 4) + e % 2
            const bool whole = j0 + KW <= low.hi && (j0 >= high.lo || j0 + KW <= a.sinks);
            bool move = false;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int h = 0; h < HALVES; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float& x = s[n][h][e];
                        x *= a.scale2;
                        if (!whole && !paged_sees(a, see[n][e & 1], j0 + h * 16 + lane / 4 + (e >= 2 ? 8 : 0))) x = -INFINITY;
                        move |= x > m[n][e & 1] + (8.f + LIFT);
                    }
            if (__any_sync(0xffffffffu, move)) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float now = fmaxf(s[n][0][e], s[n][0][e + 2]);
                        if (HALVES == 2) now = fmaxf(now, fmaxf(s[n][HALVES - 1][e], s[n][HALVES - 1][e + 2]));
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1) now = fmaxf(now, __shfl_xor_sync(0xffffffffu, now, d));
                        if (now > m[n][e] + LIFT) {
                            const float by = m[n][e] == -INFINITY ? 1.f : exp2_fast(m[n][e] - (now - LIFT));
                            m[n][e] = now - LIFT;
                            l[n][e] *= by;
#pragma unroll
                            for (int k = 0; k < KS; ++k) {
                                o[n][k][e] *= by;
                                o[n][k][e + 2] *= by;
                            }
                        }
                    }
            }
            uint32_t p[NT][HALVES][2][2];            // [..][positions 0..7, 8..15][part]
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float ref0 = m[n][0] == -INFINITY ? 0.f : m[n][0], ref1 = m[n][1] == -INFINITY ? 0.f : m[n][1];
#pragma unroll
                for (int h = 0; h < HALVES; ++h)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float p0 = exp2_fast(s[n][h][2 * e] - ref0), p1 = exp2_fast(s[n][h][2 * e + 1] - ref1);
                        l[n][0] += p0;
                        l[n][1] += p1;
                        const uint32_t high = pack2<T>(p0, p1);
                        const float2 back = unpack2<T>(high);
                        p[n][h][e][0] = turn_matrix(high);
                        p[n][h][e][1] = turn_matrix(pack2<T>(p0 - back.x, p1 - back.y));
                    }
            }
            // ---- values
            asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
            __syncwarp();
            issue(step + STAGES, stage == 0 ? STAGES - 1 : stage - 1);
            const uint32_t value_at = ring_at + stage * STAGE;
            const bool look = !whole && !one_token;
#pragma unroll
            for (int h = 0; h < HALVES; ++h) {
                const int r = h * 16 + (lane & 7) + (lane >> 4) * 8;
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    uint32_t f[4];
                    load_matrices_trans(f, value_at + r * (D * 2) + (((2 * k + (lane >> 3 & 1)) ^ (r & 7)) << 4));
                    if (look) {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (odd_pair<T>(f[e])) {
                                f[e] = without_odd<T>(f[e]);
                                odd = true;
                            }
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        mma16816<T>(o[n][k], f, p[n][h][0][0], p[n][h][1][0]);
                        mma16816<T>(o[n][k], f, p[n][h][0][1], p[n][h][1][1]);
                    }
                }
            }
            if (++stage == STAGES) stage = 0;
        }

        // ---- the warps' results: maxima and sums, then outputs in the rings' place
        asm volatile("cp.async.wait_all;" ::: "memory");
        if (odd) *(volatile int*)&found[unit & 1] = 1;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], d);
                const int r = n * 8 + 2 * (lane & 3) + e;
                if (lane < 4) stats[warp * RU + r] = make_float2(m[n][e], l[n][e]);
            }
        __syncwarp();
        float* mine = reinterpret_cast<float*>(ring);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int k = 0; k < KS; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int r = n * 8 + 2 * (lane & 3) + (e & 1);
                    if (r < rows) mine[r * OP + k * 16 + lane / 4 + (e >= 2 ? 8 : 0)] = o[n][k][e];
                }
        __syncthreads();
        const bool head = from == 0, tail = to == w.t.count;
        const bool restore = *(volatile int*)&found[unit & 1] != 0;
        if (tid == 0) found[++unit & 1] = 0;         // nobody writes the next unit's before the barrier below
        else ++unit;
        const size_t slot = (size_t)blockIdx.x * 2 + (head ? 1 : 0);
        for (int x = tid; x < rows * (D / 4); x += kFewThreads) {
            const int r = x / (D / 4), d = x % (D / 4) * 4;
            float top = -INFINITY;
#pragma unroll
            for (int y = 0; y < kFewWarps; ++y) top = fmaxf(top, stats[y * RU + r].x);
            const float ref = top == -INFINITY ? 0.f : top;
            float sum = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int y = 0; y < kFewWarps; ++y) {
                const float2 st = stats[y * RU + r];
                const float f = exp2_fast(st.x - ref);
                sum = fmaf(st.y, f, sum);
                const float4 part = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(smem + y * RING) + r * OP + d);
                if (st.x != -INFINITY) {
                    v[0] = fmaf(part.x, f, v[0]);
                    v[1] = fmaf(part.y, f, v[1]);
                    v[2] = fmaf(part.z, f, v[2]);
                    v[3] = fmaf(part.w, f, v[3]);
                }
            }
            if (restore)
                for (int e = 0; e < 4; ++e) v[e] += paged_odd_sum<T>(a, w, low.hi, high.lo, from, to, r0 + r, d + e);
            if (head && tail) {
                const bool sees = paged_sees_some(a, paged_row(a, w.s, r0 + r));
                const float inv = 1.f / sum;
                uint2 packed = make_uint2(pack2<T>(v[0] * inv, v[1] * inv), pack2<T>(v[2] * inv, v[3] * inv));
                if (!sees) packed = make_uint2(0u, 0u);
                *reinterpret_cast<uint2*>(reinterpret_cast<T*>(a.out) + paged_row_offset(a, w.s, w.h, r0 + r, a.ld_out) + d) = packed;
            } else {
                *reinterpret_cast<float4*>(a.part_o + slot * RU * D + (d * RU + r * 4)) = make_float4(v[0], v[1], v[2], v[3]);
                if (d == 0) a.part_ml[slot * RU + r] = make_float2(top, sum);
            }
        }
        if (head && !tail && tid == 0) {
            PagedPiece piece;
            piece.b = w.b;
            piece.h = w.h;
            piece.tile = w.tile;
            piece.last = w.last(a, at);
            a.pieces[blockIdx.x] = piece;
        }
        __syncthreads();
    }
    let_next_start();
}

template <typename T, int D, int NT>
static coreinfer_status launch_few(const PagedAttnArgs& a, const DeviceInfo& di, cudaStream_t st)
{
    const size_t smem = (size_t)kFewWarps * kFewStages<D, NT> * kFewStageBytes<D> + kFewWarps * 8 * NT * sizeof(float2) + 8 + paged_list_bytes(a.c.B);
    const coreinfer_status s = allow_smem<paged_few_kernel<T, D, NT>>(di, 0);
    if (s != COREINFER_OK) return s;
    CI_CUDA(launch_overlapped(paged_few_kernel<T, D, NT>, dim3(a.n_ctas), dim3(kFewThreads), smem, st, a));
    return COREINFER_OK;
}
template <typename T, int D>
static coreinfer_status few_rows(const PagedAttnArgs& a, const DeviceInfo& di, cudaStream_t st)
{
    return a.RU == 8 ? launch_few<T, D, 1>(a, di, st) : launch_few<T, D, 2>(a, di, st);
}
template <typename T>
static coreinfer_status few_dim(const PagedAttnArgs& a, const DeviceInfo& di, cudaStream_t st)
{
    if (a.c.D == 64) return few_rows<T, 64>(a, di, st);
    return a.c.D == 128 ? few_rows<T, 128>(a, di, st) : few_rows<T, 256>(a, di, st);
}

coreinfer_status paged_few(const PagedAttnArgs& a, bool f16, const DeviceInfo& di, cudaStream_t st)
{
    return f16 ? few_dim<__half>(a, di, st) : few_dim<__nv_bfloat16>(a, di, st);
}

}  // namespace coreinfer
