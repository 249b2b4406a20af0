// Attention of chunks over a paged cache on the tensor cores: 16-bit caches, many query rows per key head.
//
// What bounds it: both products and the exponentials alike.  Per SM a tile of 128 rows x 128 positions x head_dim 128 takes 1024 cycles
// of tcgen05.mma and, at 16 exponentials a cycle, 1024 cycles of those; so two row tiles run against each other: while one is in its
// softmax the other is in its products.
//
// One persistent CTA per SM; a unit is 256 query rows of one sequence and key head, as two tiles A and B of 128 that share every
// tile of 128 positions (head_dim 256: one tile of 128 rows, whose O takes half of tensor memory).
//   warps 0..7   softmax of A, two threads a row with 64 columns each (they exchange their maxima through shared memory): S from tensor memory, P back
//   warps 8..15  over it in 16 bits, maximum and sum in registers; the same for B.  They write their rows out at the end of a unit
//   warp 16      brings key and value tiles into a ring by tensor copies, a page (or 128 slots of it) a box; pages that are none
//                lie outside the map and are filled with zeros
//   warp 17      one lane issues  S = Q K^T  into tensor memory, and  O += P V  with P from tensor memory, in the order
//                PV_A(i) S_A(i+1) PV_B(i) S_B(i+1)
//   warps 18,19  bring the next unit's queries (by tensor copies where whole tokens fill a tile), and look through value tiles in which
//                some row does not see some position
// The running maximum is moved, and O rescaled, only when a row exceeds it by 2^8 (a factor that cancels in O / l): P then stays below
// 2^8, and in fp16 it is raised by 2^7 so that weights keep 11 bits down to 2^-21 of the largest.  P is rounded to the cache's type
// for the product, as tcgen05.mma takes both operands in one type: an error of half a step of each weight, which averages out to
// about the rounding of the output; the sum l is of the weights before that.
// A weight of 0 times a value that is not finite would be NaN, and positions that a row does not see, or that hold no token, may
// hold anything: in tiles where that can happen the helpers set what is not finite to 0, and at the unit's end the rows that do see such
// a value get it added.
// Every wait is bounded: one that gives up sets the status word, and all roles leave their loops.
//
// The tensor cores cut what does not fit a sum's 24 bits: a CTA's sum over n positions of values of one sign comes out up to about n / 16 x 1.3 x
// 2^-24 too small (130000 positions: 0.6 of a step of fp16), which of values of both signs is lost in the rounding.
//
// Measured from a graph, three sets of inputs, in short bursts at 1965 MHz and, where the power limit lowers the clock, over two seconds: a prompt of
// 8192 tokens x 32 heads of 128 bf16 542 us (1015 TFLOP/s of what the mask leaves) and 632 (870, 1575 MHz); 500 tokens x 40 heads, five a key head, over
// 16000 positions fp16 168 (960) and 187 us (865, 1657 MHz; under the profiler tensor pipe 53 %, exponentials 54 %, issue 39 %); 2 x 1000 x 16
// heads of 256 over 4000 170 us (485); seven sequences, windows of 1024, 32 heads of 64 fp16 150 us (354: 11 tiles a unit, four of them masked).
// ptxas spills 84 to 116 bytes a thread at 96 registers (which setmaxnreg then divides).
// A tile of 128 positions for both row tiles takes 3400 to 3700 cycles at head_dim 128, where products alone would take 2050 (tcgen05.mma
// M 128 N 128 K 16: 64 cycles each, also with A in tensor memory) and exponentials alone as many: scores, maximum, weights and product of a row tile follow
// one another (170, 450, 1300 and 1500 cycles with the hand-overs), and two row tiles do not quite hide that; starting a unit costs about
// 6000 cycles more.  Tried and slower or no better: halves of 64 positions with S doubled (N 64 products take 52 cycles for half the work),
// one thread a row, P handed over in halves, products issued by two warps, part of the exponentials as polynomials, P apart from S at head_dim 64,
// units of at most 128 rows split by tiles between both pipelines.
#include "paged_attention.cuh"
#include "tc.cuh"

#include <type_traits>

namespace coreinfer {

constexpr int kChunkThreads = 640;
constexpr int kChunkKT = kPagedChunkTile;
constexpr int kChunkMaxStages = 8;
constexpr long long kChunkWaitCycles = 3000000000LL;
constexpr float kNoMax = -INFINITY;
// Row tiles of a unit: O takes head_dim columns of tensor memory for each, beside 128 of S.
template <int D> constexpr int kChunkPipes = D == 256 ? 1 : 2;

struct ChunkArgs {
    PagedAttnArgs a;
    int k_stages, v_stages; // rings of key and of value tiles
    int box;                // slots of a tensor copy
    int sign;               // of the scale; below 0 the queries' signs are turned, at 0 they are multiplied by it
    int map_q;              // queries come by tensor copies
};

struct ChunkBars {
    uint64_t full[kChunkMaxStages], empty[kChunkMaxStages], looked[kChunkMaxStages];
    uint64_t s_full[2], p_full[2], o_full[2], q_full[2], q_empty;
    float row[2][2][128];   // by tile and half: a row's maximum of its 64 columns, at a unit's end its sum
    uint32_t tmem;
    int abort;
    int found[4];           // by unit modulo 4: number + 1 of a unit in which values were set to 0
};

// What the rows of one of the two tiles see.
struct ChunkView {
    bool any;
    int lo_min, lo_max, hi_min, hi_max;
};
__device__ __forceinline__ ChunkView chunk_view(const PagedAttnArgs& a, const PagedWalk& w, int rows, int x)
{
    ChunkView v;
    v.any = rows > x * 128;
    v.lo_min = v.lo_max = v.hi_min = v.hi_max = 0;
    if (!v.any) return v;
    const int r0 = w.tile * a.RU + x * 128, r1 = w.tile * a.RU + (rows < x * 128 + 128 ? rows : x * 128 + 128) - 1;
    const PagedRow low = paged_row(a, w.s, r0), high = paged_row(a, w.s, r1);
    v.lo_min = low.lo;
    v.lo_max = high.lo;
    v.hi_min = low.hi;
    v.hi_max = high.hi;
    return v;
}
// Some row sees some position of the tile from j on.
__device__ __forceinline__ bool chunk_needs(const PagedAttnArgs& a, const ChunkView& v, int j)
{
    return v.any && j < v.hi_max && (j + kChunkKT > v.lo_min || j < a.sinks);
}
// Every row sees all of it.
__device__ __forceinline__ bool chunk_whole(const PagedAttnArgs& a, const ChunkView& v, int j)
{
    return j + kChunkKT <= v.hi_min && (j >= v.lo_max || j + kChunkKT <= a.sinks);
}
// Some row of a tile that takes part does not: the values are looked through.
__device__ __forceinline__ bool chunk_look(const PagedAttnArgs& a, const ChunkView& va, const ChunkView& vb, int j)
{
    return (chunk_needs(a, va, j) && !chunk_whole(a, va, j)) || (chunk_needs(a, vb, j) && !chunk_whole(a, vb, j));
}

// Called by whole warps, whose lanes all get the same answer: false when the wait gave up.
__device__ __forceinline__ bool chunk_wait(uint64_t& bar, uint32_t parity, ChunkBars* s, unsigned* status)
{
    const uint32_t b = smem_u32(&bar);
    if (__all_sync(0xffffffffu, mbar_try_wait(b, parity))) return true;
    const long long t0 = clock64();
    volatile int* abort_flag = &s->abort;
    for (;;) {
        if (__all_sync(0xffffffffu, mbar_try_wait_parked(b, parity, 2000u))) return true;
        const bool late = clock64() - t0 > kChunkWaitCycles;
        if (__any_sync(0xffffffffu, late || *abort_flag)) {
            if (late) {
                *abort_flag = 1;
                atomicMax(status, (unsigned)kStatusTimeout);
            }
            return false;
        }
    }
}

// The same for one thread.
__device__ __forceinline__ bool chunk_wait_one(uint64_t& bar, uint32_t parity, ChunkBars* s, unsigned* status)
{
    const uint32_t b = smem_u32(&bar);
    if (mbar_try_wait(b, parity)) return true;
    const long long t0 = clock64();
    volatile int* abort_flag = &s->abort;
    for (;;) {
        if (mbar_try_wait_parked(b, parity, 2000u)) return true;
        if (*abort_flag) return false;
        if (clock64() - t0 > kChunkWaitCycles) {
            *abort_flag = 1;
            atomicMax(status, (unsigned)kStatusTimeout);
            return false;
        }
    }
}
// 32 bytes of a row, in one store where the address is a multiple of 32.
__device__ __forceinline__ void store32(void* to, const uint32_t* w, bool wide)
{
    if (wide)
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                     ::"l"(to), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
    else {
        reinterpret_cast<uint4*>(to)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        reinterpret_cast<uint4*>(to)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
}
// Two fp32 numbers in a register pair, for the instructions that take both at once.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair(float a, float b)
{
    f32x2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void split(f32x2 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c)
{
    f32x2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b)
{
    f32x2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ float max3_nan(float a, float b, float c)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// The maximum of 32 values in four parts; -infinity where a bit is not set.
__device__ __forceinline__ void top32(float (&top)[4], const uint32_t* f)
{
#pragma unroll
    for (int e = 0; e < 32; e += 2) top[e / 2 & 3] = max3_nan(top[e / 2 & 3], __uint_as_float(f[e]), __uint_as_float(f[e + 1]));
}
__device__ __forceinline__ void mask32(uint32_t* f, uint32_t seen)
{
#pragma unroll
    for (int e = 0; e < 32; ++e)
        if (!(seen >> e & 1u)) f[e] = 0xff800000u;
}
// Two 16-bit values times 0: NaN where they are not finite, as an infinity's or NaN's bits with those one place lower are.
template <typename T>
__device__ __forceinline__ uint32_t times_zero(uint32_t w)
{
    const uint32_t odd = w ^ without_odd<T>(w);
    return odd | odd >> 1;
}
// Bits 0 .. n - 1.
__device__ __forceinline__ uint32_t bits_below(int n) { return n <= 0 ? 0u : (n >= 32 ? 0xffffffffu : (1u << n) - 1u); }

template <typename T, int D>
__global__ void __launch_bounds__(kChunkThreads, 1) paged_chunk_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                                                                        const __grid_constant__ CUtensorMap map_q,
                                                                        const __grid_constant__ ChunkArgs g)
{
    constexpr int KT = kChunkKT;
    constexpr int BLOCKS = D / 64;
    constexpr uint32_t BLOCK = 128 * 128;            // bytes of 128 rows of 64 values
    constexpr uint32_t TILE = BLOCKS * BLOCK;
    constexpr uint32_t TYPE = std::is_same<T, __half>::value ? 0u : 1u;
    constexpr uint32_t IDESC_S = tc::idesc(TYPE, false, 128, KT);
    constexpr uint32_t IDESC_O = tc::idesc(TYPE, true, 128, D);
    constexpr float LIFT = std::is_same<T, __half>::value ? 7.f : 0.f;
    constexpr int PIPES = kChunkPipes<D>;
    const PagedAttnArgs& a = g.a;
    extern __shared__ __align__(1024) uint8_t smem[];
    uint8_t* qs = smem;                              // [PIPES][BLOCKS][128 rows][128 bytes]
    // Two rings [stages][BLOCKS][128 positions][128 bytes], of keys and of values: copies may land out of their order, and who waits for value
    // tiles alone must not take a phase of its barrier that a key tile ended for its own.
    uint8_t* ring = smem + PIPES * TILE;
    const int stages = g.k_stages + g.v_stages;
    ChunkBars* s = reinterpret_cast<ChunkBars*>(ring + (size_t)stages * TILE);
    int* at = reinterpret_cast<int*>(s + 1);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    if (tid == 0) {
        for (int i = 0; i < stages; ++i) {
            mbar_init(smem_u32(&s->full[i]), 1);
            mbar_init(smem_u32(&s->empty[i]), 1);
            mbar_init(smem_u32(&s->looked[i]), 2);
        }
        for (int x = 0; x < 2; ++x) {
            mbar_init(smem_u32(&s->s_full[x]), 1);
            mbar_init(smem_u32(&s->p_full[x]), 8);
            mbar_init(smem_u32(&s->o_full[x]), 1);
            mbar_init(smem_u32(&s->q_full[x]), 2);
        }
        mbar_init(smem_u32(&s->q_empty), 1);
        s->abort = 0;
        for (int i = 0; i < 4; ++i) s->found[i] = 0;
        mbar_fence_init();
    }
    if (warp == 17) tc::alloc(smem_u32(&s->tmem), 512);
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    const uint32_t tmem = s->tmem;
    wait_for_stream();
    const int total = paged_plan(a, at);
    if (tid == 576) paged_first_words(a);            // the thread that names the unit which others join

    if (warp >= 16) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        if (warp == 16) {
            // ------------------------------------------------------- tiles --
            int at_stage[2] = {0, 0};
            uint32_t phase[2] = {0, 0};
            bool ok = true;
            const int boxes = KT / g.box;
            PagedWalk w;
            for (w.begin(a, at, total, blockIdx.x); ok && w.more(); w.next(a, at)) {
                const int from = w.from(a), to = w.to(a);
                for (int i = from; ok && i < to; ++i) {
                    const int j = paged_tile_at(w.t, i) * KT + lane * g.box;
                    int page = lane < boxes ? paged_page(a.c, w.b, j) : 0;
                    if (page < 0) page = a.c.n_pages;            // outside the map: zeros
                    const int slot = j & ((1 << a.c.page_shift) - 1);
#pragma unroll
                    for (int kv = 0; kv < 2; ++kv) {
                        const int stage = at_stage[kv] + (kv ? g.k_stages : 0);
                        if (!(ok = chunk_wait(s->empty[stage], phase[kv] ^ 1u, s, a.status))) break;
                        const uint32_t bar = smem_u32(&s->full[stage]);
                        if (lane == 0) mbar_arrive_expect_tx(bar, TILE);
                        __syncwarp();
                        if (lane < boxes) {
                            const uint32_t dst = smem_u32(ring + (size_t)stage * TILE) + lane * g.box * 128;
#pragma unroll
                            for (int d = 0; d < BLOCKS; ++d) tc::copy_4d(dst + d * BLOCK, kv ? &map_v : &map_k, d * 64, slot, w.h, page, bar);
                        }
                        if (++at_stage[kv] == (kv ? g.v_stages : g.k_stages)) { at_stage[kv] = 0; phase[kv] ^= 1u; }
                    }
                }
            }
        } else if (warp == 17) {
            // ---------------------------------------------------- products --
            // One lane does all of it.  The tensor cores' queue holds about four products, so what lies between two groups of them has to
            // take less than those: no votes, no warp barriers, descriptors by their low words, which halves take part by two bounds.
            PagedWalk w;
            w.begin(a, at, total, blockIdx.x);
            if (tc::elect()) {
                int ks = 0, vs = 0;                              // stages of the next K and V
                uint32_t k_ph = 0, v_ph = 0, p_ph[2] = {0, 0}, q_ph[2] = {0, 0};
                bool ok = true;
                const uint32_t q_desc = tc::desc_k(smem_u32(qs)), k_desc = tc::desc_k(smem_u32(ring)), v_desc = tc::desc_mn(smem_u32(ring + (size_t)g.k_stages * TILE), BLOCK);
                auto next_k = [&]() { if (++ks == g.k_stages) { ks = 0; k_ph ^= 1u; } };
                auto scores = [&](int x, int st) {
                    const uint32_t q = q_desc + x * (TILE >> 4), k = k_desc + st * (TILE >> 4);
#pragma unroll
                    for (int d = 0; d < D / 16; ++d) {
                        const uint32_t ofs = (d / 4) * (BLOCK >> 4) + (d % 4) * 2;
                        tc::mma_ss(tmem + x * 128, q + ofs, k + ofs, tc::desc_high, IDESC_S, d > 0);
                    }
                    tc::commit(smem_u32(&s->s_full[x]));
                };
                for (; ok && w.more(); w.next(a, at)) {
                    const int from = w.from(a), to = w.to(a);
                    if (from >= to) continue;
                    const int rows = paged_unit_rows(a, w);
                    // tiles of the list that take part, below end[x]: those of the first tokens, and from first[x] on
                    int first[2], end[2];
                    const int sinks_end = (a.sinks + KT - 1) / KT - w.t.from + w.t.first_tiles;
                    const int sink_tiles = sinks_end > w.t.first_tiles ? sinks_end : w.t.first_tiles;
                    bool begun[2] = {false, false};
#pragma unroll
                    for (int x = 0; x < PIPES; ++x) {
                        const ChunkView v = chunk_view(a, w, rows, x);
                        first[x] = v.any ? (v.lo_min > 0 ? v.lo_min / KT : 0) - w.t.from + w.t.first_tiles : to;
                        end[x] = v.any ? (v.hi_max + KT - 1) / KT - w.t.from + w.t.first_tiles : 0;
                    }
                    auto needs = [&](int x, int i) { return i < end[x] && (i < sink_tiles || i >= first[x]); };
                    if (!(ok = chunk_wait_one(s->full[ks], k_ph, s, a.status))) break;
#pragma unroll
                    for (int x = 0; x < PIPES; ++x) {
                        if (x * 128 >= rows) continue;
                        if (ok) ok = chunk_wait_one(s->q_full[x], q_ph[x], s, a.status);
                        q_ph[x] ^= 1u;
                        tc::fence_after();
                        if (ok && needs(x, from)) scores(x, ks);
                    }
                    if (!ok) break;
                    tc::commit(smem_u32(&s->empty[ks]));
                    if (from + 1 == to) tc::commit(smem_u32(&s->q_empty));
                    next_k();
                    for (int i = from; i < to; ++i) {
                        // V(i), which is there when it has been looked at, and K(i + 1)
                        const bool last = i + 1 == to;
                        if (!(ok = chunk_wait_one(s->looked[vs], v_ph, s, a.status))) break;
                        if (!last && !(ok = chunk_wait_one(s->full[ks], k_ph, s, a.status))) break;
                        const uint32_t val = v_desc + vs * (TILE >> 4);
#pragma unroll
                        for (int x = 0; x < PIPES; ++x) {
                            if (ok && needs(x, i)) {
                                ok = chunk_wait_one(s->p_full[x], p_ph[x], s, a.status);
                                p_ph[x] ^= 1u;
                                tc::fence_after();
                                if (ok) {
#pragma unroll
                                    for (int k = 0; k < KT / 16; ++k)
                                        tc::mma_ts(tmem + 256 + x * 128, tmem + x * 128 + (k >> 2) * 64 + (k & 3) * 8, val + k * (16 * 128 >> 4), tc::desc_high,
                                                   IDESC_O, begun[x] || k > 0);
                                    // the last of them: the row tile's results may be read
                                    if (last || !needs(x, i + 1)) {
                                        bool more = false;
                                        for (int n = i + 2; n < to && !more; ++n) more = needs(x, n);
                                        if (last || !more) tc::commit(smem_u32(&s->o_full[x]));
                                    }
                                }
                                begun[x] = true;
                            }
                            if (ok && !last && needs(x, i + 1)) scores(x, ks);
                        }
                        if (!ok) break;
                        tc::commit(smem_u32(&s->empty[g.k_stages + vs]));
                        if (++vs == g.v_stages) { vs = 0; v_ph ^= 1u; }
                        if (!last) {
                            tc::commit(smem_u32(&s->empty[ks]));
                            if (i + 2 == to) tc::commit(smem_u32(&s->q_empty));
                            next_k();
                        }
                    }
                }
            }
            __syncwarp();
        } else {
            // ------------------------------------- queries, looks at values --
            const int t = tid - 576;
            int stage = 0, unit = 0;                             // of value tiles
            uint32_t ph = 0, q_ph = 0;
            bool ok = true;
            PagedWalk w;
            for (w.begin(a, at, total, blockIdx.x); ok && w.more(); w.next(a, at)) {
                const int from = w.from(a), to = w.to(a);
                if (from >= to) continue;
                if (t == 0 && from == 0 && to < w.t.count) {
                    PagedPiece p;
                    p.b = w.b;
                    p.h = w.h;
                    p.tile = w.tile;
                    p.last = w.last(a, at);
                    a.pieces[blockIdx.x] = p;
                }
                const int rows = paged_unit_rows(a, w);
                const ChunkView va = chunk_view(a, w, rows, 0), vb = chunk_view(a, w, rows, 1);
                if (!(ok = chunk_wait(s->q_empty, q_ph ^ 1u, s, a.status))) break;
                q_ph ^= 1u;
                if (g.map_q) {                                   // rows of a tile: 128 / share tokens, each the heads of the group
                    if (t < 2 && t * 128 < rows) {
                        const uint32_t bar = smem_u32(&s->q_full[t]);
                        mbar_arrive_expect_tx(bar, TILE);
                        const int token = w.s.first + by_share(a, w.tile * a.RU + t * 128);
#pragma unroll
                        for (int d = 0; d < BLOCKS; ++d) tc::copy_3d(smem_u32(qs) + t * TILE + d * BLOCK, &map_q, d * 64, w.h * a.share, token, bar);
                        mbar_arrive(bar);
                    }
                } else {
                // a lane brings the same 16 bytes of every row that is its own, rows STEP apart
                constexpr int CPR = D / 8, STEP = 64 / CPR;
                const int c = t % CPR, r_first = w.tile * a.RU;
                const int token_step = by_share(a, STEP), head_step = STEP - token_step * a.share;
                int token = by_share(a, r_first + t / CPR), head = r_first + t / CPR - token * a.share;
                const uint8_t* base = a.q + ((long long)w.s.first * a.ld_q + (long long)w.h * a.share * D + c * 8) * 2;
#pragma unroll
                for (int x = 0; x < PIPES; ++x) {
                    if (x * 128 < rows) {
                        const uint32_t to_tile = smem_u32(qs) + x * TILE + (c >> 3) * BLOCK;
#pragma unroll 4
                        for (int r = t / CPR; r < 128; r += STEP) {
                            const bool live = x * 128 + r < rows;
                            const uint8_t* src = base + ((long long)token * a.ld_q + head * D) * 2;
                            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to_tile + r * 128 + (((c & 7) ^ (r & 7)) << 4)),
                                         "l"(live ? src : a.q), "r"(live ? 16 : 0) : "memory");
                            token += token_step;
                            head += head_step;
                            if (head >= a.share) { head -= a.share; ++token; }
                        }
                    }
                    asm volatile("cp.async.commit_group;" ::: "memory");
                }
#pragma unroll
                for (int x = 0; x < PIPES; ++x) {
                    if (x + 1 < PIPES) asm volatile("cp.async.wait_group 1;" ::: "memory");
                    else asm volatile("cp.async.wait_group 0;" ::: "memory");
                    if (x * 128 >= rows) continue;
                    if (g.sign <= 0) {                           // each lane turns what it has brought itself
                        for (int r = t / CPR; r < 128; r += STEP) {
                            uint4* p = reinterpret_cast<uint4*>(qs + x * TILE + (c >> 3) * BLOCK + r * 128 + (((c & 7) ^ (r & 7)) << 4));
                            uint4 y = *p;
                            if (g.sign < 0) { y.x ^= 0x80008000u; y.y ^= 0x80008000u; y.z ^= 0x80008000u; y.w ^= 0x80008000u; }
                            else y = make_uint4(times_zero<T>(y.x), times_zero<T>(y.y), times_zero<T>(y.z), times_zero<T>(y.w));
                            *p = y;
                        }
                    }
                    fence_proxy_async();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&s->q_full[x]));
                }
                }
                for (int i = from; i < to; ++i) {
                    const int j = paged_tile_at(w.t, i) * KT;
                    // each tile is waited for, so that neither the ring nor this warp is ever a round ahead of the other
                    if (!(ok = chunk_wait(s->full[g.k_stages + stage], ph, s, a.status))) break;
                    if (chunk_look(a, va, vb, j)) {
                        uint4* p = reinterpret_cast<uint4*>(ring + (size_t)(g.k_stages + stage) * TILE);
                        const int hi = va.hi_max > vb.hi_max ? va.hi_max : vb.hi_max;
                        bool odd = false, wrote = false;
#pragma unroll 4
                        for (int c = t; c < (int)(TILE / 16); c += 64) {
                            uint4 x = p[c];
                            if (odd_pair<T>(x.x) || odd_pair<T>(x.y) || odd_pair<T>(x.z) || odd_pair<T>(x.w)) {
                                x.x = without_odd<T>(x.x); x.y = without_odd<T>(x.y); x.z = without_odd<T>(x.z); x.w = without_odd<T>(x.w);
                                p[c] = x;
                                wrote = true;
                                const int at_j = j + (c >> 3 & 127);     // what no row sees is not missed
                                odd = odd || (at_j < hi && (at_j >= va.lo_min || at_j < a.sinks));
                            }
                        }
                        // the product and the copy that takes the tile's place come behind these stores, whoever sees what was there
                        if (wrote) fence_proxy_async();
                        if (odd) *(volatile int*)&s->found[unit & 3] = unit + 1;
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&s->looked[stage]));
                    if (++stage == g.v_stages) { stage = 0; ph ^= 1u; }
                }
                ++unit;
            }
        }
    } else {
        // -------------------------------------------------------- softmax --
        asm volatile("setmaxnreg.inc.sync.aligned.u32 104;");
        const int x = warp >> 3, h = warp >> 2 & 1;              // with one row tile a unit the second eight warps have no rows
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t t_s = tmem + lanes + x * 128 + h * 64, t_o = tmem + lanes + 256 + x * 128 + h * (D / 2);
        const int r = (warp & 3) * 32 + lane;                    // row of the tile
        const float scale2 = g.sign ? fabsf(a.scale2) : 1.f;     // above 0: times the -infinity of what is masked it stays that
        float* mine_s = &s->row[x][h][r];
        const volatile float* other_s = &s->row[x][h ^ 1][r];
        uint32_t s_ph = 0, o_ph = 0;
        int unit = 0;
        bool ok = true;
        // The eight warps of the row tile meet at a hardware barrier.  It cannot give up by itself, so no warp goes there once some wait
        // has (the flag is looked at before), and one that leaves for that reason arrives once, for those that are there already.
        auto meet_again = [&]() {
            if (__any_sync(0xffffffffu, *(volatile int*)&s->abort)) return false;
            named_bar_sync(1 + x, 256);
            return true;
        };
        auto meet = [&](float value) {
            *mine_s = value;
            return meet_again();
        };
        PagedWalk w;
        for (w.begin(a, at, total, blockIdx.x); ok && w.more(); w.next(a, at)) {
            const int from = w.from(a), to = w.to(a);
            if (w.t.count > 0 && from >= to) continue;
            const int rows = paged_unit_rows(a, w);
            const ChunkView v = chunk_view(a, w, rows, x);
            const int row = w.tile * a.RU + x * 128 + r;
            const PagedRow see = paged_row(a, w.s, row);
            float m = kNoMax, l = 0.f;                           // m: the exponent that weights are relative to, LIFT below the maximum it was taken from
            bool begun = false;
            for (int i = from; i < to; ++i) {
                const int j = paged_tile_at(w.t, i) * KT;
                if (!chunk_needs(a, v, j)) continue;
                const bool masked = !chunk_whole(a, v, j);
                if (!(ok = chunk_wait(s->s_full[x], s_ph, s, a.status))) break;
                s_ph ^= 1u;
                tc::fence_after();
                uint32_t f0[32], f1[32];
                tc::ld32(t_s, f0);
                tc::ld32(t_s + 32, f1);
                tc::wait_ld();
                tc::settle32(f0);
                tc::settle32(f1);
                if (masked) {
                    const int hi = see.hi - j - h * 64, lo = see.lo - j - h * 64, first_few = a.sinks - j - h * 64;
                    mask32(f0, bits_below(hi) & (~bits_below(lo) | bits_below(first_few)));
                    mask32(f1, bits_below(hi - 32) & (~bits_below(lo - 32) | bits_below(first_few - 32)));
                }
                float top[4] = {kNoMax, kNoMax, kNoMax, kNoMax};
                top32(top, f0);
                top32(top, f1);
                // the other 64 columns are another warp's; what it reads here it has read before it hands its weights over, and the next
                // scores come behind that
                const float half_top = max_nan(max3_nan(top[0], top[1], top[2]), top[3]);
                if (!(ok = meet(half_top))) break;
                const float now = max_nan(half_top, *other_s) * scale2;
                const bool move = !(now <= m + (8.f + LIFT));    // also when there is no m yet, or a NaN
                if (__any_sync(0xffffffffu, move)) {
                    const float before = m;
                    const bool first = m == kNoMax;
                    if (move) m = now - LIFT;
                    if (begun && __any_sync(0xffffffffu, move && !first)) {
                        const float by = move && !first ? exp2_fast(before - m) : 1.f;
                        l *= by;
#pragma unroll 1
                        for (int c = 0; c < D / 32; ++c) {       // this warp's half of the columns
                            uint32_t o[16];
                            tc::ld16(t_o + c * 16, o);
                            tc::wait_ld();
                            tc::settle16(o);
#pragma unroll
                            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * by);
                            tc::st16(t_o + c * 16, o);
                        }
                    }
                }
                begun = true;
                const float ref = m == kNoMax ? 0.f : m;
                const f32x2 scale22 = pair(scale2, scale2), ref2 = pair(-ref, -ref);
                f32x2 sum[2] = {pair(0.f, 0.f), pair(0.f, 0.f)};
                auto weights = [&](const uint32_t* f, uint32_t to) {
                    uint32_t p[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const f32x2 y = fma2(pair(__uint_as_float(f[2 * e]), __uint_as_float(f[2 * e + 1])), scale22, ref2);
                        float p0, p1;
                        split(y, p0, p1);
                        p0 = exp2_fast(p0);
                        p1 = exp2_fast(p1);
                        sum[e & 1] = add2(sum[e & 1], pair(p0, p1));
                        p[e] = pack2<T>(p0, p1);
                    }
                    tc::st16(to, p);
                };
                weights(f0, t_s);
                weights(f1, t_s + 16);
                tc::wait_st();
                tc::fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&s->p_full[x]));
                float s0, s1;
                split(add2(sum[0], sum[1]), s0, s1);
                l += s0 + s1;
            }
            if (!ok) break;
            if (begun) {
                if (!(ok = chunk_wait(s->o_full[x], o_ph, s, a.status))) break;
                o_ph ^= 1u;
                tc::fence_after();
                if (!(ok = meet(l))) break;
                const float other = *other_s;
                if (!(ok = meet_again())) break;                 // before the next unit's maxima take its place
                l = h == 0 ? l + other : other + l;              // the same bits in both
            }
            const bool head = from == 0, tail = to == w.t.count;
            const bool mine = x * 128 + r < rows;
            const bool restore = begun && *(volatile int*)&s->found[unit & 3] == unit + 1;
            const bool wide = ((reinterpret_cast<uintptr_t>(a.out) | (uintptr_t)(a.ld_out * 2)) & 31) == 0;
            const size_t slot = (size_t)blockIdx.x * 2 + (head ? 1 : 0);
            const bool sees = paged_sees_some(a, see);
            const float inv = 1.f / l;
            constexpr int C = D / 2;                             // this warp's columns
            T* to_out = reinterpret_cast<T*>(a.out) + (mine ? paged_row_offset(a, w.s, w.h, row, a.ld_out) : 0) + h * C;
            float* to_part = a.part_o + slot * a.RU * D + (size_t)h * C * a.RU + (x * 128 + r) * 4;
            if (restore) {                                       // rare: column by column in tensor memory
                const PagedRow low = paged_row(a, w.s, w.tile * a.RU), high = paged_row(a, w.s, w.tile * a.RU + rows - 1);
#pragma unroll 1
                for (int e = 0; e < C; ++e) {
                    uint32_t word;
                    tc::ld1(t_o + e, word);
                    float y = __uint_as_float(word);
                    if (mine) y += paged_odd_sum<T>(a, w, low.hi, high.lo, from, to, row, h * C + e);
                    __syncwarp();
                    tc::st1(t_o + e, __float_as_uint(y));
                }
                tc::wait_st();
            }
            constexpr int S = C < 64 ? C : 64;                   // at a time
#pragma unroll 1
            for (int c0 = 0; c0 < C; c0 += S) {
                uint32_t o[S];
                if (begun) {
#pragma unroll
                    for (int c = 0; c < S / 32; ++c) tc::ld32(t_o + c0 + c * 32, o + c * 32);
                    tc::wait_ld();
#pragma unroll
                    for (int c = 0; c < S / 32; ++c) tc::settle32(o + c * 32);
                } else {
#pragma unroll
                    for (int e = 0; e < S; ++e) o[e] = 0u;
                }
                if (!mine) {
                } else if (head && tail) {
#pragma unroll
                    for (int c = 0; c < S / 16; ++c) {
                        uint32_t p[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            p[e] = sees ? pack2<T>(__uint_as_float(o[c * 16 + 2 * e]) * inv, __uint_as_float(o[c * 16 + 2 * e + 1]) * inv) : 0u;
                        store32(to_out + c0 + c * 16, p, wide);
                    }
                } else {
#pragma unroll
                    for (int c = 0; c < S / 4; ++c)
                        *reinterpret_cast<uint4*>(to_part + (size_t)(c0 / 4 + c) * a.RU * 4) = make_uint4(o[4 * c], o[4 * c + 1], o[4 * c + 2], o[4 * c + 3]);
                }
            }
            if (mine && !(head && tail) && h == 0) a.part_ml[slot * a.RU + x * 128 + r] = make_float2(m, l);
            tc::fence_before();                                  // the reads of O come before the next unit's products
            if (to > from) ++unit;
        }
        if (!ok) named_bar_arrive(1 + x, 256);
    }

    // Leaving: nothing may still be landing in this CTA's shared memory, and tensor memory goes back.
    tc::fence_before();
    __syncthreads();
    if (s->abort) {
        // after a wait that gave up copies may be in flight: a bounded time for them to land
        const long long t0 = clock64();
        while (clock64() - t0 < 20000000LL) __nanosleep(1000);
        __syncthreads();
    }
    let_next_start();
    if (warp == 17) {
        tc::fence_after();
        tc::dealloc(tmem, 512);
    }
}

// cuTensorMapEncodeTiled, looked up through the runtime (the library links no libcuda symbol).
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

static coreinfer_status encode_fn(EncodeTiledFn* out)
{
    static std::atomic<EncodeTiledFn> cached{nullptr};
    EncodeTiledFn f = cached.load(std::memory_order_acquire);
    if (!f) {
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult qres;
        CI_CUDA(cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qres));
        if (qres != cudaDriverEntryPointSuccess || !fn)
            CI_FAIL(COREINFER_ERR_CUDA, "cuTensorMapEncodeTiled is not available from this driver");
        f = (EncodeTiledFn)fn;
        cached.store(f, std::memory_order_release);
    }
    *out = f;
    return COREINFER_OK;
}

// A pool as [pages][heads][slots][head_dim], read in boxes of `box` slots x 64 values with the 128-byte swizzle.
static coreinfer_status pool_map(CUtensorMap* map, const Paged& c, const void* pool, bool f16, int box)
{
    EncodeTiledFn enc;
    coreinfer_status s = encode_fn(&enc);
    if (s != COREINFER_OK) return s;
    const long long page = 1LL << c.page_shift;
    // the stride of an axis of one entry is never used, but has to be one that the map takes
    const long long head_stride = c.H > 1 ? c.head_stride : c.token_stride, page_stride = c.n_pages > 1 ? c.page_stride : c.token_stride;
    const cuuint64_t dims[4] = {(cuuint64_t)c.D, (cuuint64_t)page, (cuuint64_t)c.H, (cuuint64_t)c.n_pages};
    const cuuint64_t strides[3] = {(cuuint64_t)c.token_stride * 2, (cuuint64_t)head_stride * 2, (cuuint64_t)page_stride * 2};
    const cuuint32_t boxes[4] = {64, (cuuint32_t)box, 1, 1};
    const cuuint32_t estr[4] = {1, 1, 1, 1};
    const CUresult r = enc(map, f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(pool), dims, strides, boxes, estr,
                           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) CI_FAIL(COREINFER_ERR_CUDA, "cuTensorMapEncodeTiled failed with code %d", (int)r);
    return COREINFER_OK;
}

// Queries as [tokens][heads][head_dim], read in boxes of a key head's share of 128 / share tokens.
static coreinfer_status query_map(CUtensorMap* map, const PagedAttnArgs& a, bool f16)
{
    EncodeTiledFn enc;
    coreinfer_status s = encode_fn(&enc);
    if (s != COREINFER_OK) return s;
    const cuuint64_t dims[3] = {(cuuint64_t)a.c.D, (cuuint64_t)a.c.H * a.share, (cuuint64_t)a.c.tokens};
    const cuuint64_t strides[2] = {(cuuint64_t)a.c.D * 2, (cuuint64_t)a.ld_q * 2};
    const cuuint32_t boxes[3] = {64, (cuuint32_t)a.share, (cuuint32_t)(128 / a.share)};
    const cuuint32_t estr[3] = {1, 1, 1};
    const CUresult r = enc(map, f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<uint8_t*>(a.q), dims, strides, boxes, estr,
                           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) CI_FAIL(COREINFER_ERR_CUDA, "cuTensorMapEncodeTiled failed with code %d", (int)r);
    return COREINFER_OK;
}

template <typename T, int D>
static coreinfer_status launch_chunk(ChunkArgs& g, const DeviceInfo& di, cudaStream_t st)
{
    CUtensorMap mk, mv, mq;
    const bool f16 = std::is_same<T, __half>::value;
    const int page = 1 << g.a.c.page_shift;
    g.box = page < kChunkKT ? page : kChunkKT;
    coreinfer_status s = pool_map(&mk, g.a.c, g.a.c.pool[0], f16, g.box);
    if (s != COREINFER_OK || (s = pool_map(&mv, g.a.c, g.a.c.pool[1], f16, g.box)) != COREINFER_OK) return s;
    // a box is whole tokens: shares that divide 128, and queries as they are
    g.map_q = g.sign > 0 && g.a.share <= 128 && (g.a.share & (g.a.share - 1)) == 0 && g.a.ld_q < 1LL << 38;
    if (g.map_q) {
        if ((s = query_map(&mq, g.a, f16)) != COREINFER_OK) return s;
    } else mq = mk;
    constexpr size_t TILE = D / 64 * 128 * 128;
    const size_t fixed = kChunkPipes<D> * TILE + sizeof(ChunkBars) + paged_list_bytes(g.a.c.B);
    size_t stages = (smem_room(di, 0) - fixed) / TILE;
    if (stages > kChunkMaxStages) stages = kChunkMaxStages;
    g.k_stages = (int)stages / 2;
    g.v_stages = (int)stages - g.k_stages;
    const size_t smem = fixed + stages * TILE;
    if ((s = allow_smem<paged_chunk_kernel<T, D>>(di, 0)) != COREINFER_OK) return s;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(g.a.n_ctas);
    cfg.blockDim = dim3(kChunkThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    CI_CUDA(cudaLaunchKernelEx(&cfg, paged_chunk_kernel<T, D>, mk, mv, mq, (const ChunkArgs)g));
    return COREINFER_OK;
}

template <typename T>
static coreinfer_status chunk_dim(ChunkArgs& g, const DeviceInfo& di, cudaStream_t st)
{
    if (g.a.c.D == 64) return launch_chunk<T, 64>(g, di, st);
    return g.a.c.D == 128 ? launch_chunk<T, 128>(g, di, st) : launch_chunk<T, 256>(g, di, st);
}

coreinfer_status paged_chunk(PagedAttnArgs& a, bool f16, const DeviceInfo& di, cudaStream_t st)
{
    ChunkArgs g;
    g.a = a;
    g.sign = a.scale2 > 0.f ? 1 : (a.scale2 < 0.f ? -1 : 0);
    return f16 ? chunk_dim<__half>(g, di, st) : chunk_dim<__nv_bfloat16>(g, di, st);
}

}  // namespace coreinfer
