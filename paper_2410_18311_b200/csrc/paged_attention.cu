// Attention of new tokens over a paged cache: the entry points, the form for many fp32 rows, and the kernel that joins the pieces of
// units that are cut.
//
// Four forms over one list of work: fp32 caches with up to four rows (tokens * query heads per key head) a sequence
// (paged_attention_rows.cu) and with more (here, 16 or 64 rows x 64 positions on the FMA pipe); 16-bit caches with few rows (paged_attention_few.cu) and with
// many (paged_attention_tc.cu).  The host chooses by what it knows, the average of rows: right where sequences are alike, and dear where one long piece
// comes with many decoding sequences (63 x 2000 positions and 500 tokens over 16000, 32 heads of 128 bf16: an average of 9 rows, 1700 us; as two calls
// 476).  Such a batch is better brought as two calls.
//
// Mathematics.  One pass over the positions that a unit's rows see, with a running maximum m (base 2), sum l and output o
// per row:  m' = max(m, s),  l' = 2^(m - m') l + sum 2^(s - m'),  o' = 2^(m - m') o + sum 2^(s - m') v;  out = o / l.  Pieces of
// a unit are joined by the same rule.  A row whose seen logits are all -infinity comes out NaN, as the formula says (0 / 0);
// one that sees nothing comes out 0.
#include "paged_attention.cuh"

namespace coreinfer {

// Many fp32 rows.  Blocks of 256 threads as 16 x 16; a unit is 16 RT rows over tiles of 64 positions.  A thread has RT x 4 logits (rows ty RT + r,
// positions tx + 16 e), then RT x D / 16 outputs of the same rows, so that a row's maximum and sum stay in the registers of half a warp and its
// weights are written and read by one warp.  All operands come from shared memory in 16-byte reads: at RT = 4 twelve
// wavefronts for 64 FMA instructions.  Keys, values and queries are brought by cp.async; at head_dim 128 and 256
// the weights take the keys' place, so that two blocks fit an SM at 128.  Measured: 2 x 500 tokens x 12 heads of 64 over up to 1000 positions 77 us,
// 1000 tokens x 16 heads over 2000 positions 225 us at head_dim 64, 403 at 128, 838 at 256 (as one chain of sums a unit 224, 399, 826; at 128: FMA pipe
// 54 %, shared memory's wavefronts 69 %, issue 70 %); 16 x 8 heads x 8 rows x 7600 of 128 481 us.
constexpr int kManyThreads = 256;
constexpr int kManyTile = 64;
constexpr int kManyKeep = 16;                                                        // tiles whose sums are one chain of additions
template <int D> constexpr int kManyCtas = D == 256 ? 1 : 2;                         // per SM
template <int D> constexpr bool kManyApart = D == 64;                                // weights have a place of their own
template <int D, int RT> constexpr int kManyFloats = 16 * RT * (D + 4) + kManyTile * (D + 4) + kManyTile * D + (kManyApart<D> ? 16 * RT * (kManyTile + 4) : 0);

__device__ __forceinline__ void many_copy(float* to, const float* from, bool read)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(to)), "l"(from), "r"(read ? 16 : 0) : "memory");
}

template <int D, int RT>
__global__ void __launch_bounds__(kManyThreads, kManyCtas<D>) paged_many_kernel(const __grid_constant__ PagedAttnArgs a)
{
    constexpr int RU = 16 * RT, KT = kManyTile, DP = D + 4, PP = KT + 4, NV = D / 64;
    static_assert(kManyApart<D> || RU * PP <= KT * DP, "weights in the keys' place");
    extern __shared__ __align__(16) float smem[];
    float* qs = smem;                                // [RU][DP]
    float* ks = qs + RU * DP;                        // [KT][DP]
    float* vs = ks + KT * DP;                        // [KT][D]
    float* ps = kManyApart<D> ? vs + KT * D : ks;    // [RU][PP]
    int* at = reinterpret_cast<int*>(smem + kManyFloats<D, RT>);
    const int tid = threadIdx.x, lane = tid & 31, tx = tid & 15, ty = tid >> 4;
    const float* keys = reinterpret_cast<const float*>(a.c.pool[0]);
    const float* values = reinterpret_cast<const float*>(a.c.pool[1]);
    wait_for_stream();
    const int total = paged_plan(a, at);
    if (tid == 0) paged_first_words(a);
    PagedWalk w;
    for (w.begin(a, at, total, blockIdx.x); w.more(); w.next(a, at)) {
        const int from = w.from(a), to = w.to(a);
        if (w.t.count > 0 && from >= to) continue;
        const int rows = paged_unit_rows(a, w), r0 = w.tile * RU;
        const PagedRow low = paged_row(a, w.s, r0), high = paged_row(a, w.s, r0 + rows - 1);
        // a tile's keys, then its values; what no row sees is 0
        auto fetch = [&](int i) {
            const int j0 = paged_tile_at(w.t, i) * KT;
            const int pages = lane < KT / 16 ? paged_page(a.c, w.b, j0 + lane * 16) : -1;
#pragma unroll
            for (int kv = 0; kv < 2; ++kv) {
#pragma unroll 4
                for (int x = tid; x < KT * (D / 4); x += kManyThreads) {
                    const int j = x / (D / 4), d = x % (D / 4) * 4;
                    const int page = __shfl_sync(0xffffffffu, pages, j / 16);
                    const bool read = page >= 0 && j0 + j < high.hi && (j0 + j >= low.lo || j0 + j < a.sinks);
                    const float* pool = kv ? values : keys;
                    many_copy(kv ? vs + j * D + d : ks + j * DP + d, read ? pool + paged_offset(a.c, page, w.h, j0 + j) + d : pool, read);
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
            }
        };
        __syncthreads();                             // the unit before is done with shared memory
        for (int x = tid; x < RU * (D / 4); x += kManyThreads) {
            const int r = x / (D / 4), d = x % (D / 4) * 4;
            const float* q = reinterpret_cast<const float*>(a.q);
            many_copy(qs + r * DP + d, r < rows ? q + paged_row_offset(a, w.s, w.h, r0 + r, a.ld_q) + d : q, r < rows);
        }
        if (from < to) fetch(from);
        const bool head = from == 0, tail = to == w.t.count;
        const size_t slot = (size_t)blockIdx.x * 2 + (head ? 1 : 0);
        PagedRow see[RT];
        float m[RT], l[RT], o[RT][NV][4];
        // Sums of kManyKeep tiles are added to those before, which wait in the unit's slot of the workspace (the first time there is nothing
        // yet): one chain over all positions would lose bits (8 rows x 10000 positions of 64, 16 sequences x 12 heads: error against
        // 64 bits 1.5e-6, so 0.9e-6; values that are all alike x 40000 of 256: off by 1.4e-4, so 1e-5).
        auto add_kept = [&](bool any) {
#pragma unroll
            for (int r = 0; r < RT; ++r) {
#pragma unroll
                for (int d = 1; d < 16; d <<= 1) l[r] += __shfl_xor_sync(0xffffffffu, l[r], d);
                if (!any) continue;
                const int row = ty * RT + r;
                const float2 kept = a.part_ml[slot * RU + row];
                const float by = kept.x == -INFINITY ? 0.f : exp2f(kept.x - m[r]);
                l[r] = fmaf(kept.y, by, l[r]);
#pragma unroll
                for (int n = 0; n < NV; ++n) {
                    const float4 x = *reinterpret_cast<const float4*>(a.part_o + slot * RU * D + ((tx * 4 + 64 * n) * RU + row * 4));
                    o[r][n][0] = fmaf(x.x, by, o[r][n][0]);
                    o[r][n][1] = fmaf(x.y, by, o[r][n][1]);
                    o[r][n][2] = fmaf(x.z, by, o[r][n][2]);
                    o[r][n][3] = fmaf(x.w, by, o[r][n][3]);
                }
            }
            __syncwarp();                            // a row's exponent and sum have been read by all that share it
        };
        auto keep = [&](int r) {
            const int row = ty * RT + r;
#pragma unroll
            for (int n = 0; n < NV; ++n)
                *reinterpret_cast<float4*>(a.part_o + slot * RU * D + ((tx * 4 + 64 * n) * RU + row * 4)) = make_float4(o[r][n][0], o[r][n][1], o[r][n][2], o[r][n][3]);
            if (tx == 0) a.part_ml[slot * RU + row] = make_float2(m[r], l[r]);
        };
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const int row = ty * RT + r;
            see[r] = paged_row(a, w.s, r0 + (row < rows ? row : rows - 1));
            m[r] = -INFINITY;
            l[r] = 0.f;
#pragma unroll
            for (int n = 0; n < NV; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[r][n][e] = 0.f;
        }
        for (int i = from; i < to; ++i) {
            const int j0 = paged_tile_at(w.t, i) * KT;
            const bool whole = j0 + KT <= low.hi && (j0 >= high.lo || j0 + KT <= a.sinks);
            asm volatile("cp.async.wait_group 1;" ::: "memory");
            __syncthreads();
            float s[RT][4];
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[r][e] = 0.f;
#pragma unroll 4
            for (int d = 0; d < D; d += 4) {
                float4 k[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) k[e] = *reinterpret_cast<const float4*>(ks + (tx + 16 * e) * DP + d);
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    const float4 q = *reinterpret_cast<const float4*>(qs + (ty * RT + r) * DP + d);
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[r][e] = fmaf(q.x, k[e].x, fmaf(q.y, k[e].y, fmaf(q.z, k[e].z, fmaf(q.w, k[e].w, s[r][e]))));
                }
            }
            if (!kManyApart<D>) __syncthreads();
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                float top = m[r];
                unsigned seen = 0xfu;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    s[r][e] *= a.scale2;
                    if (!whole && !paged_sees(a, see[r], j0 + tx + 16 * e)) {
                        seen &= ~(1u << e);
                        s[r][e] = -INFINITY;
                    }
                    top = fmaxf(top, s[r][e]);
                }
#pragma unroll
                for (int d = 1; d < 16; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                const float ref = top == -INFINITY ? 0.f : top;
                const float by = exp2f(m[r] - ref);
                m[r] = top;
                l[r] *= by;
#pragma unroll
                for (int n = 0; n < NV; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[r][n][e] *= by;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float p = exp2f(s[r][e] - ref);
                    l[r] += p;
                    // below 0: the row does not see the position, and no value there may reach it, as 0 times infinity would
                    ps[(ty * RT + r) * PP + tx + 16 * e] = seen >> e & 1u ? p : -1.f;
                }
            }
            asm volatile("cp.async.wait_group 0;" ::: "memory");
            __syncthreads();
            auto add = [&](auto all) {
#pragma unroll 2
                for (int j = 0; j < KT; j += 4) {
                    float p[RT][4];
#pragma unroll
                    for (int r = 0; r < RT; ++r) *reinterpret_cast<float4*>(p[r]) = *reinterpret_cast<const float4*>(ps + (ty * RT + r) * PP + j);
#pragma unroll
                    for (int x = 0; x < 4; ++x)
#pragma unroll
                        for (int n = 0; n < NV; ++n) {
                            const float4 v = *reinterpret_cast<const float4*>(vs + (j + x) * D + tx * 4 + 64 * n);
#pragma unroll
                            for (int r = 0; r < RT; ++r) {
                                if (!decltype(all)::value && p[r][x] < 0.f) continue;
                                o[r][n][0] = fmaf(p[r][x], v.x, o[r][n][0]);
                                o[r][n][1] = fmaf(p[r][x], v.y, o[r][n][1]);
                                o[r][n][2] = fmaf(p[r][x], v.z, o[r][n][2]);
                                o[r][n][3] = fmaf(p[r][x], v.w, o[r][n][3]);
                            }
                        }
                }
            };
            if (whole) add(std::true_type());
            else add(std::false_type());
            __syncthreads();
            if (i + 1 < to) fetch(i + 1);
            if ((i - from) % kManyKeep == kManyKeep - 1 && i + 1 < to) {
                add_kept(i - from >= kManyKeep);
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    keep(r);
                    l[r] = 0.f;
#pragma unroll
                    for (int n = 0; n < NV; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[r][n][e] = 0.f;
                }
                __syncwarp();
            }
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        add_kept(to - from > kManyKeep);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            const int row = ty * RT + r;
            if (row >= rows) continue;
            if (head && tail) {
                float* to_row = reinterpret_cast<float*>(a.out) + paged_row_offset(a, w.s, w.h, r0 + row, a.ld_out) + tx * 4;
                const bool any = paged_sees_some(a, see[r]);
#pragma unroll
                for (int n = 0; n < NV; ++n)
                    *reinterpret_cast<float4*>(to_row + 64 * n) = any ? make_float4(o[r][n][0] / l[r], o[r][n][1] / l[r], o[r][n][2] / l[r], o[r][n][3] / l[r])
                                                                      : make_float4(0.f, 0.f, 0.f, 0.f);
            } else keep(r);
        }
        if (head && !tail && tid == 0) {
            PagedPiece p;
            p.b = w.b;
            p.h = w.h;
            p.tile = w.tile;
            p.last = w.last(a, at);
            a.pieces[blockIdx.x] = p;
        }
    }
    let_next_start();
}

// What a launch of its own costs: 3 to 5 us of a call, mostly under the end of the kernel before; a join by the CTA that comes last would need
// counters that somebody has set to 0.
//
// Joins the pieces of a unit that is cut, AHEAD of them on the way at once: eight where units are small (a unit of few rows is often cut into 20
// pieces: 16 x 4 rows x 130000 positions 153.5 -> 151.8 us against four), four in the form for chunks (eight take 70 registers, and its 200 to 600
// blocks no longer fit side by side: 500 tokens x 40 heads over 16000 157.0 and 161.0 us).  Block (x, y) the rows y of the unit whose first tile CTA x has.  The first piece is in
// that CTA's second slot, the others in the first slots of the CTAs behind it.
constexpr int kJoinThreads = 256;
template <int D> constexpr int kJoinRows = kJoinThreads * 4 / D;         // eight rows of 32 quarters at head_dim 128
template <typename T, int D, int AHEAD>
__global__ void __launch_bounds__(kJoinThreads) paged_join_kernel(const __grid_constant__ PagedAttnArgs a)
{
    constexpr int ROWS = kJoinRows<D>;
    wait_for_stream();
    const PagedPiece p = a.pieces[blockIdx.x];
    // the second line: what another call has left there, where two overlap in one workspace against the rules
    if (p.last < 0) return;
    if (p.last >= a.n_ctas || (unsigned)p.b >= (unsigned)a.c.B || (unsigned)p.h >= (unsigned)a.c.H || p.tile >> (30 - a.ru_shift)) return;
    const PagedSeq s = paged_seq(a.c, p.b);
    const int row = blockIdx.y * ROWS + threadIdx.x % ROWS, c = threadIdx.x / ROWS * 4;
    const int global_row = p.tile * a.RU + row;
    if (row >= a.RU || global_row >= paged_rows(a, s)) return;
    const int first = blockIdx.x;
    auto slot = [&](int i) { return (size_t)i * 2 + (i == first ? 1 : 0); };
    // eight pieces' loads at once; the maximum moves from one eight to the next
    float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int i0 = first; i0 <= p.last; i0 += AHEAD) {
        float2 ml[AHEAD];
        float4 x[AHEAD];
        float top = m;
#pragma unroll
        for (int e = 0; e < AHEAD; ++e) {
            ml[e] = make_float2(-INFINITY, 0.f);
            if (i0 + e > p.last) continue;
            ml[e] = a.part_ml[slot(i0 + e) * a.RU + row];
            x[e] = *reinterpret_cast<const float4*>(a.part_o + slot(i0 + e) * a.RU * D + (c * a.RU + row * 4));
        }
#pragma unroll
        for (int e = 0; e < AHEAD; ++e) top = fmaxf(top, ml[e].x);
        const float ref = top == -INFINITY ? 0.f : top;
        if (m != -INFINITY) {
            const float by = exp2f(m - ref);
            l *= by;
#pragma unroll
            for (int d = 0; d < 4; ++d) o[d] *= by;
        }
        m = top;
#pragma unroll
        for (int e = 0; e < AHEAD; ++e) {
            const float f = exp2f(ml[e].x - ref);
            l = fmaf(ml[e].y, f, l);
            // a piece in which the row sees nothing, or nothing but weights of 0, has nothing to add
            if (ml[e].x == -INFINITY) continue;
            o[0] = fmaf(x[e].x, f, o[0]);
            o[1] = fmaf(x[e].y, f, o[1]);
            o[2] = fmaf(x[e].z, f, o[2]);
            o[3] = fmaf(x[e].w, f, o[3]);
        }
    }
    const bool sees = paged_sees_some(a, paged_row(a, s, global_row));
    T* to = reinterpret_cast<T*>(a.out) + paged_row_offset(a, s, p.h, global_row, a.ld_out) + c;
    T y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = from_f32<T>(sees ? o[e] / l : 0.f);
    if constexpr (sizeof(T) == 4) *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(y);
    else *reinterpret_cast<uint2*>(to) = *reinterpret_cast<const uint2*>(y);
}

template <int D, int RT>
static coreinfer_status launch_many(const PagedAttnArgs& a, const DeviceInfo& di, cudaStream_t st)
{
    const size_t smem = (size_t)kManyFloats<D, RT> * 4 + paged_list_bytes(a.c.B);
    const coreinfer_status s = allow_smem<paged_many_kernel<D, RT>>(di, 0);
    if (s != COREINFER_OK) return s;
    CI_CUDA(launch_overlapped(paged_many_kernel<D, RT>, dim3(a.n_ctas), dim3(kManyThreads), smem, st, a));
    return COREINFER_OK;
}
template <int D>
static coreinfer_status many_rows(const PagedAttnArgs& a, const DeviceInfo& di, cudaStream_t st)
{
    return a.RU == 16 ? launch_many<D, 1>(a, di, st) : launch_many<D, 4>(a, di, st);
}
template <typename T, int D>
static coreinfer_status launch_join(const PagedAttnArgs& a, cudaStream_t st)
{
    constexpr int ROWS = kJoinRows<D>;
    const dim3 grid(a.n_ctas, (a.RU + ROWS - 1) / ROWS);
    if (a.RU <= 16) CI_CUDA(launch_overlapped(paged_join_kernel<T, D, 8>, grid, dim3(kJoinThreads), 0, st, a));
    else CI_CUDA(launch_overlapped(paged_join_kernel<T, D, 4>, grid, dim3(kJoinThreads), 0, st, a));
    return COREINFER_OK;
}
template <typename T>
static coreinfer_status pick_join(const PagedAttnArgs& a, cudaStream_t st)
{
    if (a.c.D == 64) return launch_join<T, 64>(a, st);
    return a.c.D == 128 ? launch_join<T, 128>(a, st) : launch_join<T, 256>(a, st);
}

static coreinfer_status pick_many(const PagedAttnArgs& a, const DeviceInfo& di, cudaStream_t st)
{
    if (a.c.D == 64) return many_rows<64>(a, di, st);
    return a.c.D == 128 ? many_rows<128>(a, di, st) : many_rows<256>(a, di, st);
}

static size_t round16(size_t n) { return (n + 15) / 16 * 16; }

// Which form a call takes, by what the host knows (the lengths of the batch's pieces are on the device).
enum PagedFormKind { kFormMany, kFormRows, kFormFew, kFormChunk };
struct PagedForm {
    PagedFormKind kind;
    int RU, KT, ctas;           // rows of a unit, positions of a tile, CTAs
    int cost;                   // what starting and ending a unit takes, in tiles
};
static PagedForm paged_form(coreinfer_dtype dtype, int D, int B, int share, int tokens)
{
    const long long rows = ((long long)tokens * share + B - 1) / B;
    if (dtype == COREINFER_F32 && rows <= kPagedRowsMost) return {kFormRows, rows == 1 ? 1 : kPagedRowsMost, paged_rows_tile(D), rows == 1 ? 2 * 148 : 148, 2};
    // 16 or 64 rows a unit: 6 rows over 3000 positions 60 and 87 us at head_dim 128, 130 and 177 at 256; 24 rows 90.0 and 89.3, 199 and 178 (48 and 54 at
    // 64).
    if (dtype == COREINFER_F32) return {kFormMany, rows <= 16 ? 16 : 64, kManyTile, 148 * (D == 256 ? 1 : 2), 1};
    // By the rows of a sequence and key head on the average.  In the form for few and in that for chunks: 15 rows of 128 x 4096
    // of 9000 positions 32.7 and 41.0 us, 16 of 128 x 100000 71 and 88, 12 of 64 x 4000 26.7 and 31.5, 16 of 256 41.0 and 47.2.  One row x 4000 of 128 75 and 101 us.
    // A unit's start and end take about what two tiles do; counted as three, fewer units are cut (prompt of 8192 tokens 536 -> 529 us, 4 sequences of 64
    // rows over 6000 positions 33.0 -> 31.8, 500 tokens over 16000 158.3 -> 159.0; head_dim 256, whose tiles take longer, 160.4 -> 162.9).
    if (rows > 16) return {kFormChunk, paged_chunk_rows(D), kPagedChunkTile, kPagedChunkCtas, D == 256 ? 2 : 3};
    const PagedFewShape few = paged_few_shape(D, (int)rows);
    return {kFormFew, few.RU, few.KT, few.ctas, 2};
}
// A status word (16 bytes), the pieces, their exponents and sums, their outputs (from a multiple of 32 bytes on).
static size_t paged_workspace(const PagedForm& f, int D)
{
    return 16 + round16(f.ctas * sizeof(PagedPiece)) + round16((size_t)f.ctas * 2 * f.RU * sizeof(float2)) + 16 + (size_t)f.ctas * 2 * f.RU * D * sizeof(float);
}

}  // namespace coreinfer

using namespace coreinfer;

extern "C" {

size_t coreinfer_paged_attention_workspace_bytes(const coreinfer_paged_cache* cache, int32_t q_heads, int32_t tokens)
{
    Paged c;
    if (paged_take(cache, &c) != COREINFER_OK || q_heads < 1 || q_heads % c.H != 0 || tokens < 1) return 0;
    // fewer tokens may take the other form: the larger of the two
    const size_t a = paged_workspace(paged_form(cache->dtype, c.D, c.B, q_heads / c.H, tokens), c.D);
    const size_t b = paged_workspace(paged_form(cache->dtype, c.D, c.B, q_heads / c.H, 1), c.D);
    return a > b ? a : b;
}

coreinfer_status coreinfer_paged_attention(const coreinfer_paged_cache* cache, const int32_t* start, int32_t tokens,
                                           const void* q, int64_t ld_q, int32_t q_heads, float scale,
                                           int32_t window, int32_t sinks, void* out, int64_t ld_out,
                                           void* workspace, size_t workspace_bytes, void* cuda_stream)
{
    PagedAttnArgs a = {};
    coreinfer_status s = paged_take(cache, &a.c);
    if (s != COREINFER_OK) return s;
    const coreinfer_dtype dtype = cache->dtype;
    if (q_heads < 1 || q_heads % a.c.H != 0)
        CI_FAIL(COREINFER_ERR_INVALID_ARG, "q_heads %d is not a multiple of kv_heads %d", q_heads, a.c.H);
    if (q_heads > 4096) CI_FAIL(COREINFER_ERR_UNSUPPORTED, "q_heads %d: at most 4096", q_heads);
    if (tokens < 1) CI_FAIL(COREINFER_ERR_INVALID_ARG, "tokens must be >= 1");
    if ((long long)tokens * q_heads > 1LL << 29) CI_FAIL(COREINFER_ERR_UNSUPPORTED, "tokens %d: too many for one call", tokens);
    if (!start || !aligned_to(start, 4)) CI_FAIL(COREINFER_ERR_INVALID_ARG, "start NULL or misaligned");
    if (!rows_fit(q, ld_q, q_heads, a.c.D, dtype) || !rows_fit(out, ld_out, q_heads, a.c.D, dtype))
        CI_FAIL(COREINFER_ERR_INVALID_ARG, "q / out NULL, not 16-byte aligned, or strides too small or not multiples of 16 bytes");
    if (window < 0 || sinks < 0) CI_FAIL(COREINFER_ERR_INVALID_ARG, "window and sinks must be >= 0");
    if (window > 1 << 30 || sinks > 1 << 30) CI_FAIL(COREINFER_ERR_UNSUPPORTED, "window and sinks: at most 2^30");
    if (!isfinite(scale * kLog2e)) CI_FAIL(COREINFER_ERR_INVALID_ARG, "scale, and scale * log2(e), must be finite");
    if (!workspace || !aligned16(workspace)) CI_FAIL(COREINFER_ERR_WORKSPACE, "workspace is NULL or misaligned");
    paged_set_share(a, q_heads / a.c.H);
    const PagedForm f = paged_form(dtype, a.c.D, a.c.B, a.share, tokens);
    // the list of work counts in 32 bits: row tiles of all sequences, each with all tiles of the table at most
    if ((double)a.c.H * ((double)tokens * a.share / f.RU + a.c.B) * ((double)a.c.cap / f.KT + 1 + f.cost) >= 2147483648.0)
        CI_FAIL(COREINFER_ERR_UNSUPPORTED, "%d tokens x %d heads over a table of %d positions: too much for one call", tokens, q_heads, a.c.cap);
    const size_t need = paged_workspace(f, a.c.D);
    if (workspace_bytes < need) CI_FAIL(COREINFER_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", workspace_bytes, need);
    DeviceInfo di;
    if ((s = device_info(&di)) != COREINFER_OK) return s;
    a.c.start = start;
    a.c.tokens = tokens;
    a.q = (const uint8_t*)q;
    a.out = (uint8_t*)out;
    a.ld_q = ld_q;
    a.ld_out = ld_out;
    a.window = window;
    a.sinks = window ? sinks : 0;
    a.scale2 = scale * kLog2e;
    a.RU = f.RU;
    a.KT = f.KT;
    for (a.ru_shift = 0; 1 << a.ru_shift < a.RU;) ++a.ru_shift;
    for (a.kt_shift = 0; 1 << a.kt_shift < a.KT;) ++a.kt_shift;
    a.cost = f.cost;
    a.n_ctas = f.ctas;
    a.status = (unsigned*)workspace;
    uint8_t* ws = (uint8_t*)workspace + 16;
    a.pieces = (PagedPiece*)ws;
    ws += round16(f.ctas * sizeof(PagedPiece));
    a.part_ml = (float2*)ws;
    ws += round16((size_t)f.ctas * 2 * f.RU * sizeof(float2));
    a.part_o = (float*)(((uintptr_t)ws + 31) & ~(uintptr_t)31);
    cudaStream_t st = (cudaStream_t)cuda_stream;
    if (f.kind == kFormChunk) s = paged_chunk(a, dtype == COREINFER_F16, di, st);
    else if (f.kind == kFormRows) s = paged_rows_f32(a, di, st);
    else s = f.kind == kFormFew ? paged_few(a, dtype == COREINFER_F16, di, st) : pick_many(a, di, st);
    if (s != COREINFER_OK) return s;
    if (dtype == COREINFER_F32) return pick_join<float>(a, st);
    return dtype == COREINFER_BF16 ? pick_join<__nv_bfloat16>(a, st) : pick_join<__half>(a, st);
}

}  // extern "C"
