// Attention of one to four query rows over a paged fp32 cache, split over its positions.
//
// What bounds it: the bytes of the slots that are seen, each read once: at four bytes a value a product and a sum per value and row leave the
// FMA pipe at a tenth for one row, so no matrix instruction (which would need fp32 in three parts) is worth its layout.  A slot is
// head_dim / 4 lanes of 16 bytes straight into registers: a logit is a lane's four products and a sum over the lanes, an output a lane's own.
//
// Persistent CTAs of 8 warps over the common list.  A tile is 8 pieces of 8 loads a lane (16, 8 or 4 slots), one per warp; each warp keeps its
// own maximum, sum and output, asks for the next piece's keys as soon as it has used the last ones and for its values after
// that, and no warp waits for another before the end of a unit.
//
// Measured from a graph, three sets of inputs: 8 x 12 heads x up to 4001 positions of 64 41 us (3800 GB/s), 16 x 8 heads x up to 7600 of 128 135 us, four
// rows of them 404 us (as far from the bytes as one CTA an SM and four sums over the lanes a slot leave it), 12 heads x 77 7 us (launch,
// list, page, keys, join: one latency after the other).  One row spills 120 to 152 bytes a thread at the 128 registers that two CTAs an SM have.
#include "paged_attention.cuh"

namespace coreinfer {

constexpr int kRowsWarps = 8;
constexpr int kRowsThreads = 32 * kRowsWarps;
constexpr int kRowsKeep = 32;                         // tiles whose sums are one chain of additions: 256 of a lane at most

template <int D, int R>
__global__ void __launch_bounds__(kRowsThreads, R == 1 ? 2 : 1) paged_rows_kernel(const __grid_constant__ PagedAttnArgs a)
{
    constexpr int LPK = D / 4 < 32 ? D / 4 : 32;     // lanes of a slot
    constexpr int KPL = 32 / LPK;                    // slots of a load
    constexpr int VPL = D / 4 / LPK;                 // loads of a slot
    constexpr int NB = 8 * KPL / VPL;                // slots of a piece
    constexpr int NL = NB / KPL;                     // slots of a piece that a lane has a part of
    constexpr int KT = NB * kRowsWarps;
    extern __shared__ __align__(16) float smem[];
    float* outs = smem;                              // [warps][R][D]
    float2* stats = reinterpret_cast<float2*>(outs + kRowsWarps * R * D);            // [warps][R]
    int* at = reinterpret_cast<int*>(stats + kRowsWarps * R);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, d0 = lane % LPK * 4;
    wait_for_stream();
    const int total = paged_plan(a, at);
    if (tid == 0) paged_first_words(a);
    PagedWalk w;
    for (w.begin(a, at, total, blockIdx.x); w.more(); w.next(a, at)) {
        const int from = w.from(a), to = w.to(a);
        if (w.t.count > 0 && from >= to) continue;
        const int rows = paged_unit_rows(a, w), r0 = w.tile * R;
        const PagedRow low = paged_row(a, w.s, r0), high = paged_row(a, w.s, r0 + rows - 1);
        int pages = -1;                              // of the next 32 tiles, a lane each
        auto position = [&](int i) { return paged_tile_at(w.t, i) * KT + warp * NB; };
        // slots x = 0 .. NL - 1 of a lane: position + x * KPL + lane / LPK; what no row sees is 0
        auto fetch = [&](int kv, int i, float4 (&to_regs)[NL][VPL]) {
            const int j0 = position(i), page = __shfl_sync(0xffffffffu, pages, (i - from) & 31);
            const float* src = reinterpret_cast<const float*>(a.c.pool[kv]) + paged_offset(a.c, page < 0 ? 0 : page, w.h, j0) + d0;
#pragma unroll
            for (int x = 0; x < NL; ++x) {
                const int k = x * KPL + lane / LPK, j = j0 + k;
                const bool read = page >= 0 && j < high.hi && (j >= low.lo || j < a.sinks);
#pragma unroll
                for (int y = 0; y < VPL; ++y)
                    to_regs[x][y] = read ? *reinterpret_cast<const float4*>(src + k * a.c.token_stride + y * 128) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
        };
        auto fetch_pages = [&](int i) {
            if (((i - from) & 31) == 0) pages = i + lane < to ? paged_page(a.c, w.b, position(i + lane)) : -1;
        };
        float4 k[NL][VPL], v[NL][VPL];
        if (from < to) {
            fetch_pages(from);
            fetch(0, from, k);
            fetch(1, from, v);
        }
        float4 q[R][VPL], o[R][VPL];
        PagedRow see[R];
        float m[R], l[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float* src = reinterpret_cast<const float*>(a.q) + (r < rows ? paged_row_offset(a, w.s, w.h, r0 + r, a.ld_q) : 0) + d0;
#pragma unroll
            for (int y = 0; y < VPL; ++y) {
                q[r][y] = r < rows ? *reinterpret_cast<const float4*>(src + y * 128) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
            see[r] = paged_row(a, w.s, r0 + (r < rows ? r : rows - 1));
            m[r] = -INFINITY;
        }
        // The sums of kRowsKeep tiles are added to those before, which wait where the unit's results go: one chain over thousands of
        // positions would lose bits (values that are all alike x 40000 positions: off by 4e-5, so 3e-6; 16 x 8 heads x 7600 of 128: error against
        // 64 bits 3.6e-7, so 3.2e-7).
        for (int i0 = from;; i0 += kRowsKeep) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            l[r] = 0.f;
#pragma unroll
            for (int y = 0; y < VPL; ++y) o[r][y] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
        const int end = i0 + kRowsKeep < to ? i0 + kRowsKeep : to;
        for (int i = i0; i < end; ++i) {
            const int j0 = position(i);
            float s[R][NL];
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int x = 0; x < NL; ++x) {
                    float t = 0.f;
#pragma unroll
                    for (int y = 0; y < VPL; ++y)
                        t = fmaf(q[r][y].x, k[x][y].x, fmaf(q[r][y].y, k[x][y].y, fmaf(q[r][y].z, k[x][y].z, fmaf(q[r][y].w, k[x][y].w, t))));
                    s[r][x] = t;
                }
            if (i + 1 < to) {
                // a lane's pages last for 32 tiles: the values of this one are here already
                fetch_pages(i + 1);
                fetch(0, i + 1, k);
            }
            const bool whole = j0 + NB <= low.hi && (j0 >= high.lo || j0 + NB <= a.sinks);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float top = -INFINITY;
#pragma unroll
                for (int x = 0; x < NL; ++x) {
#pragma unroll
                    for (int d = 1; d < LPK; d <<= 1) s[r][x] += __shfl_xor_sync(0xffffffffu, s[r][x], d);
                    s[r][x] *= a.scale2;
                    if (!whole && !paged_sees(a, see[r], j0 + x * KPL + lane / LPK)) s[r][x] = -INFINITY;
                    top = fmaxf(top, s[r][x]);
                }
#pragma unroll
                for (int d = LPK; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                if (top > m[r]) {                    // the same in all lanes
                    const float by = m[r] == -INFINITY ? 1.f : exp2f(m[r] - top);
                    m[r] = top;
                    l[r] *= by;
#pragma unroll
                    for (int y = 0; y < VPL; ++y) { o[r][y].x *= by; o[r][y].y *= by; o[r][y].z *= by; o[r][y].w *= by; }
                }
                const float ref = m[r] == -INFINITY ? 0.f : m[r];
#pragma unroll
                for (int x = 0; x < NL; ++x) {
                    const float p = exp2f(s[r][x] - ref);
                    l[r] += p;
                    // a weight of 0 must not meet what its row does not see
                    if (whole || paged_sees(a, see[r], j0 + x * KPL + lane / LPK)) {
#pragma unroll
                        for (int y = 0; y < VPL; ++y) {
                            o[r][y].x = fmaf(p, v[x][y].x, o[r][y].x);
                            o[r][y].y = fmaf(p, v[x][y].y, o[r][y].y);
                            o[r][y].z = fmaf(p, v[x][y].z, o[r][y].z);
                            o[r][y].w = fmaf(p, v[x][y].w, o[r][y].w);
                        }
                    }
                }
            }
            if (i + 1 < to) fetch(1, i + 1, v);
        }
        // the slots of a load, then the warps
#pragma unroll
        for (int r = 0; r < R; ++r) {
#pragma unroll
            for (int d = LPK; d < 32; d <<= 1) {
                l[r] += __shfl_xor_sync(0xffffffffu, l[r], d);
#pragma unroll
                for (int y = 0; y < VPL; ++y) {
                    o[r][y].x += __shfl_xor_sync(0xffffffffu, o[r][y].x, d);
                    o[r][y].y += __shfl_xor_sync(0xffffffffu, o[r][y].y, d);
                    o[r][y].z += __shfl_xor_sync(0xffffffffu, o[r][y].z, d);
                    o[r][y].w += __shfl_xor_sync(0xffffffffu, o[r][y].w, d);
                }
            }
            float* out = outs + (warp * R + r) * D + d0;
            if (i0 > from) {
                const float2 kept = stats[warp * R + r];
                const float by = kept.x == -INFINITY ? 0.f : exp2f(kept.x - m[r]);
                l[r] = fmaf(kept.y, by, l[r]);
#pragma unroll
                for (int y = 0; y < VPL; ++y) {
                    const float4 x = *reinterpret_cast<const float4*>(out + y * 128);
                    o[r][y] = make_float4(fmaf(x.x, by, o[r][y].x), fmaf(x.y, by, o[r][y].y), fmaf(x.z, by, o[r][y].z), fmaf(x.w, by, o[r][y].w));
                }
                __syncwarp();
            }
            if (lane < LPK) {
#pragma unroll
                for (int y = 0; y < VPL; ++y) *reinterpret_cast<float4*>(out + y * 128) = o[r][y];
            }
            if (lane == 0) stats[warp * R + r] = make_float2(m[r], l[r]);
        }
        if (end >= to) break;
        __syncwarp();
        }
        __syncthreads();
        const bool head = from == 0, tail = to == w.t.count;
        const size_t slot = (size_t)blockIdx.x * 2 + (head ? 1 : 0);
        for (int x = tid; x < rows * (D / 4); x += kRowsThreads) {
            const int r = x / (D / 4), d = x % (D / 4) * 4;
            float top = -INFINITY, sum = 0.f;
#pragma unroll
            for (int y = 0; y < kRowsWarps; ++y) top = fmaxf(top, stats[y * R + r].x);
            const float ref = top == -INFINITY ? 0.f : top;
            float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int y = 0; y < kRowsWarps; ++y) {
                const float2 st = stats[y * R + r];
                const float f = exp2f(st.x - ref);
                sum = fmaf(st.y, f, sum);
                if (st.x == -INFINITY) continue;
                const float4 part = *reinterpret_cast<const float4*>(outs + (y * R + r) * D + d);
                t.x = fmaf(part.x, f, t.x);
                t.y = fmaf(part.y, f, t.y);
                t.z = fmaf(part.z, f, t.z);
                t.w = fmaf(part.w, f, t.w);
            }
            if (head && tail) {
                const bool sees = paged_sees_some(a, paged_row(a, w.s, r0 + r));
                const float4 y = sees ? make_float4(t.x / sum, t.y / sum, t.z / sum, t.w / sum) : make_float4(0.f, 0.f, 0.f, 0.f);
                *reinterpret_cast<float4*>(reinterpret_cast<float*>(a.out) + paged_row_offset(a, w.s, w.h, r0 + r, a.ld_out) + d) = y;
            } else {
                *reinterpret_cast<float4*>(a.part_o + slot * R * D + (d * R + r * 4)) = t;
                if (d == 0) a.part_ml[slot * R + r] = make_float2(top, sum);
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

template <int D, int R>
static coreinfer_status launch_rows(const PagedAttnArgs& a, const DeviceInfo& di, cudaStream_t st)
{
    const size_t smem = (size_t)kRowsWarps * R * (D * sizeof(float) + sizeof(float2)) + paged_list_bytes(a.c.B);
    const coreinfer_status s = allow_smem<paged_rows_kernel<D, R>>(di, 0);
    if (s != COREINFER_OK) return s;
    CI_CUDA(launch_overlapped(paged_rows_kernel<D, R>, dim3(a.n_ctas), dim3(kRowsThreads), smem, st, a));
    return COREINFER_OK;
}
template <int D>
static coreinfer_status rows_count(const PagedAttnArgs& a, const DeviceInfo& di, cudaStream_t st)
{
    return a.RU == 1 ? launch_rows<D, 1>(a, di, st) : launch_rows<D, kPagedRowsMost>(a, di, st);
}

coreinfer_status paged_rows_f32(const PagedAttnArgs& a, const DeviceInfo& di, cudaStream_t st)
{
    if (a.c.D == 64) return rows_count<64>(a, di, st);
    return a.c.D == 128 ? rows_count<128>(a, di, st) : rows_count<256>(a, di, st);
}

}  // namespace coreinfer
